// few_grads.h - both gradients of a few rows, dX = dS W and dW = dS^T X, in one pass over the weight.
//
// With few rows (up to 64 in bf16, 128 in f32) both contractions are as large as the weight: W is read once, dW written once, and nothing else is of any size; in f32 the
// matrix unit bounds more than 48.
// A wavefront takes 16 NB columns of W and a run of its rows, 32 (bf16) or 16 (f32) at a time, straight from memory into registers: the lane that loads eight (four)
// consecutive columns of a row owns them as one column of each of eight (four) matrix blocks - which column of W a block's column is, is free to choose - so that the pieces of
// a step are the operands of dX after a transpose of 8 x 8 values inside the lane (bf16), or as they are (f32).  Nothing passes through LDS and no
// wavefront waits for another; the loads of the next two steps are out while a step is computed.  dW's blocks are laid such that a lane ends with
// sixteen bytes of a row, and lane pairs exchange halves, so that a store writes whole lines.  dX is a sum over all rows of W: few_dx_kernel adds the runs'.
// us of the pair of contractions, and here (TB/s of W and dW): 61 rows, H 2048, V 32000 86 and 67 (3.9); 36, 5120, 50257 357 and 233 (4.4); 20, 3584, 152064 679 and 444 (4.9);
// 3, 3584, 126849 579 and 355 (5.1); f32 4 rows, 2048, 152064 1636 and 443 (5.6); 48 rows, 3584, 152064 3070 and 1120 (3.9);
// 64 and 128 rows 3110 and 1350, 3570 and 2620, 103 and 107 TF of the 152 that a large product reaches.
// dS is wanted in the order of both operands, and small: few_ds_kernel writes two copies.  The wavefronts of a workgroup take the same run and
// neighbouring columns, so that they find its dS in their L1.
#pragma once
#include "epilogues.h"

namespace rlk {

// Rows whose gradients these kernels take, by type.  bf16: more come as fast from the pair of contractions, whose tiles of 256 rows they fill better (us, pair and here: 100 rows, H 3584,
// V 152064 685 and 691, 128 rows, H 1024, V 50000 68 and 74 with eight blocks of 16 tokens).  f32: eight blocks are what the registers hold; 128 rows, H 5120, V 151936 take 5100 and 3880,
// H 2648, V 32000 580 and 430, H 512, V 1000 35 and 28.
constexpr int kFewGradRows = 64, kFewGradRowsF32 = 128;
constexpr int kFewSplits = 256;          // runs of the vocabulary, at most

struct FewGrads {
  const void* W; const void* X; int V, H;
  const int* x_rows; const int* n_real;  // [compact row] its row of X (-1: one of zeros)
  const void* ds1;                       // bf16 [V / 32][tokens][32], f32 [V / 16][tokens][16]
  const void* ds2;                       // [V][tokens rounded up to 32 (bf16)]
  void* dW;
  float* part;                           // [splits][tokens][H]
  int splits, steps;                     // runs of the vocabulary; steps of a wavefront
};
// Elements of a row of the second copy
template <class T> constexpr int few_pitch(int nt) { return sizeof(T) == 2 && nt == 1 ? 32 : nt * 16; }
template <class T> constexpr int few_step() { return sizeof(T) == 2 ? 32 : 16; }

// A run's dX, to the partial buffer.  acc: [token block][column block]; column of block j, lane n: NB n + j.
template <int NT, int NB>
__device__ __attribute__((always_inline)) inline void few_dx_out(const floatx4 (&acc)[NT][NB], const FewGrads& j, int split, int h0) {
  constexpr int PER = NB < 4 ? NB : 4;
  typedef float piece __attribute__((ext_vector_type(PER)));
  const int lane = threadIdx.x & 63, g = lane >> 4, h = h0 + (lane & 15) * NB;
#pragma unroll
  for (int b = 0; b < NT; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < NB; q += PER) {
        piece v;
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = acc[b][q + e][i];
        if (h + q < j.H) *reinterpret_cast<piece*>(j.part + ((int64_t)split * 16 * NT + b * 16 + g * 4 + i) * j.H + h + q) = v;       // (H % 4 == 0)
      }
}

// Sixteen bytes of a row, where the row starts at any element; whole lines in non-temporal stores
template <class V, class T>
__device__ __attribute__((always_inline)) inline void few_store(T* p, const V& v, bool lines) {
  typedef unsigned any16 __attribute__((ext_vector_type(4), aligned(2)));
  if (lines) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t*>(p));
  else *reinterpret_cast<any16*>(p) = __builtin_bit_cast(u32x4_t, v);
}

// steps [first, last), the loads of the next DEPTH - 1 on their way
constexpr int kFewGradStages = 3;
template <class S, int DEPTH, class LOAD, class COMPUTE>
__device__ __attribute__((always_inline)) inline void few_walk(int first, int last, LOAD load, COMPUTE compute) {
  if (first >= last) return;
  S s[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH - 1; ++i) load(s[i], first + i);
  for (int step = first; step < last; step += DEPTH) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      if (step + i < last) {
        load(s[(i + DEPTH - 1) % DEPTH], step + i + DEPTH - 1);
        compute(s[i], step + i);
      }
    }
  }
}

// TO: type of dW.  grid: columns x splits.
template <int NT, class TO>
__global__ __launch_bounds__(256, 1) void few_grads_bf16_kernel(FewGrads j) {
  constexpr int NB = 8, T = 16 * NT, P = few_pitch<bf16_t>(NT), KS = P / 32, HW = 16 * NB;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, n = lane & 15, odd = n & 1;
  const int hs = (j.H + HW - 1) / HW, waves = blockDim.x >> 6, cols = (hs + waves - 1) / waves, split = (int)blockIdx.x / cols;
  const int h0 = ((int)blockIdx.x % cols * waves + w) * HW;
  if (h0 >= j.H) return;
  const int rows = *j.n_real;
  const bf16_t* X = static_cast<const bf16_t*>(j.X);
  TO* dW = static_cast<TO*>(j.dW);
  const bool lines = (int64_t)j.H * sizeof(TO) % 128 == 0 && (reinterpret_cast<uintptr_t>(dW) & 127) == 0;

  // X^T: block k, row m of it is column 32 (k / 2) + 8 (m / 4) + 4 (k % 2) + m % 4
  bf16x8 x[KS][NB];
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = s * 32 + g * 8 + i;
      const int row = t < rows ? j.x_rows[t] : -1;
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        const int h = h0 + 32 * (k >> 1) + 8 * (n >> 2) + 4 * (k & 1) + (n & 3);
        x[s][k][i] = row >= 0 && h < j.H ? X[(int64_t)row * j.H + h] : (bf16_t)0.f;
      }
    }

  typedef unsigned piece __attribute__((ext_vector_type(NB / 2)));      // NB columns of a row
  const int hl = h0 + n * NB < j.H ? h0 + n * NB : j.H - NB;           // (H % 8 == 0; what is loaded past the last column is not stored)
  const bf16_t* Wl = static_cast<const bf16_t*>(j.W) + hl;
  const uint4* d1 = static_cast<const uint4*>(j.ds1);
  const uint4* d2 = static_cast<const uint4*>(j.ds2);
  const int first = split * j.steps, all = (j.V + 31) / 32;
  const int last = first + j.steps < all ? first + j.steps : all;
  floatx4 acc[NT][NB];
#pragma unroll
  for (int b = 0; b < NT; ++b)
#pragma unroll
    for (int k = 0; k < NB; ++k) acc[b][k] = floatx4{0.f, 0.f, 0.f, 0.f};

  struct Step { piece w[8]; uint4 a[NT], b[2][KS]; };
  auto load = [&](Step& s, int step) __attribute__((always_inline)) {
    step = step < last ? step : last - 1;                               // (past the end: loaded again, not used)
    const int v0 = step * 32;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int v = v0 + g * 8 + i;
      s.w[i] = *reinterpret_cast<const piece*>(Wl + (int64_t)(v < j.V ? v : j.V - 1) * j.H);
    }
#pragma unroll
    for (int b = 0; b < NT; ++b) s.a[b] = d1[((int64_t)step * T + b * 16 + n) * 4 + g];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int q = 0; q < KS; ++q) s.b[u][q] = d2[(int64_t)(v0 + u * 16 + n) * (P / 8) + q * 4 + g];
  };
  auto compute = [&](const Step& s, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < NB; ++k) {                                      // dX: the lane's column k of its eight rows
      u32x4_t f;
#pragma unroll
      for (int d = 0; d < 4; ++d) f[d] = __builtin_amdgcn_perm(s.w[2 * d + 1][k >> 1], s.w[2 * d][k >> 1], k & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int b = 0; b < NT; ++b)
        acc[b][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, s.a[b]), __builtin_bit_cast(bf16x8, f), acc[b][k], 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {                                       // dW: sixteen rows, lane n has row n
      floatx4 d[NB];
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        d[k] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < KS; ++q) d[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[q][k], __builtin_bit_cast(bf16x8, s.b[u][q]), d[k], 0, 0, 0);
      }
      const int v = step * 32 + u * 16 + n;
      if constexpr (sizeof(TO) == 2) {
#pragma unroll
        for (int k = 0; k < NB / 4; ++k) {                              // 64 columns: a line
          u32x4_t h[2], other;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (bf16_t)d[4 * k + 2 * q + (e >> 2)][e & 3];
            h[q] = __builtin_bit_cast(u32x4_t, o);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) other[e] = (unsigned)__builtin_amdgcn_mov_dpp((int)(odd ? h[0][e] : h[1][e]), 0xB1, 0xF, 0xF, true);
          const int at = h0 + k * 64 + odd * 32 + g * 8;
          if (at >= j.H) continue;
          if ((v & ~1) < j.V) few_store(dW + (int64_t)(v & ~1) * j.H + at, odd ? other : h[0], lines);
          if ((v | 1) < j.V) few_store(dW + (int64_t)(v | 1) * j.H + at, odd ? h[1] : other, lines);
        }
      } else {
        if (v >= j.V) continue;
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          const int at = h0 + 32 * (k >> 1) + 8 * g + 4 * (k & 1);
          if (at < j.H) few_store(dW + (int64_t)v * j.H + at, d[k], false);
        }
      }
    }
  };
  few_walk<Step, kFewGradStages>(first, last, load, compute);
  few_dx_out<NT, NB>(acc, j, split, h0);
}

// f32: v_mfma_f32_16x16x4, 64 columns of a wavefront, 16 rows of W a step: lane group g loads rows 4 g .. 4 g + 3, and k-step s contracts row s of each group
// (32 columns where there are more than 64 rows: what a wavefront holds of X and dX fits its registers)
constexpr int few_f32_blocks(int nt) { return nt > 4 ? 2 : 4; }
template <int NT>
__global__ __launch_bounds__(256, 1) void few_grads_f32_kernel(FewGrads j) {
  constexpr int T = 16 * NT, NB = few_f32_blocks(NT), HW = 16 * NB;
  typedef float wide __attribute__((ext_vector_type(NB)));
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, n = lane & 15, odd = n & 1;
  const int hs = (j.H + HW - 1) / HW, waves = blockDim.x >> 6, cols = (hs + waves - 1) / waves, split = (int)blockIdx.x / cols;
  const int h0 = ((int)blockIdx.x % cols * waves + w) * HW;
  if (h0 >= j.H) return;
  const int rows = *j.n_real;
  const float* X = static_cast<const float*>(j.X);
  float* dW = static_cast<float*>(j.dW);
  const bool lines = j.H % 32 == 0 && (reinterpret_cast<uintptr_t>(dW) & 127) == 0;

  float x[4 * NT][NB];                                                  // X^T: token 16 b + 4 g + s of k-step (b, s), column 16 k + n
#pragma unroll
  for (int s = 0; s < 4 * NT; ++s) {
    const int t = (s >> 2) * 16 + g * 4 + (s & 3);
    const int row = t < rows ? j.x_rows[t] : -1;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int h = h0 + 16 * k + n;
      x[s][k] = row >= 0 && h < j.H ? X[(int64_t)row * j.H + h] : 0.f;
    }
  }
  const int hl = h0 + n * NB < j.H ? h0 + n * NB : j.H - NB;
  const float* Wl = static_cast<const float*>(j.W) + hl;
  const floatx4* d1 = static_cast<const floatx4*>(j.ds1);
  const floatx4* d2 = static_cast<const floatx4*>(j.ds2);
  const int first = split * j.steps, all = (j.V + 15) / 16;
  const int last = first + j.steps < all ? first + j.steps : all;
  floatx4 acc[NT][NB];
#pragma unroll
  for (int b = 0; b < NT; ++b)
#pragma unroll
    for (int k = 0; k < NB; ++k) acc[b][k] = floatx4{0.f, 0.f, 0.f, 0.f};

  struct Step { wide w[4]; floatx4 a[NT], b[NT]; };
  auto load = [&](Step& s, int step) __attribute__((always_inline)) {
    step = step < last ? step : last - 1;
    const int v0 = step * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int v = v0 + g * 4 + i;
      const wide* p = reinterpret_cast<const wide*>(Wl + (int64_t)(v < j.V ? v : j.V - 1) * j.H);
      if (lines) s.w[i] = __builtin_nontemporal_load(p);                // (otherwise lines are shared with the neighbour: 2 rows, H 4904, V 151936 2340 -> 2130 us)
      else s.w[i] = *p;
    }
#pragma unroll
    for (int b = 0; b < NT; ++b) {
      s.a[b] = d1[((int64_t)step * T + b * 16 + n) * 4 + g];
      s.b[b] = d2[(int64_t)(v0 + n) * (T / 4) + b * 4 + g];
    }
  };
  auto compute = [&](const Step& s, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int b = 0; b < NT; ++b) acc[b][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(s.a[b][i], s.w[i][k], acc[b][k], 0, 0, 0);
    floatx4 d[NB];
#pragma unroll
    for (int k = 0; k < NB; ++k) d[k] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4 * NT; ++q)
#pragma unroll
      for (int k = 0; k < NB; ++k) d[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[q][k], s.b[q >> 2][q & 3], d[k], 0, 0, 0);
    const int v = step * 16 + n;
#pragma unroll
    for (int k = 0; k < NB / 2; ++k) {                                  // 32 columns: a line
      floatx4 other;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        other[e] = __uint_as_float((unsigned)__builtin_amdgcn_mov_dpp((int)__float_as_uint(odd ? d[2 * k][e] : d[2 * k + 1][e]), 0xB1, 0xF, 0xF, true));
      const int at = h0 + k * 32 + odd * 16 + g * 4;
      if (at >= j.H) continue;
      if ((v & ~1) < j.V) few_store(dW + (int64_t)(v & ~1) * j.H + at, odd ? other : d[2 * k], lines);
      if ((v | 1) < j.V) few_store(dW + (int64_t)(v | 1) * j.H + at, odd ? d[2 * k + 1] : other, lines);
    }
  };
  few_walk<Step, kFewGradStages>(first, last, load, compute);
  few_dx_out<NT, NB>(acc, j, split, h0);
}

// dX: the runs' sums added in a fixed order, to the rows that count, 0 to those without entries (x_rows < 0) whatever W holds: 64 columns of a row by a workgroup, thread (q, k) = (i % 16, i / 16) adds up runs k, k + 16, ... of four of them
template <class T>
__global__ __launch_bounds__(256) void few_dx_kernel(const float* part, int splits, int tokens, const int* row_map, const int* x_rows, const int* n_real, int H, T* dX) {
  __shared__ floatx4 sum[16][16];
  const int hb = (H + 63) / 64, t = (int)blockIdx.x / hb, q = threadIdx.x & 15, k = threadIdx.x >> 4, h = ((int)blockIdx.x % hb) * 64 + q * 4;
  if (t >= *n_real) return;
  floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
  if (h < H)
    for (int k0 = k; k0 < splits; k0 += 64) {                             // four loads in flight
      floatx4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) if (k0 + 16 * i < splits) v[i] = *reinterpret_cast<const floatx4*>(part + ((int64_t)(k0 + 16 * i) * tokens + t) * H + h);
#pragma unroll
      for (int i = 0; i < 4; ++i) if (k0 + 16 * i < splits) s += v[i];
    }
  sum[k][q] = s;
  __syncthreads();
  if (k || h >= H) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += sum[i][q];
  T* o = dX + (int64_t)row_map[t] * H + h;
  const bool empty = x_rows[t] < 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = empty ? (T)0.f : (T)s[e];
}

}  // namespace rlk
