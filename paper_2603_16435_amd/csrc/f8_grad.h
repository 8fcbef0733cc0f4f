// f8_grad.h - the weight gradient out of an 8-bit checkpoint:  dW[n, k] = sum_t dy[t, n] x[t, k],  x in 8-bit rows, dy in bf16 or f32, dW f32.
//
// The sum runs over tokens while the scales of x run along k, so no 8-bit MFMA can take them.  A restored value is exact in bf16, though (four
// significant bits times a power of two), so that the products of the bf16 MFMA are exact.  The checkpoint is restored, transposed, into the slab-tiled work buffer
// that the hot kernel's A operand is read from (x^T [k][t], zeros past the last token), dy is its K-major B operand as it is stored:
//     C[k, n] = sum_t x^T[k, t] dy[t, n] = dW[n, k],   a lane holding four consecutive k of one row of dW.
// f32 dy goes as three bf16 terms, dy = d0 + d1 + d2 to 2^-24 of it (and to 2^-133, where bf16 ends: dy below 2^-109), one contraction over three times the tokens, the smallest term first: each product is exact, and
// three at the rate of the bf16 pipes take a third of the time of one on the f32 pipes.  (32749 tokens of 3584 x 3584 in bf16: 610 us, 1.38 PFLOP/s, and 122 to restore x and pack dy, 5.8 TB/s.)  (Three launches of a third each: 95 us where one takes a fraction, 3001 tokens of 1157 x 1163.)  Tokens are
// taken a chunk at a time.
#pragma once
#include "epilogues.h"
#include "f8_rows.h"

namespace rlk {

constexpr int kGradChunk = 32768;         // tokens restored at a time, with their copies
constexpr int kGradTerms = 3;

// What the two contractions of the backward pass read, in one launch: workgroups [0, pack_blocks) pack dy, the next restore_blocks restore x^T of a chunk, the rest copy dy.
template <class T> struct F8GradPrep {
  const T* dy; int64_t lddy, M; int N; F8Out packed; int pack_blocks;          // all rows of dy
  const uint8_t *codes, *scales; int fmt, tokens, Kp, Ks; bf16_t* xt; int pad, copies, restore_blocks;          // `pad` tokens, a multiple of 128; `copies` of them side by side
  const T* chunk; int Np; bf16_t* terms;                                       // rows of dy of the chunk
};

// A token whose x is not finite counts as nothing where its dy is zero (a masked one): such values are restored as zeros.
// x^T: a workgroup restores 64 tokens x 128 k and writes 128 rows of 64 tokens, whole lines.
template <class T> __device__ __attribute__((always_inline)) inline void f8_restore_t(const F8GradPrep<T>& j, int block, bf16_t* lds) {
  constexpr int kPitch = 66;              // elements of a row in LDS
  const int across = j.pad / 64, kb = block / across, t0 = (block - kb * across) * 64, k0 = kb * 128, tid = threadIdx.x, c = (tid & 15) * 8;
  u32x2_t code[4];
  unsigned s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + i * 16 + (tid >> 4);
    code[i] = u32x2_t{0, 0}; s[i] = 127;
    if (t < j.tokens) { code[i] = *reinterpret_cast<const u32x2_t*>(j.codes + (int64_t)t * j.Kp + k0 + c); s[i] = j.scales[(int64_t)t * j.Ks + kb]; }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v[8];
    f8_restore8(code[i], s[i], j.fmt, v);
    unsigned bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) bad |= __builtin_isfinite(v[e]) ? 0u : 1u;
    if (__any(bad)) {                     // sixteen lanes hold a token's values: they look through its dy
      const int t = t0 + i * 16 + (tid >> 4);
      bad = max_of_16(bad);
      unsigned found = bad ^ 1u;
      for (int n = c; __any(!found && n - c < j.N); n += 128) {
        const Raw8<T> d = raw_load(j.chunk + (int64_t)t * j.lddy + n, t < j.tokens ? j.N - n : 0);
        unsigned any = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) any |= raw_get(d, e) == 0.f ? 0u : 1u;
        found |= max_of_16(any);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = found ? v[e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) lds[(c + e) * kPitch + i * 16 + (tid >> 4)] = (bf16_t)v[e];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = i * 32 + (tid >> 3), t = (tid & 7) * 8;
    const unsigned* p = reinterpret_cast<const unsigned*>(lds + k * kPitch + t);       // (4-byte aligned: the pitch is even)
    const u32x4_t v = {p[0], p[1], p[2], p[3]};
    for (int q = 0; q < j.copies; ++q) *reinterpret_cast<u32x4_t*>(j.xt + tiled_index(k0 + k, q * j.pad + t0 + t, (int64_t)j.copies * j.pad)) = v;
  }
}

// dy of a chunk into aligned rows of bf16, `pad` of them with zeros past the last token: as it is, or in three terms of as many rows each, the smallest first.
template <class T> __device__ __attribute__((always_inline)) inline void f8_grad_terms(const F8GradPrep<T>& j, int block, int blocks) {
  constexpr int TERMS = sizeof(T) == 4 ? kGradTerms : 1;
  const int chunks = j.Np / 8;
  const int64_t all = (int64_t)j.pad * chunks, term = (int64_t)j.pad * j.Np;
  for (int64_t q = (int64_t)block * 256 + threadIdx.x; q < all; q += (int64_t)blocks * 256) {
    const int64_t t = q / chunks;
    const int n = (int)(q - t * chunks) * 8;
    const Raw8<T> r = raw_load(j.chunk + t * j.lddy + n, t < j.tokens ? j.N - n : 0);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = raw_get(r, e);
#pragma unroll
    for (int k = TERMS - 1; k >= 0; --k) {
      float head[8];                                                // (a finite value's first term is finite: what lies between bf16's end and f32's goes to the second)
#pragma unroll
      for (int e = 0; e < 8; ++e) head[e] = TERMS > 1 && k == TERMS - 1 && finite_bits(v[e]) > 0x7f7f0000u ? copysignf(__uint_as_float(0x7f7f0000u), v[e]) : v[e];
      const Raw8<bf16_t> b = raw_make<bf16_t>(head);
      *reinterpret_cast<u32x4_t*>(j.terms + k * term + t * j.Np + n) = b.v;
      if constexpr (TERMS > 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float hi = raw_get(b, e);
          v[e] = __builtin_isfinite(hi) ? v[e] - hi : 0.f;          // exact; what is not finite is in the first term alone
        }
      }
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void f8_grad_prep_kernel(F8GradPrep<T> j) {
  __shared__ bf16_t lds[128 * 66];
  const int b = blockIdx.x;
  if (b < j.pack_blocks) f8_pack_rows(j.dy, j.M, j.lddy, j.N, j.packed, b, j.pack_blocks);
  else if (b < j.pack_blocks + j.restore_blocks) f8_restore_t(j, b - j.pack_blocks, lds);
  else f8_grad_terms(j, b - j.pack_blocks - j.restore_blocks, (int)gridDim.x - j.pack_blocks - j.restore_blocks);
}

// Tile of dW^T, written as dW; or a slice's share of it to the workspace, [slice][N][ldw] likewise.
struct EpiF8Grad {
  typedef NoPre Pre;
  template <class L> __device__ Pre preload(const TileCtx&, const GemmDims&) const { return Pre(); }
  static constexpr bool kSwap = false, kSplit = true, kPermute = false, kGatherB = false;
  __device__ void keep_alive() const { dW[0] = 0.f; }
  float* dW; int64_t ldw; int N, K; int accumulate;
  float* part; int64_t ldp;                   // slices: rows of ldp floats

  // A lane holds four consecutive k of one row of dW in each of two neighbouring blocks, a pair of lanes thus two rows: they swap halves, so that a store writes eight rows
  // in whole lines of 128 bytes instead of sixteen in halves, past the caches (NT) where the rows lie on lines.  256 KB a tile: with few tokens it is what a tile waits for.
  template <int MB, int NB, bool ACC, bool EDGE, bool NT>
  __device__ __attribute__((always_inline)) void tile(floatx4 (&acc)[MB][NB], const TileCtx& c, float* out, int64_t ld) const {
    const int r = c.lane & 15, p = r & 1, k0 = c.m0 + p * 16 + (c.lane >> 4) * 4;
#pragma unroll
    for (int bj = 0; bj < NB; ++bj) {
      const int n = c.n0 + bj * 16 + (r & ~1);                       // the pair's first row
      float* const q[2] = {out + (int64_t)n * ld + k0, out + (int64_t)(n + 1) * ld + k0};
      auto left = [&](int w, int i) __attribute__((always_inline)) { return !EDGE ? 4 : n + w < N ? K - k0 - i * 32 : 0; };
      floatx4 old[2][MB / 2];
      if (ACC) {
#pragma unroll
        for (int i = 0; i < MB / 2; ++i)
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            if (left(w, i) >= 4) old[w][i] = *reinterpret_cast<const floatx4_any*>(q[w] + i * 32);
            else {
#pragma unroll
              for (int e = 0; e < 4; ++e) old[w][i][e] = e < left(w, i) ? q[w][i * 32 + e] : 0.f;
            }
          }
      }
#pragma unroll
      for (int i = 0; i < MB / 2; ++i) {
        floatx4 v[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a = acc_read<true>(acc[2 * i][bj], e), b = acc_read<true>(acc[2 * i + 1][bj], e);
          const float recv = __uint_as_float((unsigned)__builtin_amdgcn_mov_dpp((int)__float_as_uint(p ? a : b), 0xB1, 0xF, 0xF, true));
          v[0][e] = p ? recv : a; v[1][e] = p ? b : recv;
          if (ACC) { v[0][e] += old[0][i][e]; v[1][e] += old[1][i][e]; }
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          if (NT) __builtin_nontemporal_store(v[w], reinterpret_cast<floatx4*>(q[w] + i * 32));
          else if (left(w, i) >= 4) *reinterpret_cast<floatx4_any*>(q[w] + i * 32) = v[w];
          else {
#pragma unroll
            for (int e = 0; e < 3; ++e) if (e < left(w, i)) q[w][i * 32 + e] = v[w][e];
          }
        }
      }
    }
  }
  template <class L, int MB, int NB, int BM, int BN, int WAVES_M, int WAVES_N, bool AGPR>
  __device__ __attribute__((always_inline)) void run(typename L::acc_t (&acc)[MB][NB], const TileCtx& c, unsigned char*, const GemmDims&, const Pre&) const {
    const bool edge = c.m0 + MB * 16 > K || c.n0 + NB * 16 > N;
    if (c.slices > 1) {
      float* p = part + (int64_t)c.slice * N * ldp;
      if (edge) tile<MB, NB, false, true, false>(acc, c, p, ldp); else tile<MB, NB, false, false, false>(acc, c, p, ldp);
    } else if (accumulate) {
      if (edge) tile<MB, NB, true, true, false>(acc, c, dW, ldw); else tile<MB, NB, true, false, false>(acc, c, dW, ldw);
    } else {
      const bool lines = ldw % 32 == 0 && (reinterpret_cast<uintptr_t>(dW) & 127) == 0;
      if (edge) tile<MB, NB, false, true, false>(acc, c, dW, ldw); else if (lines) tile<MB, NB, false, false, true>(acc, c, dW, ldw); else tile<MB, NB, false, false, false>(acc, c, dW, ldw);
    }
  }
};

template <class Tune>
__global__ __launch_bounds__(256)
void f8_grad_kernel(const bf16_t* __restrict__ A, const bf16_t* __restrict__ B, GemmDims d, EpiF8Grad epi) {
  __shared__ __attribute__((aligned(1024))) unsigned char stage0[kHotStageBytes];
  __shared__ __attribute__((aligned(1024))) unsigned char stage1[kHotStageBytes];
  gemm_nt_bf16_tile<EpiF8Grad, Tune, false, true>(A, B, d, epi, blockIdx.x, stage0, stage1);
}

// The slices added in order onto dW.
__global__ __launch_bounds__(256) void f8_grad_slices_kernel(const float* part, int slices, int N, int K, int64_t ldp, float* dW, int64_t ldw, int accumulate) {
  const int k4 = (K + 3) / 4;
  const int64_t all = (int64_t)N * k4, stride = (int64_t)N * ldp;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < all; q += (int64_t)gridDim.x * 256) {
    const int64_t n = q / k4;
    const int k = (int)(q - n * k4) * 4, left = K - k;
    const float* p = part + n * ldp + k;
    floatx4 s = *reinterpret_cast<const floatx4*>(p);
    for (int i0 = 1; i0 < slices; i0 += 4) {
      floatx4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = i0 + i < slices ? *reinterpret_cast<const floatx4*>(p + (i0 + i) * stride) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) s += v[i];
    }
    float* o = dW + n * ldw + k;
#pragma unroll
    for (int e = 0; e < 4; ++e) if (e < left) o[e] = accumulate ? o[e] + s[e] : s[e];
  }
}

}  // namespace rlk
