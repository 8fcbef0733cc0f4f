// f8_grad.h - the weight gradient out of an 8-bit checkpoint:  dW[n, k] = sum_t dy[t, n] x[t, k],  x in 8-bit rows, dy in bf16 or f32, dW f32.
//
// The sum runs over tokens while the scales of x run along k, so no 8-bit MFMA can take them.  A restored value is exact in bf16, though (four
// significant bits times a power of two), so that the products of the bf16 MFMA are exact.  The checkpoint is restored, transposed, into the slab-tiled work buffer
// that the hot kernel's A operand is read from (x^T [k][t], zeros past the last token), dy is its K-major B operand as it is stored:
//     C[k, n] = sum_t x^T[k, t] dy[t, n] = dW[n, k],   a lane holding four consecutive k of one row of dW.
// f32 dy goes as three bf16 terms, dy = d0 + d1 + d2 to 2^-24 of it, one contraction over three times the tokens, the smallest term first: each product is exact, and
// three at the rate of the bf16 pipes take a third of the time of one on the f32 pipes.  (Three launches of a third each: 95 us where one takes a fraction, 3001 tokens of 1157 x 1163.)  Tokens are
// taken a chunk at a time.
#pragma once
#include "epilogues.h"
#include "f8_rows.h"

namespace rlk {

constexpr int kGradChunk = 32768;         // tokens restored at a time, with their copies
constexpr int kGradTerms = 3;

// x^T of a chunk: a workgroup restores 64 tokens x 128 k and writes 128 rows of 64 tokens, whole lines.  `pad` tokens in all, a multiple of 128; `copies` of them side by side.
__global__ __launch_bounds__(256) void f8_restore_t_kernel(const uint8_t* codes, const uint8_t* scales, int fmt, int tokens, int Kp, int Ks, bf16_t* xt, int pad, int copies) {
  constexpr int kPitch = 66;              // elements of a row in LDS
  __shared__ bf16_t lds[128 * kPitch];
  const int t0 = blockIdx.x * 64, k0 = blockIdx.y * 128, tid = threadIdx.x, c = (tid & 15) * 8;
  u32x2_t code[4];
  unsigned s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + i * 16 + (tid >> 4);
    code[i] = u32x2_t{0, 0}; s[i] = 127;
    if (t < tokens) { code[i] = *reinterpret_cast<const u32x2_t*>(codes + (int64_t)t * Kp + k0 + c); s[i] = scales[(int64_t)t * Ks + blockIdx.y]; }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v[8];
    f8_restore8(code[i], s[i], fmt, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) lds[(c + e) * kPitch + i * 16 + (tid >> 4)] = (bf16_t)v[e];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = i * 32 + (tid >> 3), t = (tid & 7) * 8;
    const unsigned* p = reinterpret_cast<const unsigned*>(lds + k * kPitch + t);       // (4-byte aligned: the pitch is even)
    const u32x4_t v = {p[0], p[1], p[2], p[3]};
    for (int c = 0; c < copies; ++c) *reinterpret_cast<u32x4_t*>(xt + tiled_index(k0 + k, c * pad + t0 + t, (int64_t)copies * pad)) = v;
  }
}

// dy of a chunk into aligned rows of bf16, `pad` of them with zeros past the last token: as it is, or in three terms of as many rows each, the smallest first.
template <class T>
__global__ __launch_bounds__(256) void f8_grad_terms_kernel(const T* dy, int64_t ld, int tokens, int pad, int N, int Np, bf16_t* out) {
  constexpr int TERMS = sizeof(T) == 4 ? kGradTerms : 1;
  const int chunks = Np / 8;
  const int64_t all = (int64_t)pad * chunks, term = (int64_t)pad * Np;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < all; q += (int64_t)gridDim.x * 256) {
    const int64_t t = q / chunks;
    const int n = (int)(q - t * chunks) * 8;
    const Raw8<T> r = raw_load(dy + t * ld + n, t < tokens ? N - n : 0);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = raw_get(r, e);
#pragma unroll
    for (int k = TERMS - 1; k >= 0; --k) {
      const Raw8<bf16_t> b = raw_make<bf16_t>(v);
      *reinterpret_cast<u32x4_t*>(out + k * term + t * Np + n) = b.v;
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

// Tile of dW^T, written as dW; or a slice's share of it to the workspace, [slice][N][ldw] likewise.
struct EpiF8Grad {
  typedef NoPre Pre;
  template <class L> __device__ Pre preload(const TileCtx&, const GemmDims&) const { return Pre(); }
  static constexpr bool kSwap = false, kSplit = true, kPermute = false, kGatherB = false;
  __device__ void keep_alive() const { dW[0] = 0.f; }
  float* dW; int64_t ldw; int N, K; int accumulate;
  float* part; int64_t ldp;                   // slices: rows of ldp floats

  template <int MB, int NB, bool ACC, bool EDGE>
  __device__ __attribute__((always_inline)) void tile(floatx4 (&acc)[MB][NB], const TileCtx& c, float* out, int64_t ld) const {
    const int col = c.lane & 15, g = c.lane >> 4;
#pragma unroll
    for (int bj = 0; bj < NB; ++bj) {
      const int n = c.n0 + bj * 16 + col;
      float* q = out + (int64_t)n * ld + c.m0 + g * 4;
      floatx4 old[MB];
      if (ACC) {
#pragma unroll
        for (int bi = 0; bi < MB; ++bi) {
          if (!EDGE) old[bi] = *reinterpret_cast<const floatx4_any*>(q + bi * 16);
          else {
#pragma unroll
            for (int e = 0; e < 4; ++e) old[bi][e] = n < N && c.m0 + bi * 16 + g * 4 + e < K ? q[bi * 16 + e] : 0.f;
          }
        }
      }
#pragma unroll
      for (int bi = 0; bi < MB; ++bi) {
        floatx4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = acc_read<true>(acc[bi][bj], e); if (ACC) v[e] += old[bi][e]; }
        if (!EDGE) *reinterpret_cast<floatx4_any*>(q + bi * 16) = v;
        else {
#pragma unroll
          for (int e = 0; e < 4; ++e) if (n < N && c.m0 + bi * 16 + g * 4 + e < K) q[bi * 16 + e] = v[e];
        }
      }
    }
  }
  template <class L, int MB, int NB, int BM, int BN, int WAVES_M, int WAVES_N, bool AGPR>
  __device__ __attribute__((always_inline)) void run(typename L::acc_t (&acc)[MB][NB], const TileCtx& c, unsigned char*, const GemmDims&, const Pre&) const {
    const bool edge = c.m0 + MB * 16 > K || c.n0 + NB * 16 > N;
    if (c.slices > 1) {
      float* p = part + (int64_t)c.slice * N * ldp;
      if (edge) tile<MB, NB, false, true>(acc, c, p, ldp); else tile<MB, NB, false, false>(acc, c, p, ldp);
    } else if (accumulate) {
      if (edge) tile<MB, NB, true, true>(acc, c, dW, ldw); else tile<MB, NB, true, false>(acc, c, dW, ldw);
    } else {
      if (edge) tile<MB, NB, false, true>(acc, c, dW, ldw); else tile<MB, NB, false, false>(acc, c, dW, ldw);
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
