// distill.h - scoring with top alternatives, and distillation from a teacher's top entries: kernels and C ABI of include/rl_distill.h.
//
// Both keep a chunk's logits in f32, and beside them a record of every 64 vocabulary entries of a token, made where the logits are in registers:
// their maximum and softmax sums.  A record is 1/16 of what it stands for, and nearly everything after the contraction is answered from the records:
//  * logsumexp and entropy are sums over them;
//  * the K largest logits of a row lie in the K groups with the largest maxima (ties of maxima to the lower group: K maxima come before any element
//    of another group, in the order by value, then by index), so K of V / 64 groups are read;
//  * the sum over all tokens that a teacher's list does not name is the sum over the groups without a listed token, from their records, and over the
//    others from the logits, with the listed ones left out: never a difference of two sums, which would have no digit left where the list has nearly
//    all of the probability.
// What is read of the logits once more is the whole chunk, by the backward, which turns it into dS in one pass.
//
// Sums: those of a group in f32, of groups in f64, the group of the largest logit once more in f64; each exponential is taken of a difference to the group's or the row's maximum (formed before it is
// scaled), so that what carries the sum carries no error of the shift.
#pragma once
#include "../../include/rl_distill.h"
#include "few_grads.h"

namespace rlk {

constexpr int kDefaultChunkRowsDistill = 16384;   // 10 GB of logits and 5 of dS at the 7B head
constexpr int kMostChunkRows = 1 << 20;           // (launches of a chunk stay below 2^32 threads)
constexpr int kGroup = 64;                        // vocabulary entries of a record

// ------------------------------------------------------------------ logits and records
// Bound by the contraction, whose tile the epilogue ends.  us in turn with the forward that keeps no logits: 5664 rows at the 7B head (H 3584, V 152064) 4660 (1325 TF) and 4236, 10 % behind it, 4099 rows,
// H 5120, V 151936 4667 (1366 TF) and 4350, 7 %: the store of the logits (3.4 GB of f32) and three operations and an exponential for each.
//
// Record of 64 logits of a token, x largest (raw), y sum exp(zs (z - x)), z sum of those times (z - x); w unused.
//
// In what order the 64 are added: bf16 (kPermute, a lane holds eight consecutive entries of each half of the group): the sixteen of a lane in order, then lanes 16
// apart, then 32.  f32, by quads of four consecutive entries Q = 0 .. 15: over bits 2 and 3 of Q in order, then bit 1, then bit 0, which both
// block shapes of the f32 kernels can do: a token's sums do not depend on the tile it is in.
//
// Where the record of group g and token t lies: those of four groups, a tile's 256 entries, are neighbours, so that a row's records are pieces of 64 bytes (a row by
// itself takes a whole line for each piece; with one record a piece the row kernels waited for L2: 4.5 k rows of V 152064 126 us), and a tile's are one piece of memory.
__device__ inline int64_t rec_index(int g, int t, int ldr) { return ((int64_t)(g >> 2) * ldr + t) * 4 + (g & 3); }
template <class T>
struct EpiScore {
  typedef NoPre Pre;
  template <class L> __device__ Pre preload(const TileCtx&, const GemmDims&) const { return Pre(); }
  static constexpr bool kSwap = false;
  static constexpr bool kSplit = false;
  static constexpr bool kPermute = true;
  static constexpr bool kNaturalB = true;
  static constexpr bool kGatherB = true;
  __device__ void keep_alive() const { z[0] = 0.f; }
  float* z; int64_t ldz;      // logits, slab-tiled like the bf16 work buffers: a tile of 256 x 256 is one piece of memory
  float4* rec; int ldr;       // [vocabulary / 256][chunk rows][4]
  int V;
  float zs;                   // inverse temperature

  // sixteen logits of a lane (entries (r / 8) 32 + g 8 + r % 8 of the group), of its token n; even and odd lanes have neighbouring tokens
  template <bool PAD>
  __device__ __attribute__((always_inline)) float4 group16(const float (&v)[16], int g, int vleft) const {
    const float NEG = -__builtin_inff(), c = zs * kLog2e;
    auto in = [&](int r) __attribute__((always_inline)) { return !PAD || (r >> 3) * 32 + g * 8 + (r & 7) < vleft; };
    float mx = NEG, a, b;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, in(r) ? v[r] : NEG);
    lane_pair<16>(mx, a, b); mx = fmaxf(a, b);
    lane_pair<32>(mx, a, b); mx = fmaxf(a, b);
    const float ms = mx == NEG ? 0.f : mx;
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float d = v[r] - ms, e = in(r) ? __builtin_amdgcn_exp2f(d * c) : 0.f;
      s += e;
      u = in(r) ? __builtin_fmaf(e, d, u) : u;
    }
    lane_pair<16>(s, a, b); s = a + b;
    lane_pair<32>(s, a, b); s = a + b;
    lane_pair<16>(u, a, b); u = a + b;
    lane_pair<32>(u, a, b); u = a + b;
    return make_float4(mx, s, u, 0.f);
  }

  // MB = 8 block rows (128 permuted rows) of NB columns.  A lane has eight consecutive entries of its token, two quads; lanes eight apart exchange one each, so that a store writes whole lines
  // of 128 bytes, those of eight neighbouring tokens.  (Tokens eight and more apart, as with permuted columns, lie 2 KiB and more apart and meet the same memory channels:
  // 16 k rows at the 7B head 13.33 ms.)
  template <int MB, int NB, bool AGPR>
  __device__ __attribute__((always_inline)) void permuted(floatx4 (&acc)[MB][NB], const TileCtx& c) const {
    static_assert(MB == 8, "128 rows");
    const int g = c.lane >> 4, p = (c.lane >> 3) & 1;
    const int vleft = V - c.m0;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int bj = 0; bj < NB; ++bj) {
        float v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = acc_read<AGPR>(acc[4 * j + (r >> 2)][bj], r & 3);
        const int n = c.n0 + bj * 16 + (c.lane & 15), lo = n - 8 * p, hi = lo + 8;
        const float4 q = vleft < j * 64 + 64 ? group16<true>(v, g, vleft - j * 64) : group16<false>(v, g, 64);
        if (g == (NB >= 4 ? bj / (NB / 4) : bj) && n < c.Nv) rec[rec_index(c.m0 / kGroup + j, n, ldr)] = q;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          floatx4 a, b;                                             // the lower lane's token, the upper lane's
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int x = (int)__float_as_uint(v[h * 8 + e]), y = (int)__float_as_uint(v[h * 8 + 4 + e]);
            a[e] = __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(x, y, 0x128, 0xF, 0xC, false));       // upper lanes: the lower's second quad
            b[e] = __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(y, x, 0x128, 0xF, 0x3, false));       // lower lanes: the upper's first
          }
          const int at = c.m0 + j * 64 + h * 32 + g * 8 + p * 4;
          if (lo < c.Nv) __builtin_nontemporal_store(a, reinterpret_cast<floatx4*>(z + tiled_index(lo, at, ldz)));
          if (hi < c.Nv) __builtin_nontemporal_store(b, reinterpret_cast<floatx4*>(z + tiled_index(hi, at, ldz)));
        }
      }
  }

  // general and f32 kernels: rows in their natural order
  template <class L, int MB, int NB>
  __device__ __attribute__((always_inline)) void natural(typename L::acc_t (&acc)[MB][NB], const TileCtx& c) const {
    constexpr int PER = kGroup / L::kBlk;                        // blocks of a group
    static_assert(MB % PER == 0, "a wavefront has whole groups");
    const float NEG = -__builtin_inff(), cs = zs * kLog2e;
#pragma unroll
    for (int bj = 0; bj < NB; ++bj) {
      const int n = c.n0 + L::col(bj, c.lane);
#pragma unroll
      for (int k = 0; k < MB / PER; ++k) {
        const int vleft = V - c.m0 - k * kGroup;
        float mx = NEG, a, b;
        auto in = [&](int bi, int i) __attribute__((always_inline)) { return L::row(bi, i, c.lane) < vleft; };
#pragma unroll
        for (int bi = 0; bi < PER; ++bi)
#pragma unroll
          for (int i = 0; i < L::kRegs; ++i) mx = fmaxf(mx, in(bi, i) ? acc[k * PER + bi][bj][i] : NEG);
        lane_pair<32>(mx, a, b); mx = fmaxf(a, b);
        if constexpr (L::kBlk == 16) { lane_pair<16>(mx, a, b); mx = fmaxf(a, b); }
        const float ms = mx == NEG ? 0.f : mx;
        float s[2] = {0.f, 0.f}, u[2] = {0.f, 0.f};              // (32 x 32 blocks: by bit 1 of the quad)
#pragma unroll
        for (int bi = 0; bi < PER; ++bi)
#pragma unroll
          for (int i = 0; i < L::kRegs; ++i) {
            const int w = L::kBlk == 32 ? (i >> 2) & 1 : 0;
            const float d = acc[k * PER + bi][bj][i] - ms, e = in(bi, i) ? __builtin_amdgcn_exp2f(d * cs) : 0.f;
            s[w] += e;
            u[w] = in(bi, i) ? __builtin_fmaf(e, d, u[w]) : u[w];
          }
        auto join = [&](float (&x)[2]) __attribute__((always_inline)) {
          float r;
          if constexpr (L::kBlk == 32) { r = x[0] + x[1]; lane_pair<32>(r, a, b); r = a + b; }
          else { lane_pair<32>(x[0], a, b); r = a + b; lane_pair<16>(r, a, b); r = a + b; }
          return r;
        };
        const float S = join(s), U = join(u);
        if (n < c.Nv) {
          if (c.lane < L::kBlk) rec[rec_index(c.m0 / kGroup + k, n, ldr)] = make_float4(mx, S, U, 0.f);
#pragma unroll
          for (int bi = 0; bi < PER; ++bi)
#pragma unroll
            for (int i = 0; i < L::kRegs; i += 4) {
              floatx4 o;
#pragma unroll
              for (int e = 0; e < 4; ++e) o[e] = acc[k * PER + bi][bj][i + e];
              *reinterpret_cast<floatx4*>(z + tiled_index(n, c.m0 + k * kGroup + L::row(bi, i, c.lane), ldz)) = o;
            }
        }
      }
    }
  }

  template <class L, int MB, int NB>
  __device__ __attribute__((always_inline)) void half_tile(typename L::acc_t (&acc)[MB][NB], const TileCtx& c, const int (&)[NB]) const {
    permuted<MB, NB, false>(acc, c);
  }
  template <class L, int MB, int NB, int BM, int BN, int WAVES_M, int WAVES_N, bool AGPR>
  __device__ __attribute__((always_inline)) void run(typename L::acc_t (&acc)[MB][NB], const TileCtx& c, unsigned char*, const GemmDims&, const Pre&) const {
    if constexpr (AGPR) permuted<MB, NB, true>(acc, c);
    else natural<L, MB, NB>(acc, c);
  }
};

// PREP: with the preparation, by workgroup 0; the others work out which rows count for themselves (local_rows).
template <int BN, bool NT, bool PREP>
__global__ __launch_bounds__(256, 1)
void score_few_kernel(const bf16_t* __restrict__ W, const bf16_t* __restrict__ X, GemmDims d, EpiScore<bf16_t> epi, const int* ids_c, SmallPrep s, RowFill f) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[few_lds_bytes<BN>()];
  if constexpr (PREP) {
    if (blockIdx.x == 0) { prep_small<256, kFewTokens>(s, f, AdvJob{}); return; }
    __shared__ LocalRows<kFewTokens> l;
    local_rows<256>(s, l);
    logits_few_tile<BN, NT>(W, X, d, epi, (int)blockIdx.x - 1, l.n, l.rows, l.ids, smem);
  } else {
    const int left = *d.n_real;
    logits_few_tile<BN, NT>(W, X, d, epi, blockIdx.x, left < d.N ? left : d.N, d.b_rows, ids_c, smem);
  }
}

// f32 logits of a few tokens, up to 64.  Bound by reading the weight once, which the tiles of gemm_f32.h, 64 tokens wide, and the narrow ones, which leave most CUs without work where the
// vocabulary is small, are far from (us, TB/s of W: 4 tokens, H 2048, V 152064 366, 3.4; 2 tokens, H 5120, V 32000 216, 3.0; 3 tokens, V 5726 169, 0.7).  A workgroup takes a group of
// 64 vocabulary entries; KS sets of four wavefronts share K, each wavefront 16 entries.  Slabs of 32 k go straight into LDS, as whole lines (loaded into the operands' registers, 64 bytes of a row by
// four lanes, L1 bounds it: 325 us for the first of the three), two ahead of the one computed on; of up to 16 tokens in one set five workgroups fit a CU's LDS (four with the preparation inside), of 32 tokens in four sets or 64 in two one.  v_mfma_f32_16x16x4, lane group g with k = 16 s + 4 g + e of a slab in its
// k-step (s, e).  What the sets found is added in order in LDS, and the record made there.  (The order of a logit's sum is not that of the other f32 kernels: scored with more than 64
// rows, a token's last bit may be another.)
constexpr int kFewF32Stages = 3;
template <int NT, int KS> constexpr int few_f32_lds_bytes() {
  constexpr int stages = KS * kFewF32Stages * (kGroup + 16 * NT) * kSlabBytes, part = KS * kGroup * (16 * NT + 1) * 4;
  return stages > part ? stages : part;
}
template <int NT, int KS, bool STREAM, bool PREP>
__global__ __launch_bounds__(256 * KS) void score_few_f32_kernel(const float* __restrict__ W, const float* __restrict__ X, GemmDims d, EpiScore<float> epi, SmallPrep sp, RowFill f) {
  constexpr int T = 16 * NT, P = T + 1, BK = 32, STAGES = kFewF32Stages, A_BYTES = kGroup * kSlabBytes, STAGE = A_BYTES + T * kSlabBytes, XL = NT < 2 ? 1 : NT / 2, LOADS = 2 + XL;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[few_f32_lds_bytes<NT, KS>()];
  float (*part)[kGroup][P] = reinterpret_cast<float (*)[kGroup][P]>(smem);       // (when the slabs are done with)
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = w & 3, set = w >> 2;
  int rows, group = blockIdx.x;
  if constexpr (PREP) {
    if (blockIdx.x == 0) { prep_small<256 * KS, kFewTokens>(sp, f, AdvJob{}); return; }
    __shared__ LocalRows<kFewTokens> l;
    local_rows<256 * KS>(sp, l);
    rows = l.n; --group;
    d.b_rows = l.rows;
  } else rows = *d.n_real;
  const int K = d.K, v0 = group * kGroup;
  if (rows <= 0) return;
  unsigned char* mine = smem + set * STAGES * STAGE;
  // loads of a slab, eight rows each: sixteen rows of W by a wavefront, a quarter of X's (of 16: by wavefronts 0 and 2, 1 and 3 alike)
  const float* src[LOADS];
  int chunk[LOADS], at[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int to = j < 2 ? r * 16 + j * 8 : (NT == 1 ? r & 1 : r * XL + j - 2) * 8, lr = to + (lane >> 3);
    chunk[j] = (lane & 7) ^ ((lr >> 1) & 7);
    const float* row;
    if (j < 2) row = W + (int64_t)(v0 + lr < d.M ? v0 + lr : d.M - 1) * d.lda;
    else row = X + (int64_t)d.b_rows[lr < rows ? lr : rows - 1] * d.ldb;
    src[j] = row + chunk[j] * 4;
    at[j] = (j < 2 ? 0 : A_BYTES) + to * kSlabBytes;
  }
  const int steps = (K + BK - 1) / BK, per = (steps + KS - 1) / KS, first = set * per, last = first + per < steps ? first + per : steps;
  auto issue = [&](int i) __attribute__((always_inline)) {               // the i-th slab of the set
    const int k = (first + i < steps ? first + i : steps - 1) * BK;       // past the end: a harmless re-load keeps the count of loads
    unsigned char* stage = mine + i % STAGES * STAGE;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const void* p = k + chunk[j] * 4 < K ? (const void*)(src[j] + k) : (const void*)&kZeroChunk;       // (K % 4 == 0)
      const unsigned to = (unsigned)(size_t)(lds_ptr_t)(stage + at[j]);
      if (STREAM && j < 2) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" :: "v"(p), "s"(to) : "memory");
      else load16_to_lds_lanes(p, stage + at[j]);
    }
  };
  floatx4 acc[NT];
#pragma unroll
  for (int b = 0; b < NT; ++b) acc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int frow = lane & 15, fq = lane >> 4, swz = (frow >> 1) & 7;
  __builtin_amdgcn_s_waitcnt(0x0F70);       // vmcnt(0): what was fetched above is not among the loads counted below
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) issue(i);
  constexpr int PEND = (STAGES - 2) * LOADS;
  for (int i = 0; i < per; ++i) {
    __builtin_amdgcn_s_waitcnt(0x0070 | (PEND & 15) | (PEND >> 4) << 14);       // all but the slab behind this one; lgkmcnt(0)
    __syncthreads();                        // ... in every wavefront, and the stage filled next has been read
    issue(i + STAGES - 1);
    const unsigned char* stage = mine + i % STAGES * STAGE;
    if (first + i < last) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int slot = ((s * 4 + fq) ^ swz) << 4;
        const floatx4 a = *reinterpret_cast<const floatx4*>(stage + (r * 16 + frow) * kSlabBytes + slot);
        floatx4 x[NT];
#pragma unroll
        for (int b = 0; b < NT; ++b) x[b] = *reinterpret_cast<const floatx4*>(stage + A_BYTES + (b * 16 + frow) * kSlabBytes + slot);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int b = 0; b < NT; ++b) acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], x[b][e], acc[b], 0, 0, 0);
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0070);       // no load into LDS may be in flight when it gets another use
  __syncthreads();
#pragma unroll
  for (int b = 0; b < NT; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[set][r * 16 + fq * 4 + i][b * 16 + frow] = acc[b][i];
  __syncthreads();
  // logits to memory, a token's 64 in a row; the sums stay in the first set's place
  for (int e = threadIdx.x; e < kGroup * T; e += 256 * KS) {
    const int t = e / kGroup, i = e % kGroup;
    float z = part[0][i][t];
#pragma unroll
    for (int k = 1; k < KS; ++k) z += part[k][i][t];
    part[0][i][t] = z;
    if (t < rows) epi.z[tiled_index(t, v0 + i, epi.ldz)] = z;
  }
  __syncthreads();
  // record: four lanes of a token, sixteen entries each
  const int t = (int)threadIdx.x >> 2, q = threadIdx.x & 3, vleft = epi.V - v0;
  if (t >= rows || t >= T) return;
  const float NEG = -__builtin_inff(), c = epi.zs * kLog2e;
  float z[16], mx = NEG, s = 0.f, u = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) { z[i] = part[0][q * 16 + i][t]; mx = fmaxf(mx, q * 16 + i < vleft ? z[i] : NEG); }
  mx = fmaxf(mx, __shfl_xor(mx, 1)); mx = fmaxf(mx, __shfl_xor(mx, 2));
  const float ms = mx == NEG ? 0.f : mx;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float dd = z[i] - ms, e = __builtin_amdgcn_exp2f(dd * c);
    if (q * 16 + i < vleft) { s += e; u = __builtin_fmaf(e, dd, u); }
  }
  s += __shfl_xor(s, 1); s += __shfl_xor(s, 2);
  u += __shfl_xor(u, 1); u += __shfl_xor(u, 2);
  if (q == 0) epi.rec[rec_index(group, t, epi.ldr)] = make_float4(mx, s, u, 0.f);
}

// ------------------------------------------------------------------ a row, by a workgroup
__device__ inline float wave_max(float v) { for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o)); return v; }

// Order of logits as unsigned numbers: -0 is 0, what is no number comes before everything.
__device__ inline unsigned order_key(float z) {
  const unsigned u = __float_as_uint(z + 0.f);
  return z != z ? 0u : u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ inline float key_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// Sums under a running maximum (raw units, c = log2(e) / temperature).  Not-a-numbers stay in s.
struct Online {
  float m = -__builtin_inff();
  double s = 0.0, u = 0.0;
  __device__ __attribute__((always_inline)) void raise(float mm, float c) {
    if (!(mm > m)) return;
    if (m != -__builtin_inff()) {
      const double f = (double)__builtin_amdgcn_exp2f((m - mm) * c);
      u = f * (u + (double)(m - mm) * s);
      s *= f;
    }
    m = mm;
  }
  __device__ __attribute__((always_inline)) void add(const float4& q, float c) {       // a record with a maximum of at most m
    if (q.x > -__builtin_inff()) {
      const float d = q.x - m, f = __builtin_amdgcn_exp2f(d * c);
      s += (double)f * (double)q.y;
      u += (double)f * ((double)q.z + (double)d * (double)q.y);
    } else if (q.y != q.y) s = __builtin_nan("");
  }
};

constexpr int kTopThreads = 256, kTopWaves = kTopThreads / 64;
constexpr int kTopBatch = 16;           // groups looked at between two looks at how full the list is
constexpr int kTopList = 2048, kTopRoom = kTopList - kTopBatch * kGroup;

struct TopJob {
  const float* z; int64_t ldz; const float4* rec; int ldr, groups, V, K;
  float zs;
  const int *row_map, *ids_c, *cpos;
  const Ctrl* ctrl;
  int chunk_start, chunk_rows;
  int64_t R;
  int row_blocks;                       // workgroups with rows; the rest write what rows that do not count read
  float *logprob, *lse, *entropy; int32_t* ids; float* lp;
};

// Sums over a workgroup, each with one barrier: the next one writes the other half of its words.
struct BlockSum {
  int (*words)[kTopWaves]; int lane, w, flip;
  __device__ __attribute__((always_inline)) int operator()(int of_wave) {
    flip ^= 1;
    if (lane == 0) words[flip][w] = of_wave;
    __syncthreads();
    int c = 0;
#pragma unroll
    for (int i = 0; i < kTopWaves; ++i) c += words[flip][i];
    return c;
  }
};
// The largest x of which `count` says that at least K are no smaller, from its bit `bit` down; done early where exactly K are.  c: how many.
template <class X, class COUNT>
__device__ __attribute__((always_inline)) inline X least_of_best(int bit, int K, int& c, COUNT count) {
  X x = 0;
  for (; bit >= 0 && c != K; --bit) {
    const X cand = x | (X)1 << bit;
    const int n = count(cand);
    if (n >= K) { x = cand; c = n; }
  }
  return x;
}

// The group of the largest logit m is added once more, logit by logit in f64: beside the largest's 1 an f32 sum keeps nothing of what a nearly certain token leaves to the others, and its entropy,
// its log-probability and the gradient of a list that names it are just that.  A wavefront's first such group, -1 where it has none (of equal ones in several wavefronts each its own; there the 1s say all).
template <int REG>
__device__ __attribute__((always_inline)) inline int top_group(const float4 (&q)[REG], float m, int w) {
  int top = -1;
#pragma unroll
  for (int i = 0; i < REG; ++i) {
    const unsigned long long at = __ballot(m > -__builtin_inff() && q[i].x == m);
    if (at && top < 0) top = i * kTopThreads + w * 64 + __builtin_ctzll(at);
  }
  return top;
}

// A row by a workgroup of 256: every thread holds up to REG records.  Bound by the latency of a chain of short steps, so a row is spread over a
// workgroup and its records are read once; neighbouring rows, which share the records' lines, go to one XCD.  Where maxima or logits are equal the lower index is
// the better one: a second search, over the index, parts the groups, and candidates are pairs (key, token) that are all different.
// 5.7 k rows, V 152064, K 20 108 us (the records alone 215 MB, 2.0 TB/s; 114 with six workgroups a CU instead of seven, which the part for logits of -inf takes where it may), 4.1 k rows,
// K 128 135; one row 17, 48 rows of V 32000 10.
template <int REG>
__global__ __launch_bounds__(kTopThreads, REG <= 10 ? 7 : 2) void top_kernel(TopJob j) {
  __shared__ float red_m[kTopWaves];
  __shared__ double red_s[kTopWaves], red_u[kTopWaves];
  __shared__ int words[2][kTopWaves];
  __shared__ int n_sel, n_list;
  __shared__ int sel[RL_TOP_MAX_K];
  __shared__ unsigned long long list[kTopList];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  if ((int)blockIdx.x >= j.row_blocks) {
    const int64_t step = (int64_t)(gridDim.x - j.row_blocks) * kTopWaves;
    for (int64_t r = (int64_t)(blockIdx.x - j.row_blocks) * kTopWaves + w; r < j.R; r += step) {
      if (j.cpos[r] >= 0) continue;
      for (int k = lane; k < j.K; k += 64) {
        if (j.ids) j.ids[r * j.K + k] = -1;
        if (j.lp) j.lp[r * j.K + k] = 0.f;
      }
    }
    return;
  }
  int left = j.ctrl->n_real - j.chunk_start, t;
  left = left < j.chunk_rows ? left : j.chunk_rows;
  if (left <= 0 || !run_of_block(blockIdx.x, left, t)) return;
  const float c = j.zs * kLog2e, NEG = -__builtin_inff();
  const int tg = j.chunk_start + t, row = j.row_map[tg], K = j.K;
  const float zy = j.logprob ? j.z[tiled_index(t, j.ids_c[tg], j.ldz)] : 0.f;

  float4 q[REG];
  float m = NEG;
#pragma unroll
  for (int i = 0; i < REG; ++i) {
    const int b = i * kTopThreads + tid;
    q[i] = make_float4(NEG, 0.f, 0.f, 0.f);
    if (b < j.groups) q[i] = j.rec[rec_index(b, t, j.ldr)];
  }
#pragma unroll
  for (int i = 0; i < REG; ++i) m = fmaxf(m, q[i].x);
  m = wave_max(m);
  if (lane == 0) red_m[w] = m;
  if (tid == 0) { n_sel = 0; n_list = 0; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kTopWaves; ++i) m = fmaxf(m, red_m[i]);
  double s = 0.0, u = 0.0;
  const int top = top_group(q, m, w);
  const float zt = top >= 0 && top * kGroup + lane < j.V ? j.z[tiled_index(t, top * kGroup + lane, j.ldz)] : NEG;
#pragma unroll
  for (int i = 0; i < REG; ++i) {
    if (i * kTopThreads + tid == top) continue;
    if (q[i].x > NEG) {
      const float d = q[i].x - m, f = __builtin_amdgcn_exp2f(d * c);
      s += (double)f * (double)q[i].y;
      u += (double)f * ((double)q[i].z + (double)d * (double)q[i].y);
    } else if (q[i].y != q[i].y) s = __builtin_nan("");
  }
  if (zt != NEG) { const float d = zt - m; const double e = __builtin_amdgcn_exp2f(d * c); s += e; u += e * (double)d; }
  s = wave_sum(s); u = wave_sum(u);
  if (lane == 0) { red_s[w] = s; red_u[w] = u; }
  __syncthreads();
  s = red_s[0]; u = red_u[0];
#pragma unroll
  for (int i = 1; i < kTopWaves; ++i) { s += red_s[i]; u += red_u[i]; }
  if (u != u && s == s && j.entropy) {
    // A logit, or a difference to the largest, is -inf: e d was 0 times that.  Its probability is 0, and so is its part: the row once more, by its logits.
    u = 0.0;
    for (int v = tid; v < j.V; v += kTopThreads) {
      const float d = j.z[tiled_index(t, v, j.ldz)] - m, e = __builtin_amdgcn_exp2f(d * c);
      if (e > 0.f) u += (double)e * (double)d;
    }
    u = wave_sum(u);
    __syncthreads();                                              // (red_u has been read)
    if (lane == 0) red_u[w] = u;
    __syncthreads();
    u = red_u[0];
#pragma unroll
    for (int i = 1; i < kTopWaves; ++i) u += red_u[i];
  }
  const double ln = log(s);
  if (tid == 0) {
    if (j.lse) j.lse[row] = (float)((double)j.zs * (double)m + ln);
    if (j.logprob) j.logprob[row] = (float)((double)j.zs * ((double)zy - (double)m) - ln);
    if (j.entropy) { const double h = ln - (double)j.zs * u / s; j.entropy[row] = (float)(h < 0.0 ? 0.0 : h); }
  }
  if (!j.ids && !j.lp) return;

  // the groups that hold them
  BlockSum sum{words, lane, w, 0};
  unsigned key[REG];
#pragma unroll
  for (int i = 0; i < REG; ++i) key[i] = order_key(q[i].x);
  auto count = [&](auto f) __attribute__((always_inline)) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < REG; ++i) n += (int)__popcll(__ballot(i * kTopThreads + tid < j.groups && f(key[i], i * kTopThreads + tid)));
    return sum(n);
  };
  unsigned long long least = 0;                                   // pairs below it are not among the K best
  unsigned x = 0;
  int last = j.groups;                                            // of the groups with x itself, those below this one
  if (j.groups > K) {
    int n = j.groups;
    x = least_of_best<unsigned>(31, K, n, [&](unsigned cand) { return count([&](unsigned k, int) { return k >= cand; }); });
    if (n != K) {                                                 // more equal the K-th than there is room for
      const int room = K - count([&](unsigned k, int) { return k > x; });
      last = 0;                                                   // the largest bound with at most `room` below it
      for (int bit = 30 - __builtin_clz(RL_TOP_MAX_V / kGroup); bit >= 0; --bit) {
        const int cand = last | 1 << bit;
        if (count([&](unsigned k, int b) { return k == x && b < cand; }) <= room) last = cand;
      }
    }
    least = (unsigned long long)x << 32;
  }
#pragma unroll
  for (int i = 0; i < REG; ++i) {
    const int b = i * kTopThreads + tid;
    if (b < j.groups && (key[i] > x || (key[i] == x && b < last))) sel[atomicAdd(&n_sel, 1)] = b;
  }
  __syncthreads();
  const int ns = n_sel;

  auto keep_best = [&](int n) {                                   // the best K of n > K pairs, anywhere in the list
    unsigned long long p[kTopList / kTopThreads];
#pragma unroll
    for (int i = 0; i < kTopList / kTopThreads; ++i) p[i] = i * kTopThreads + tid < n ? list[i * kTopThreads + tid] : 0ull;
    least = least_of_best<unsigned long long>(63, K, n, [&](unsigned long long cand) {
      int k = 0;
#pragma unroll
      for (int i = 0; i < kTopList / kTopThreads; ++i) k += (int)__popcll(__ballot(p[i] >= cand));
      return sum(k);
    });
    __syncthreads();
    if (tid == 0) n_list = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTopList / kTopThreads; ++i) if (p[i] >= least) list[atomicAdd(&n_list, 1)] = p[i];
    __syncthreads();
  };
  int n = 0;
  for (int s0 = 0; s0 < ns; s0 += kTopBatch) {
    float z[kTopBatch / kTopWaves];
    int at[kTopBatch / kTopWaves];
#pragma unroll
    for (int k = 0; k < kTopBatch / kTopWaves; ++k) {
      const int i = s0 + k * kTopWaves + w;
      at[k] = sel[i < ns ? i : s0] * kGroup + lane;
      z[k] = j.z[tiled_index(t, at[k], j.ldz)];
      if (i >= ns || at[k] >= j.V) z[k] = __builtin_nanf("");     // (none)
    }
#pragma unroll
    for (int k = 0; k < kTopBatch / kTopWaves; ++k) {
      const unsigned long long p = (unsigned long long)order_key(z[k]) << 32 | (0xffffffffu - (unsigned)at[k]);
      const unsigned long long in = __ballot(z[k] == z[k] && p >= least);
      int base = 0;
      if (lane == 0 && in) base = atomicAdd(&n_list, (int)__popcll(in));
      base = __shfl(base, 0);
      if (in >> lane & 1) list[base + (int)__popcll(in & ((1ull << lane) - 1ull))] = p;
    }
    __syncthreads();
    n = n_list;
    if (n > kTopRoom || (s0 + kTopBatch >= ns && n > 2 * kTopThreads)) { keep_best(n); n = n_list; }
    __syncthreads();
  }

  // in order: each counts those before it
  for (int i = tid; i < n; i += kTopThreads) {
    const unsigned long long p = list[i];
    int rank = 0;
    for (int k = 0; k < n; ++k) rank += list[k] > p;
    if (rank >= K) continue;
    if (j.ids) j.ids[(int64_t)row * K + rank] = (int)(0xffffffffu - (unsigned)p);
    if (j.lp) j.lp[(int64_t)row * K + rank] = (float)((double)j.zs * ((double)key_value((unsigned)(p >> 32)) - (double)m) - ln);
  }
  for (int i = n + tid; i < K; i += kTopThreads) {                // (fewer numbers than K in the row)
    if (j.ids) j.ids[(int64_t)row * K + i] = -1;
    if (j.lp) j.lp[(int64_t)row * K + i] = __builtin_nanf("");
  }
}
static void launch_top(const TopJob& j, unsigned blocks, hipStream_t s) {
  static_assert(RL_TOP_MAX_V <= 32 * kTopThreads * kGroup, "the largest vocabulary's records fit the registers");
  const int reg = (j.groups + kTopThreads - 1) / kTopThreads;
  auto kern = reg <= 2 ? top_kernel<2> : reg <= 4 ? top_kernel<4> : reg <= 10 ? top_kernel<10> : top_kernel<32>;
  kern<<<blocks, kTopThreads, 0, s>>>(j);
}

// ------------------------------------------------------------------ distillation, a row
// What the backward needs of a row: dS = f exp(zs (z - m) - l) at tokens that the list does not name, in log2 units.
struct DistillRow { float m, l2, f, pad; };
struct DistillJob {
  const float* z; int64_t ldz; const float4* rec; int ldr, groups, V, K;
  float zs;
  const int *row_map, *cstart;
  const Ctrl* ctrl;
  int chunk_start, chunk_rows, B;
  const int32_t* t_ids; const float* t_lp;
  int rest, token_mean;
  float scale;
  float *row_loss, *lse;
  double* term;                         // [compact row] this row's part of the loss
  int* info;                            // [compact row] entries left out, bit 30: empty
  int* x_rows;                          // [compact row] its row of hidden states, -1 if empty: a gradient of 0 times what is no number would be none.  NULL without backward
  DistillRow* rows; int* p_ids; float* p_val;          // [chunk row], [chunk row][K]: the tokens that are listed and their dS (-1: none); NULL without backward
};
// Sequence of compact row t: the last i with cstart[i] <= t, 64 at a time.
__device__ inline int sequence_of(const int* cstart, int B, int t, int lane) {
  int lo = 0, n = B;                    // among [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64, i = lane * step;
    const int c = __popcll(__ballot(i < n && cstart[lo + i] <= t)) - 1;
    lo += c * step;
    n = n - c * step < step ? n - c * step : step;
  }
  return lo;
}

// A row by a workgroup, as in top_kernel, and bound as it is; thread i < K has entry i of the list.  3 k rows, V 152064, K 20 52 us, 4.5 k rows, K 64 112.
template <int REG>
__global__ __launch_bounds__(kTopThreads) void distill_row_kernel(DistillJob j) {
  constexpr int kWords = RL_TOP_MAX_V / kGroup / 32;
  __shared__ unsigned bits[kWords];                               // groups with a listed token
  __shared__ int ids[RL_TOP_MAX_K], sel[RL_TOP_MAX_K];            // tokens (-1: none); groups with one, by their first entry
  __shared__ int words[2][kTopWaves];
  __shared__ float red_m[3][kTopWaves];
  __shared__ double red[2][4][kTopWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int left = j.ctrl->n_real - j.chunk_start, t;
  left = left < j.chunk_rows ? left : j.chunk_rows;
  if (left <= 0 || !run_of_block(blockIdx.x, left, t)) return;
  const int tg = j.chunk_start + t, row = j.row_map[tg], K = j.K;
  const float c = j.zs * kLog2e, NEG = -__builtin_inff();
  const bool bucket = j.rest == RL_REST_BUCKET;

  float4 q[REG];
#pragma unroll
  for (int i = 0; i < REG; ++i) {
    const int b = i * kTopThreads + tid;
    q[i] = make_float4(NEG, 0.f, 0.f, 0.f);
    if (b < j.groups) q[i] = j.rec[rec_index(b, t, j.ldr)];
  }
  double share = 0.0;                                             // (wavefronts 0 and 1, as all that is asked of entries)
  if (w < 2) {
    if (j.token_mean) share = 1.0 / (double)j.ctrl->n_real;
    else {
      const int i = sequence_of(j.cstart, j.B, tg, lane);
      share = 1.0 / ((double)j.B * (double)(j.cstart[i + 1] - j.cstart[i]));
    }
  }
  int id = -1;
  float lp = NEG;
  if (tid < K) { id = j.t_ids[(int64_t)row * K + tid]; lp = j.t_lp[(int64_t)row * K + tid]; }
  bool in = id >= 0 && id < j.V;
  bool out = id != -1 && !in;                                     // left out
  if (tid < RL_TOP_MAX_K) ids[tid] = in ? id : -1;
  for (int b = tid; b < (j.groups + 31) / 32; b += kTopThreads) bits[b] = 0u;
  const float zi = in ? j.z[tiled_index(t, id, j.ldz)] : 0.f;
  __syncthreads();
  bool head = in;                                                 // first of its group
  auto before = [&](int o, bool earlier) __attribute__((always_inline)) {
    if (earlier && o >= 0) {
      if (o == id) { out |= in; in = false; }
      if (o / kGroup == id / kGroup) head = false;
    }
  };
  if (w < 2) {
    const int first = ids[lane], own = w == 0 ? first : ids[64 + lane];
    if (w == 1) for (int i = 0; i < 64; ++i) before(__builtin_amdgcn_readlane(first, i), true);
    for (int i = 0; i < K - w * 64 && i < 64; ++i) before(__builtin_amdgcn_readlane(own, i), i < lane);
  }
  BlockSum count{words, lane, w, 0};
  const unsigned long long heads = __ballot(head);
  // (a word each: entries left out, entries, heads of the first wavefront)
  const int tally = count((int)__popcll(__ballot(out)) | (int)__popcll(__ballot(in)) << 8 | (int)__popcll(heads) << 16);
  const int left_out = tally & 255, ns = tally >> 16;
  const bool empty = (tally >> 8 & 255) == 0;
  if (head) {
    const int at = (int)__popcll(heads & ((1ull << lane) - 1ull)) + (w == 1 ? words[count.flip][0] >> 16 : 0);
    sel[at] = id / kGroup;
    atomicOr(&bits[id / kGroup >> 5], 1u << (id / kGroup & 31));
  }
  __syncthreads();

  // tokens that are not listed, of groups with a listed one: each lane its own running sum
  Online r;
  if (bucket)
    for (int s0 = w; s0 < ns; s0 += 4 * kTopWaves) {
      float z[4];
      int g[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = s0 + k * kTopWaves;
        g[k] = sel[i < ns ? i : s0];
        z[k] = j.z[tiled_index(t, g[k] * kGroup + lane, j.ldz)];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (s0 + k * kTopWaves >= ns) continue;
        unsigned long long named = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int o = ids[h * 64 + lane];
          for (unsigned long long m = __ballot(o >= 0 && o / kGroup == g[k]); m; m &= m - 1) named |= 1ull << (ids[h * 64 + __builtin_ctzll(m)] & 63);
        }
        if (g[k] * kGroup + lane >= j.V || (named >> lane & 1)) continue;
        if (z[k] != z[k]) r.s = __builtin_nan("");
        r.raise(z[k], c);
        r.add(make_float4(z[k], 1.f, 0.f, 0.f), c);
      }
    }
  // and of the others, by their records; all tokens
  bool plain[REG];
  float m = NEG, mr = r.m, ml = wave_max(in ? lp : NEG);
#pragma unroll
  for (int i = 0; i < REG; ++i) {
    const int b = i * kTopThreads + tid;
    plain[i] = bucket && b < j.groups && !(bits[b >> 5] >> (b & 31) & 1u);
    m = fmaxf(m, q[i].x);
    if (plain[i]) mr = fmaxf(mr, q[i].x);
  }
  m = wave_max(m); mr = wave_max(mr);
  if (lane == 0) { red_m[0][w] = m; red_m[1][w] = mr; red_m[2][w] = ml; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kTopWaves; ++i) { m = fmaxf(m, red_m[0][i]); mr = fmaxf(mr, red_m[1][i]); ml = fmaxf(ml, red_m[2][i]); }
  const int top = top_group(q, m, w);
  const float zt = top >= 0 && top * kGroup + lane < j.V ? j.z[tiled_index(t, top * kGroup + lane, j.ldz)] : NEG;
  Online o;
  o.m = m;
  r.raise(mr, c);
#pragma unroll
  for (int i = 0; i < REG; ++i) {
    const int b = i * kTopThreads + tid;
    if (b >= j.groups) continue;
    if (b != top) o.add(q[i], c);
    if (plain[i]) r.add(q[i], c);
  }
  if (zt != NEG) o.s += (double)__builtin_amdgcn_exp2f((zt - m) * c);
  auto sum4 = [&](int half, double (&v)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = wave_sum(v[k]);
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) red[half][k][w] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = red[half][k][0];
#pragma unroll
      for (int i = 1; i < kTopWaves; ++i) v[k] += red[half][k][i];
    }
  };
  if (ml == NEG) ml = 0.f;
  const double lt = bucket ? (double)lp : (double)lp - (double)ml;
  double p = in ? exp(lt) : 0.0;                                  // (exact: 1 - sum p may be small)
  double v[4] = {o.s, r.s, p, 0.0};
  sum4(0, v);
  double ln = 0.0, lnr = 0.0, lq = 0.0, q_in = 0.0, lqr = 0.0, P = 0.0, pr = 0.0, part[4] = {0.0, 0.0, 0.0, 0.0};
  if (w < 2) {
    ln = log(v[0]);
    // (q in f64: P q - p of a token that both are nearly certain of is far below either)
    if (in) { lq = (double)j.zs * ((double)zi - (double)m) - ln; q_in = exp(lq); part[1] = q_in; }
    double lnp = 0.0;
    if (bucket) {
      lnr = log(v[1]);
      lqr = (double)j.zs * ((double)mr - (double)m) + lnr - ln;   // log of the others' probability
      pr = 1.0 - v[2]; pr = pr < 0.0 ? 0.0 : pr;
      if (mr == NEG && v[1] == 0.0) pr = 0.0;                     // (the list names all tokens)
      P = v[2] + pr;
    } else if (v[2] != 0.0) {
      lnp = log(v[2]);
      p /= v[2];
      P = 1.0;
    }
    if (p > 0.0 || p != p) part[0] = p * (lt - lnp - lq);
  }
  sum4(1, part);
  if (w >= 2) return;
  const bool nothing = empty || P == 0.0;
  // The others' probability: out of their own sum where they have less than half of it, and 1 less the listed ones' where those have; so it is off by 1e-7 of the smaller, and
  // a list of next to nothing, whose KL is smaller still, is not drowned by it.
  double qr;
  if (part[1] <= 0.5) { qr = 1.0 - part[1]; lqr = log1p(-part[1]); }
  else qr = exp(lqr);
  double kl = part[0];
  if (pr > 0.0) kl += pr * (log(pr) - lqr);
  if (nothing) kl = 0.0;
  const double coef = (double)j.scale * share, f = coef * (double)j.zs;
  if (tid == 0) {
    if (j.lse) j.lse[row] = (float)((double)j.zs * (double)m + ln);
    if (j.row_loss) j.row_loss[row] = (float)kl;
    j.term[tg] = coef * kl;
    j.info[tg] = left_out | (nothing ? 1 << 30 : 0);
  }
  if (!j.rows) return;
  // dS at the others, coef zs q (P - pr / q_r).  With a bucket relative to their own sum, q / q_r (P q_r - pr): nothing overflows where q_r is small
  if (tid == 0) {
    DistillRow d{m, (float)(ln * 1.4426950408889634), nothing ? 0.f : (float)(f * P), 0.f};
    if (pr > 0.0 && !nothing) { d.m = mr; d.l2 = (float)(lnr * 1.4426950408889634); d.f = (float)(f * (P * qr - pr)); }
    j.rows[t] = d;
    j.x_rows[tg] = nothing ? -1 : row;
  }
  if (tid < K) {
    j.p_ids[(int64_t)t * K + tid] = in && !nothing ? id : -1;
    j.p_val[(int64_t)t * K + tid] = (float)(f * (P * q_in - p));
  }
}
static void launch_distill_rows(const DistillJob& j, int64_t rows, hipStream_t s) {
  const int reg = (j.groups + kTopThreads - 1) / kTopThreads;
  auto kern = reg <= 2 ? distill_row_kernel<2> : reg <= 4 ? distill_row_kernel<4> : reg <= 10 ? distill_row_kernel<10> : distill_row_kernel<32>;
  kern<<<(unsigned)((rows + kXcds - 1) / kXcds * kXcds), kTopThreads, 0, s>>>(j);
}

// ------------------------------------------------------------------ dS
__device__ __attribute__((always_inline)) inline float ds_entry(float z, const DistillRow& d, float c) {
  return d.f == 0.f ? 0.f : d.f * __builtin_amdgcn_exp2f((z - d.m) * c - d.l2);
}

struct DsJob { const float* z; int64_t ldz; const DistillRow* rows; const Ctrl* ctrl; int chunk_start, V; float zs; };

// bf16: logits and dS are both slab-tiled, a pass over memory in order; a workgroup takes a slab (256 rows, 64 vocabulary entries).  Rows of a slab without a token become 0,
// as does the padding of the vocabulary.  dS is rounded to bf16, once, by at most 2^-8 of each entry: it is an operand of both contractions, and the matrix unit's rate for f32 operands is a tenth of
// that for bf16; two bf16 terms of each entry would double the two contractions, 60 % of a call.  Both gradients are off by 2.2e-3 to 2.5e-3 of their norm where rounding the exact result gives 1.7e-3.  Bound by memory, six bytes a logit: 4.5 k rows, V 152064 780 us, 5.3 TB/s.
__device__ __attribute__((always_inline)) inline void ds_block(int block, const DsJob& j, bf16_t* dS) {
  const int slabs = (int)(j.ldz / 64), tile = block / slabs, slab = block % slabs;
  const int left = j.ctrl->n_real - j.chunk_start - tile * 256;
  if (left <= 0) return;
  const int64_t at = ((int64_t)tile * slabs + slab) * 16384;
  const int e0 = (threadIdx.x & 7) * 8, v0 = slab * 64 + e0;
  const float c = j.zs * kLog2e;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    floatx4 x[4][2];
    DistillRow d[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int n = (h * 4 + k) * 32 + (threadIdx.x >> 3);
      d[k].f = 0.f;
      x[k][0] = x[k][1] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (n < left) {
        d[k] = j.rows[tile * 256 + n];
        const floatx4* p = reinterpret_cast<const floatx4*>(j.z + at + n * 64 + e0);
        x[k][0] = __builtin_nontemporal_load(p); x[k][1] = __builtin_nontemporal_load(p + 1);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int n = (h * 4 + k) * 32 + (threadIdx.x >> 3);
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = (bf16_t)(v0 + e < j.V ? ds_entry(x[k][e >> 2][e & 3], d[k], c) : 0.f);
      store_stream(dS + at + n * 64 + e0, o);
    }
  }
}

// f32: dS (NULL: not wanted) and dS^T, row-major; 64 rows x 64 vocabulary entries of a workgroup, 16 bytes a lane both ways.  Rows up to the next multiple of 64 become 0.
__device__ __attribute__((always_inline)) inline void ds_f32_block(int block, const DsJob& j, float* dS, int64_t ld_ds, float* dST, int64_t ld_dst, float (&tile)[64][65]) {
  const int vb = (int)(j.ldz / 64), n0 = block / vb * 64, m0 = block % vb * 64;
  const int left = j.ctrl->n_real - j.chunk_start;
  if (n0 >= left) return;
  const int q = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const float c = j.zs * kLog2e;
  floatx4 x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int n = n0 + ty + 16 * k;
    x[k] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (n < left) x[k] = *reinterpret_cast<const floatx4*>(j.z + tiled_index(n, m0 + q * 4, j.ldz));
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = ty + 16 * k, n = n0 + r;
    DistillRow d{0.f, 0.f, 0.f, 0.f};
    if (n < left) d = j.rows[n];
    floatx4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) { o[e] = m0 + q * 4 + e < j.V ? ds_entry(x[k][e], d, c) : 0.f; tile[r][q * 4 + e] = o[e]; }
    if (dS) *reinterpret_cast<floatx4*>(dS + (int64_t)n * ld_ds + m0 + q * 4) = o;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int v = ty + 16 * k;
    floatx4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = tile[q * 4 + e][v];
    *reinterpret_cast<floatx4*>(dST + (int64_t)(m0 + v) * ld_dst + n0 + q * 4) = o;
  }
}

// loss, and the counts: a workgroup, each thread its rows in order
struct FinishJob { const double* term; const int* info; const Ctrl* ctrl; const rl_stats* st; float* loss; rl_distill_stats* out; };
__device__ inline void distill_finish(const FinishJob& j) {
  __shared__ double sh[16];
  __shared__ int cnt[2];
  if (threadIdx.x < 2) cnt[threadIdx.x] = 0;
  __syncthreads();
  const int n = j.ctrl->n_real, step = blockDim.x;
  double s = 0.0;
  int bad = 0, empty = 0;
  for (int i0 = threadIdx.x; i0 < n; i0 += 8 * step) {            // (eight loads in flight)
    double t[8];
    int f[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) { const int i = i0 + k * step; t[k] = i < n ? j.term[i] : 0.0; f[k] = i < n ? j.info[i] : 0; }
#pragma unroll
    for (int k = 0; k < 8; ++k) { s += t[k]; bad += f[k] & 0xffff; empty += f[k] >> 30; }
  }
  s = block_sum(s, sh);
  atomicAdd(&cnt[0], bad); atomicAdd(&cnt[1], empty);
  __syncthreads();
  if (threadIdx.x == 0) {
    j.loss[0] = (float)s;
    if (j.out) *j.out = rl_distill_stats{n, cnt[0], cnt[1], j.st->n_bad_seq};
  }
}
__global__ __launch_bounds__(1024) void distill_finish_kernel(FinishJob j) { distill_finish(j); }

// dS of a chunk, and beside it what else is wanted by then: X^T, in the first chunk's launch the rows of dX that do not count as 0, in the last one's the loss (term != NULL).  Workgroups, in
// this order: the loss, n_ds, n_xt, and the rest.
struct XtJob { const void* x; int64_t R; int H, cols, n_ds, n_xt, fast; const int *x_rows, *cpos; void *xt, *dX; int tc; };
template <class T>
__global__ __launch_bounds__(256) void distill_ds_kernel(DsJob j, T* dS, int64_t ld_ds, T* dST, int64_t ld_dst, XtJob x, FinishJob fin) {
  __shared__ union { float f[64][65]; unsigned b[64][33]; bf16_t h[64][65]; } tile;
  int b = blockIdx.x;
  if (fin.term) {
    if (b == 0) { distill_finish(fin); return; }
    --b;
  }
  if (b < x.n_ds) {
    if constexpr (sizeof(T) == 2) ds_block(b, j, dS); else ds_f32_block(b, j, dS, ld_ds, dST, ld_dst, tile.f);
    return;
  }
  b -= x.n_ds;
  const T* X = static_cast<const T*>(x.x);
  T* XT = static_cast<T*>(x.xt);
  if (b < x.n_xt) {
    const int bx = b % x.cols, by = b / x.cols;
    if constexpr (sizeof(T) == 2) {
      if (x.fast) transpose_bf16_block(bx, by, tile.b, X, x.H, x.tc, x.H, x.x_rows, j.ctrl, j.chunk_start, 1, nullptr, nullptr, XT, x.tc, x.tc);
      else transpose_block(TransposeJob<T>{X, x.H, x.tc, x.H, x.x_rows, j.ctrl, j.chunk_start, 1, nullptr, nullptr, XT, x.tc, x.tc, true}, bx, by, tile.h);
    } else transpose_block(TransposeJob<T>{X, x.H, x.tc, x.H, x.x_rows, j.ctrl, j.chunk_start, 1, nullptr, nullptr, XT, x.tc, x.tc, false}, bx, by, tile.f);
    return;
  }
  b -= x.n_xt;
  const int64_t step = (int64_t)((int)gridDim.x - (fin.term ? 1 : 0) - x.n_ds - x.n_xt) * 4;
  for (int64_t r = (int64_t)b * 4 + (threadIdx.x >> 6); r < x.R; r += step) zero_masked_row(r, x.cpos, static_cast<T*>(x.dX), x.R, x.H);
}

// The same for few rows (few_grads.h): `tokens` rows in two copies, those without a token 0; 64 vocabulary entries of a workgroup, which looks through the rows' lists for them itself (p_ids, p_val, K).
template <class T>
__global__ __launch_bounds__(256) void few_ds_kernel(DsJob j, const int* p_ids, const float* p_val, int K, int tokens, int pitch, T* ds1, T* ds2, XtJob x, FinishJob fin) {
  constexpr int STEP = few_step<T>(), PER = 16 / sizeof(T);
  __shared__ T tile[sizeof(T) == 2 ? kFewGradRows : kFewGradRowsF32][64 + 16 / sizeof(T) / 4];
  int b = blockIdx.x;
  if (fin.term) {
    if (b == 0) { distill_finish(fin); return; }
    --b;
  }
  if (b >= x.n_ds) {
    const int64_t step = (int64_t)((int)gridDim.x - (fin.term ? 1 : 0) - x.n_ds) * 4;
    for (int64_t r = (int64_t)(b - x.n_ds) * 4 + (threadIdx.x >> 6); r < x.R; r += step) zero_masked_row(r, x.cpos, static_cast<T*>(x.dX), x.R, x.H);
    return;
  }
  const int left = j.ctrl->n_real, m = threadIdx.x & 63, v = b * 64 + m;
  const float c = j.zs * kLog2e;
  for (int t0 = threadIdx.x >> 6; t0 < pitch; t0 += 16) {              // (pitch is a multiple of 16; four loads in flight)
    float z[4];
    DistillRow d[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int t = t0 + 4 * k;
      z[k] = 0.f; d[k].f = 0.f;
      if (t < left) { z[k] = j.z[tiled_index(t, v, j.ldz)]; d[k] = j.rows[t]; }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) tile[t0 + 4 * k][m] = (T)(v < j.V ? ds_entry(z[k], d[k], c) : 0.f);
  }
  __syncthreads();
  const int n = (left < tokens ? left : tokens) * K;
  for (int i0 = threadIdx.x; i0 < n; i0 += 8 * 256) {
    int id[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) id[k] = i0 + 256 * k < n ? p_ids[i0 + 256 * k] : -1;
#pragma unroll
    for (int k = 0; k < 8; ++k) if (id[k] >= 0 && id[k] >> 6 == b) tile[(i0 + 256 * k) / K][id[k] & 63] = (T)p_val[i0 + 256 * k];
  }
  __syncthreads();
  typedef T piece __attribute__((ext_vector_type(16 / sizeof(T))));
  const int cols = pitch / PER;
  for (int e = threadIdx.x; e < 64 * cols; e += 256) {
    const int r = e / cols, t0 = e % cols * PER;
    piece o;
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = tile[t0 + i][r];
    *reinterpret_cast<piece*>(ds2 + (int64_t)(b * 64 + r) * pitch + t0) = o;
  }
  for (int e = threadIdx.x; e < tokens * (64 / PER); e += 256) {         // pieces of 64 bytes a token and step
    const int t = e / (64 / PER), m0 = e % (64 / PER) * PER, v0 = b * 64 + m0;
    piece o;
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = tile[t][m0 + i];
    *reinterpret_cast<piece*>(ds1 + ((int64_t)(v0 / STEP) * tokens + t) * STEP + v0 % STEP) = o;
  }
}

// dS of the listed tokens over what the pass wrote there
template <class T>
__global__ __launch_bounds__(256) void distill_patch_kernel(const int* ids, const float* val, int K, const Ctrl* ctrl, int chunk_start, int chunk_rows, T* dS, int64_t ld_ds,
                                                            T* dST, int64_t ld_dst) {
  int left = ctrl->n_real - chunk_start;
  left = left < chunk_rows ? left : chunk_rows;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)left * K) return;
  const int v = ids[i], t = (int)(i / K);
  if (v < 0) return;
  if (dS) dS[operand_index(sizeof(T) == 2, t, v, ld_ds)] = (T)val[i];
  if (sizeof(T) == 4) dST[(int64_t)v * ld_dst + t] = (T)val[i];
}

// ------------------------------------------------------------------ host side
struct HeadPlan {
  Plan p;
  int K, groups;
  int few_nt, few_splits, few_steps;        // few rows (few_grads.h): blocks of 16 tokens (0: not few), runs of the vocabulary, steps of a wavefront
  size_t off_z, off_rec, off_stats, off_term, off_info, off_rows, off_pids, off_pval, off_xrows, off_dw, off_few, total;
};

static int few_cols(int dtype, int nt) { return dtype == RL_BF16 ? 128 : 16 * few_f32_blocks(nt); }       // of a wavefront
// Batches of so few rows that both gradients are one pass over the weight, and their launch: a wavefront on each SIMD (us with 768, 1024, 1536, 2048 wavefronts: 36 rows, H 5120,
// V 50257 266 233 269 242; 3 rows, H 3584, V 126849 368 355 409 358; 61 rows, H 2048, V 32000 69 67 85 85).
static void few_plan(HeadPlan& h) {
  const Plan& p = h.p;
  h.few_nt = 0;
  if (p.R > (p.dtype == RL_BF16 ? kFewGradRows : kFewGradRowsF32)) return;
  const int nt = p.R <= 16 ? 1 : p.R <= 32 ? 2 : p.dtype == RL_BF16 || (p.R > 48 && p.R <= 64) ? 4 : p.R <= 48 ? 3 : p.R <= 96 ? 6 : 8;
  const int cols = few_cols(p.dtype, nt), step = p.dtype == RL_BF16 ? 32 : 16;
  const int hs = (p.H + cols - 1) / cols, all = (p.V + step - 1) / step;
  int splits = 4 * kHotSlots / hs;
  splits = splits < 1 ? 1 : splits > kFewSplits ? kFewSplits : splits;
  h.few_steps = (all + splits - 1) / splits;
  h.few_splits = (all + h.few_steps - 1) / h.few_steps;
  h.few_nt = nt;
}

// (log2(e) / t is what differences of logits are multiplied with: 0 times an infinity is no number)
static bool good_temperature(float t) { return t == 0.f || (t > 0.f && t <= 3.0e38f && 1.f / t * kLog2e <= 3.4028234e38f); }

static rl_status head_plan(const rl_batch* b, int K, int chunk_rows, float temperature, bool bwd, bool distill, bool round_dw, HeadPlan& h) {
  if (!b) return RL_ERR_NULL;
  if (!good_temperature(temperature)) return RL_ERR_RANGE;
  if (chunk_rows < 0) return RL_ERR_SHAPE;
  rl_batch one = *b;
  one.P = 1;
  rl_params prm{};
  prm.chunk_rows = !chunk_rows ? kDefaultChunkRowsDistill : chunk_rows < kMostChunkRows ? chunk_rows : kMostChunkRows;
  prm.temperature = temperature;
  prm.backward_mode = RL_BWD_RECOMPUTE;
  const rl_status st = make_plan(&one, &prm, bwd, h.p);
  if (st != RL_OK) return st;
  if (K < 1 || K > RL_TOP_MAX_K || b->V > RL_TOP_MAX_V) return RL_ERR_SHAPE;
  Plan& p = h.p;
  p.keep = false; p.small_grads = false;
  h.K = K; h.groups = p.Vp / kGroup;
  size_t o = p.total;
  auto take = [&](size_t bytes) { size_t at = o; o += up256(bytes); return at; };
  const size_t tc = (size_t)p.Tc, R = (size_t)p.R;
  h.off_z = take(4 * tc * (size_t)p.Vp);
  h.off_rec = take(sizeof(float4) * tc * (size_t)h.groups);
  h.off_stats = h.off_term = h.off_info = h.off_rows = h.off_pids = h.off_pval = h.off_xrows = h.off_dw = h.off_few = 0;
  h.few_nt = 0;
  if (distill) {
    h.off_stats = take(sizeof(rl_stats));
    h.off_term = take(8 * R); h.off_info = take(4 * R);
    if (bwd) {
      h.off_rows = take(sizeof(DistillRow) * tc);
      h.off_pids = take(4 * tc * (size_t)K); h.off_pval = take(4 * tc * (size_t)K);
      h.off_xrows = take(4 * R);
      few_plan(h);
      if (h.few_nt) h.off_few = take(4 * (size_t)h.few_splits * (size_t)h.few_nt * 16 * (size_t)p.H);
      if (round_dw && p.n_chunks > 1) h.off_dw = take(4 * (size_t)p.V * (size_t)p.H);
    }
  }
  h.total = o;
  return RL_OK;
}

// Outputs that meet an input or one another.
struct Span { const void* p; size_t n; };
static bool overlap(const Span* out, int n_out, const Span* in, int n_in) {
  for (int i = 0; i < n_out; ++i) {
    for (int k = 0; k < n_in; ++k) if (meets(out[i].p, out[i].n, in[k].p, in[k].n)) return true;
    for (int k = 0; k < i; ++k) if (meets(out[i].p, out[i].n, out[k].p, out[k].n)) return true;
  }
  return false;
}

// Whether the logits come from a kernel for few tokens, and whether that does the preparation as well: up to three rounds of workgroups, as few_prepare says.
constexpr int kFewScoreF32 = 64;
static bool few_scores(const rl_batch* b, const Plan& p) {
  if ((reinterpret_cast<uintptr_t>(b->weight) | reinterpret_cast<uintptr_t>(b->hidden)) % 16) return false;
  // bf16: up to 64 tokens always, up to 128 where the hot kernel's tiles fill the chip worse (few_tokens).  us of the hot kernel and here: 3 tokens, H 3584, V 126849 227 and 177, 40 tokens
  // 215 and 165, 100 tokens 216 and 217; 3 tokens, H 5120, V 50257 137 and 106; 60, H 2048, V 100000 130 and 119; 1, H 1024, V 60000 38 and 30.  (Same bits.)
  if (p.dtype == RL_BF16) return p.R <= 64 || (p.R <= kFewTokens && (p.tiles_v + 127) / 128 % 2);
  return p.R <= kFewScoreF32;
}
static PrepJob head_prep(const rl_batch* b, const Plan& p, const Ptrs& q, const rl_outputs& out, hipStream_t s) {
  PrepJob job{};
  run_prep(b, p, q, nullptr, out, AdvJob{}, job, s, few_scores(b, p) && few_prepare(p));
  return job;
}

// Sets of wavefronts of score_few_f32_kernel that share K, where the groups alone do not fill the chip.  us with 1, 2, 4 sets: 3 tokens, H 5120, V 5726 (90 groups) 62 47 44, V 32000 (500) 111 99 104;
// 30 tokens, H 768, V 50257 (786) 45 47 56; 2 tokens, H 216, V 152064 34 41 56; 7 tokens, H 768, V 5462 13.9 12.7 11.7.
static int few_f32_sets(int blocks, int H) { return blocks >= 640 || H < 256 ? 1 : blocks >= 256 || H < 512 ? 2 : 4; }
template <int NT, bool STREAM, bool PREP> static auto few_f32_sets_kernel(int ks) {
  if constexpr (NT == 4) return ks == 1 ? score_few_f32_kernel<NT, 1, STREAM, PREP> : score_few_f32_kernel<NT, 2, STREAM, PREP>;            // (LDS holds two sets of 64 tokens)
  else return ks == 1 ? score_few_f32_kernel<NT, 1, STREAM, PREP> : ks == 2 ? score_few_f32_kernel<NT, 2, STREAM, PREP> : score_few_f32_kernel<NT, 4, STREAM, PREP>;
}
template <bool STREAM, bool PREP> static auto few_f32_kernel(int64_t rows, int ks) {
  return rows <= 16 ? few_f32_sets_kernel<1, STREAM, PREP>(ks) : rows <= 32 ? few_f32_sets_kernel<2, STREAM, PREP>(ks) : few_f32_sets_kernel<4, STREAM, PREP>(ks);
}
template <bool NT, bool PREP> static auto few_bf16_kernel(int64_t rows) { return rows <= 64 ? score_few_kernel<64, NT, PREP> : score_few_kernel<128, NT, PREP>; }

template <class T>
static void score_chunk(const rl_batch* b, const HeadPlan& h, const Ptrs& q, int c0, float* z, float4* rec, const PrepJob& prep, hipStream_t s) {
  const Plan& p = h.p;
  const T* X = static_cast<const T*>(b->hidden);
  const T* W = static_cast<const T*>(b->weight);
  GemmDims d{};
  d.M = p.V; d.N = p.Tc; d.K = p.H; d.lda = p.H; d.ldb = p.H;
  d.b_rows = q.row_map + c0; d.b_span = p.R; d.n_real = &q.ctrl->n_real; d.chunk_start = c0; d.dyn = 2; d.group_m = TuneLogits::kBand;
  const EpiScore<T> e{z, p.Vp, rec, p.Tc, p.V, p.inv_tau};
  ProfScope ps(RL_PROF_GEMM_FWD, s);
  if (few_scores(b, p)) {
    const bool large = (int64_t)p.V * p.H * sizeof(T) > (int64_t)256 << 20;                  // (more than the memory-side cache holds, see few_streams_w)
    if constexpr (sizeof(T) == 2) {
      const bool nt = large && p.H % 64 == 0 && reinterpret_cast<uintptr_t>(W) % 128 == 0;
      auto kern = prep.on ? (nt ? few_bf16_kernel<true, true>(p.R) : few_bf16_kernel<false, true>(p.R)) : (nt ? few_bf16_kernel<true, false>(p.R) : few_bf16_kernel<false, false>(p.R));
      kern<<<2 * p.tiles_v + prep.on, 256, 0, s>>>(W, X, d, e, q.ids_c, prep.s, prep.f);
    } else {
      const int blocks = p.Vp / kGroup, sets = few_f32_sets(blocks, p.H), ks = p.R > 32 && sets > 2 ? 2 : sets;
      auto kern = prep.on ? (large ? few_f32_kernel<true, true>(p.R, ks) : few_f32_kernel<false, true>(p.R, ks)) : (large ? few_f32_kernel<true, false>(p.R, ks) : few_f32_kernel<false, false>(p.R, ks));
      kern<<<blocks + prep.on, 256 * ks, 0, s>>>(W, X, d, e, prep.s, prep.f);
    }
    return;
  }
  launch_gemm<TuneLogits>(W, X, d, e, s);
}

static int64_t chunk_bound(const Plan& p, int c0) { return p.R - c0 < p.Tc ? p.R - c0 : p.Tc; }      // rows of the chunk, at most

template <class TO> static auto few_grads_kernel(int nt) { return nt == 1 ? few_grads_bf16_kernel<1, TO> : nt == 2 ? few_grads_bf16_kernel<2, TO> : few_grads_bf16_kernel<4, TO>; }
// dS, then both gradients, of a batch of few rows; beside dS the loss and the rows of dX that do not count
template <class T>
static void run_few_grads(const rl_batch* b, const HeadPlan& h, const Ptrs& q, unsigned char* w, const DsJob& ds, const FinishJob& fin, const rl_distill_outputs* out, bool round, hipStream_t s) {
  const Plan& p = h.p;
  const int tokens = 16 * h.few_nt, pitch = few_pitch<T>(h.few_nt);
  T* ds1 = static_cast<T*>(q.ds);
  T* ds2 = sizeof(T) == 2 ? ds1 + (int64_t)kFewGradRows * p.Vp : static_cast<T*>(q.dst);          // (room for 256 rows)
  float* part = (float*)(w + h.off_few);
  const int n_ds = p.Vp / 64, zero = (int)((p.R + 3) / 4);
  {
    ProfScope ps(RL_PROF_GEMM_DS, s);
    few_ds_kernel<T><<<1 + n_ds + zero, 256, 0, s>>>(ds, (const int*)(w + h.off_pids), (const float*)(w + h.off_pval), h.K, tokens, pitch, ds1, ds2,
                                                     XtJob{nullptr, p.R, p.H, 0, n_ds, 0, 0, nullptr, q.cpos, nullptr, out->d_hidden, p.Tc}, fin);
  }
  ProfScope ps(RL_PROF_GEMM_BWD, s);
  const FewGrads j{b->weight, b->hidden, p.V, p.H, (const int*)(w + h.off_xrows), &q.ctrl->n_real, ds1, ds2, out->d_weight, part, h.few_splits, h.few_steps};
  const int cols = few_cols(p.dtype, h.few_nt), hs = (p.H + cols - 1) / cols, waves = hs < 4 ? hs : 4, blocks = (hs + waves - 1) / waves * h.few_splits;
  if constexpr (sizeof(T) == 2) {
    auto kern = round ? few_grads_kernel<bf16_t>(h.few_nt) : few_grads_kernel<float>(h.few_nt);
    kern<<<blocks, 64 * waves, 0, s>>>(j);
  } else {
    auto kern = h.few_nt == 1 ? few_grads_f32_kernel<1> : h.few_nt == 2 ? few_grads_f32_kernel<2> : h.few_nt == 3 ? few_grads_f32_kernel<3> : h.few_nt == 4 ? few_grads_f32_kernel<4>
                : h.few_nt == 6 ? few_grads_f32_kernel<6> : few_grads_f32_kernel<8>;
    kern<<<blocks, 64 * waves, 0, s>>>(j);
  }
  few_dx_kernel<T><<<(unsigned)(p.R * ((p.H + 63) / 64)), 256, 0, s>>>(part, h.few_splits, tokens, q.row_map, j.x_rows, &q.ctrl->n_real, p.H, static_cast<T*>(out->d_hidden));
}

template <class T>
static void run_distill(const rl_batch* b, const HeadPlan& h, const Ptrs& q, unsigned char* w, const int32_t* t_ids, const float* t_lp, const rl_distill_params* prm,
                        const rl_distill_outputs* out, bool bwd, const PrepJob& prep, hipStream_t s) {
  const Plan& p = h.p;
  float* z = (float*)(w + h.off_z);
  float4* rec = (float4*)(w + h.off_rec);
  const T* X = static_cast<const T*>(b->hidden);
  const T* W = static_cast<const T*>(b->weight);
  T* dS = static_cast<T*>(q.ds); T* dST = static_cast<T*>(q.dst);
  const bool round = prm->d_weight_dtype == RL_BF16;
  float* dw = !round ? static_cast<float*>(out->d_weight) : h.off_dw ? (float*)(w + h.off_dw) : nullptr;
  DistillRow* rows = bwd ? (DistillRow*)(w + h.off_rows) : nullptr;
  int* p_ids = (int*)(w + h.off_pids);
  float* p_val = (float*)(w + h.off_pval);
  int* x_rows = bwd ? (int*)(w + h.off_xrows) : nullptr;
  const FinishJob fin{(const double*)(w + h.off_term), (const int*)(w + h.off_info), q.ctrl, (const rl_stats*)(w + h.off_stats), out->loss, out->stats};
  const bool few = bwd && h.few_nt && reinterpret_cast<uintptr_t>(W) % 16 == 0;
  if (bwd && !few && !p.k_major_w) {
    ProfScope ps(RL_PROF_TRANSPOSE, s);
    launch_transpose<T>(dim3((p.Vp + 63) / 64, (p.H + 63) / 64), s, W, p.H, p.V, p.H, nullptr, q.ctrl, 0, 0, nullptr, nullptr, static_cast<T*>(q.wt), p.Vp, p.Vp, p.tiled);
  }
  for (int ch = 0; ch < p.n_chunks; ++ch) {
    const int c0 = ch * p.Tc;
    const int64_t n = chunk_bound(p, c0);
    score_chunk<T>(b, h, q, c0, z, rec, prep, s);
    {
      ProfScope ps(RL_PROF_COMBINE, s);
      launch_distill_rows(DistillJob{z, p.Vp, rec, p.Tc, h.groups, p.V, h.K, p.inv_tau, q.row_map, q.cstart, q.ctrl, c0, p.Tc, p.B, t_ids, t_lp, prm->rest,
                                     prm->aggregation == RL_AGG_TOKEN, prm->scale == 0.f ? 1.f : prm->scale, out->row_loss, out->lse,
                                     (double*)(w + h.off_term), (int*)(w + h.off_info), x_rows, rows, p_ids, p_val}, n, s);
    }
    if (!bwd) continue;
    if (few) {
      run_few_grads<T>(b, h, q, w, DsJob{z, p.Vp, rows, q.ctrl, c0, p.V, p.inv_tau}, fin, out, round, s);
      continue;
    }
    {
      ProfScope ps(RL_PROF_GEMM_DS, s);
      const int tile = sizeof(T) == 2 ? 256 : 64, cols = (int)((n + 255) / 256 * 4);
      const int n_ds = (int)((n + tile - 1) / tile * (p.Vp / 64)), n_xt = cols * ((p.H + 63) / 64);
      const int64_t zero = ch ? 0 : (p.R + 3) / 4;
      T* plain = sizeof(T) == 4 && p.k_major_w ? nullptr : dS;
      const bool last = ch + 1 == p.n_chunks;
      distill_ds_kernel<T><<<(unsigned)(last + n_ds + n_xt + (zero < 16384 ? zero : 16384)), 256, 0, s>>>(
          DsJob{z, p.Vp, rows, q.ctrl, c0, p.V, p.inv_tau}, plain, p.Vp, dST, p.Tc,
          XtJob{X, p.R, p.H, cols, n_ds, n_xt, reinterpret_cast<uintptr_t>(X) % 16 == 0, x_rows, q.cpos, q.xt, out->d_hidden, p.Tc}, last ? fin : FinishJob{});
      distill_patch_kernel<T><<<(unsigned)((n * h.K + 255) / 256), 256, 0, s>>>(p_ids, p_val, h.K, q.ctrl, c0, p.Tc, plain, p.Vp, dST, p.Tc);
    }
    contract_grads<T>(b, p, q, ch, out->d_hidden, dw, s, round ? static_cast<bf16_t*>(out->d_weight) : nullptr, x_rows);
  }
  if (bwd) return;
  ProfScope ps(RL_PROF_LOSS, s);
  distill_finish_kernel<<<1, 1024, 0, s>>>(fin);
}

}  // namespace rlk

using namespace rlk;

extern "C" {

int32_t rl_default_chunk_rows_distill(void) { return kDefaultChunkRowsDistill; }

static rl_status top_plan(const rl_batch* b, const rl_top_params* prm, HeadPlan& h) {
  if (!b || !prm) return RL_ERR_NULL;
  const rl_status st = head_plan(b, prm->top_k, prm->chunk_rows, prm->temperature, false, false, false, h);
  if (st != RL_OK) return st;
  return prm->top_k > b->V ? RL_ERR_SHAPE : RL_OK;
}

rl_status rl_token_top_logprobs_workspace_bytes(const rl_batch* b, const rl_top_params* prm, size_t* bytes) {
  if (!bytes) return RL_ERR_NULL;
  HeadPlan h;
  const rl_status st = top_plan(b, prm, h);
  if (st == RL_OK) *bytes = h.total;
  return st;
}

rl_status rl_token_top_logprobs(const rl_batch* b, const rl_top_params* prm, const rl_top_outputs* out, void* ws, size_t ws_bytes, void* stream) {
  if (!b || !prm || !out) return RL_ERR_NULL;
  if (!b->hidden || !b->weight || !b->mask || !b->cu_seqlens || (out->logprob && !b->token_ids)) return RL_ERR_NULL;
  if (!out->logprob && !out->lse && !out->entropy && !out->top_ids && !out->top_logprob) return RL_ERR_NULL;
  HeadPlan h;
  const rl_status st = top_plan(b, prm, h);
  if (st != RL_OK) return st;
  const Plan& p = h.p;
  const size_t R = (size_t)p.R;
  const Span in[] = {{b->hidden, p.esz * R * p.H}, {b->weight, p.esz * (size_t)p.V * p.H}, {b->token_ids, 4 * R}, {b->mask, R}, {b->cu_seqlens, 4 * ((size_t)p.B + 1)}};
  const Span outs[] = {{out->logprob, 4 * R}, {out->lse, 4 * R}, {out->entropy, 4 * R}, {out->top_ids, 4 * R * h.K}, {out->top_logprob, 4 * R * h.K}};
  if (overlap(outs, 5, in, 5)) return RL_ERR_RANGE;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) || ws_bytes < h.total) return RL_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const Ptrs q = carve(ws, p);
  unsigned char* w = static_cast<unsigned char*>(ws);
  float* z = (float*)(w + h.off_z);
  float4* rec = (float4*)(w + h.off_rec);
  rl_outputs cleared{};
  cleared.logprob = out->logprob; cleared.lse = out->lse; cleared.entropy = out->entropy;
  const PrepJob prep = head_prep(b, p, q, cleared, s);
  for (int ch = 0; ch < p.n_chunks; ++ch) {
    const int c0 = ch * p.Tc;
    if (p.dtype == RL_BF16) score_chunk<bf16_t>(b, h, q, c0, z, rec, prep, s);
    else score_chunk<float>(b, h, q, c0, z, rec, prep, s);
    ProfScope ps(RL_PROF_COMBINE, s);
    const unsigned blocks = (unsigned)((chunk_bound(p, c0) + kXcds - 1) / kXcds * kXcds);
    const int64_t all = (p.R + kTopWaves - 1) / kTopWaves;
    const unsigned fill = ch == 0 && (out->top_ids || out->top_logprob) ? (unsigned)(all < 4096 ? all : 4096) : 0;
    const TopJob j{z, p.Vp, rec, p.Tc, h.groups, p.V, h.K, p.inv_tau, q.row_map, q.ids_c, q.cpos, q.ctrl, c0, p.Tc, p.R, (int)blocks,
                   out->logprob, out->lse, out->entropy, out->top_ids, out->top_logprob};
    launch_top(j, blocks + fill, s);
  }
  return hipGetLastError() == hipSuccess ? RL_OK : RL_ERR_HIP;
}

static rl_status distill_plan(const rl_batch* b, const rl_distill_params* prm, bool bwd, HeadPlan& h) {
  if (!b || !prm) return RL_ERR_NULL;
  if (prm->d_weight_dtype != RL_F32 && !(prm->d_weight_dtype == RL_BF16 && b->dtype == RL_BF16)) return RL_ERR_DTYPE;
  if (prm->rest != RL_REST_BUCKET && prm->rest != RL_REST_RENORMALISE) return RL_ERR_RANGE;
  if (prm->aggregation != RL_AGG_SEQUENCE && prm->aggregation != RL_AGG_TOKEN) return RL_ERR_RANGE;
  if (!(prm->scale >= -3.0e38f && prm->scale <= 3.0e38f)) return RL_ERR_RANGE;
  return head_plan(b, prm->top_k, prm->chunk_rows, prm->temperature, bwd, true, prm->d_weight_dtype == RL_BF16, h);
}

rl_status rl_distill_workspace_bytes(const rl_batch* b, const rl_distill_params* prm, int32_t want_backward, size_t* bytes) {
  if (!bytes) return RL_ERR_NULL;
  HeadPlan h;
  const rl_status st = distill_plan(b, prm, want_backward != 0, h);
  if (st == RL_OK) *bytes = h.total;
  return st;
}

rl_status rl_distill_loss_fwd_bwd(const rl_batch* b, const int32_t* t_ids, const float* t_lp, const rl_distill_params* prm, const rl_distill_outputs* out,
                                  void* ws, size_t ws_bytes, void* stream) {
  if (!b || !prm || !out) return RL_ERR_NULL;
  if (!b->hidden || !b->weight || !b->mask || !b->cu_seqlens || !t_ids || !t_lp || !out->loss) return RL_ERR_NULL;
  const bool bwd = out->d_hidden || out->d_weight;
  if (bwd && (!out->d_hidden || !out->d_weight)) return RL_ERR_NULL;
  HeadPlan h;
  const rl_status st = distill_plan(b, prm, bwd, h);
  if (st != RL_OK) return st;
  const Plan& p = h.p;
  const size_t R = (size_t)p.R, K = (size_t)h.K, xb = p.esz * R * p.H;
  const Span in[] = {{b->weight, p.esz * (size_t)p.V * p.H}, {b->mask, R}, {b->cu_seqlens, 4 * ((size_t)p.B + 1)}, {t_ids, 4 * R * K}, {t_lp, 4 * R * K},
                     {b->hidden, xb}};
  const Span outs[] = {{out->loss, 4}, {out->row_loss, 4 * R}, {out->lse, 4 * R}, {out->stats, sizeof(rl_distill_stats)},
                       {out->d_weight, (size_t)(prm->d_weight_dtype == RL_BF16 ? 2 : 4) * p.V * p.H}, {out->d_hidden, xb}};
  if (overlap(outs, 5, in, 6) || overlap(&outs[5], 1, in, out->d_hidden == b->hidden ? 5 : 6) || overlap(outs, 6, in, 0)) return RL_ERR_RANGE;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) || ws_bytes < h.total) return RL_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const Ptrs q = carve(ws, p);
  unsigned char* w = static_cast<unsigned char*>(ws);
  rl_batch no_ids = *b;
  no_ids.token_ids = nullptr;
  rl_outputs cleared{};
  cleared.logprob = out->row_loss; cleared.lse = out->lse; cleared.stats = (rl_stats*)(w + h.off_stats);
  const PrepJob prep = head_prep(&no_ids, p, q, cleared, s);
  if (p.dtype == RL_BF16) run_distill<bf16_t>(b, h, q, w, t_ids, t_lp, prm, out, bwd, prep, s);
  else run_distill<float>(b, h, q, w, t_ids, t_lp, prm, out, bwd, prep, s);
  return hipGetLastError() == hipSuccess ? RL_OK : RL_ERR_HIP;
}

}  // extern "C"
