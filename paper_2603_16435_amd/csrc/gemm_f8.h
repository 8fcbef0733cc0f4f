// gemm_f8.h - product of two matrices of 8-bit rows (f8_rows.h):  y[m, n] = sum_k x[m, k] w[n, k]
//
// A slab is one block of 128 k: 128 bytes of a row, one 16x16x128 MFMA a block of the tile, which multiplies the two blocks' scales in by itself
// (v_mfma_scale_f32_16x16x128_f8f6f4; operands in either format) and adds in f32.  Rows are padded to whole blocks with zeros, so K has no tail.
// An operand is 32 bytes a lane: row l % 16, and which 32 of the 128 k a lane group l / 16 holds is free as long as both operands agree (the sum does not care,
// and the scale is one for all 128).
// That MFMA adds eight products at a time on a common exponent, what is below about 2^-13 of the largest of the eight being cut off, and in f32 from there on
// (measured: 2.6e-5 of the result at K = 128).  Where y is bf16 that is a hundredth of y's own rounding, and taken: one value in a hundred is rounded the other way (4e-4 of the result),
// the error against 64 bits is 1.66204e-3 where correct rounding has 1.66198e-3 (4096 x 2048 x 3584, normal values), and no side is preferred; where y is f32 the operands are restored to bf16, which is
// exact, on their way to 16x16x32 bf16 MFMAs, whose products and sums are those of f32, at half the rate (kExact).
// The operands are exchanged (w first): a lane then holds four consecutive n of one row of y.
//
//  * f8_gemm_kernel  general: BM x BN tile, four wavefronts, cut along K where there are few tiles.
//  * f8_hot_kernel   256 x 256 tile, for many tiles and bf16 outputs.
//  * f8_few_kernel   up to 16 rows of x: bound by reading w.
#pragma once
#include <type_traits>

#include "f8_rows.h"

namespace rlk {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));

struct F8Operand { const uint8_t* codes; const uint8_t* scales; int rows, Kp, Ks; };

// 64 lanes x 4 bytes, an address per lane, to 256 bytes of LDS at l
__device__ __attribute__((always_inline)) inline void load4_to_lds_lanes(const void* g, void* l) {
  const unsigned lds = (unsigned)(size_t)(lds_ptr_t)l;      // uniform
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" :: "v"(g), "s"(lds) : "memory");
}

// acc += x-block * w-block; byte 0 of sx / sw: the scales of the lane's row
template <int FX, int FW> __device__ __attribute__((always_inline)) inline void mfma_f8(floatx4& acc, const i32x8_t& w, const i32x8_t& x, unsigned sw, unsigned sx) {
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, FW, FX, 0, (int)sw, 0, (int)sx);
}

// The 32 codes of an operand and their scale as four operands of 16x16x32 bf16 MFMAs.
struct ExactOperand { u32x4_t v[4]; };
template <int F> __device__ __attribute__((always_inline)) inline ExactOperand exact_operand(const i32x8_t& c, unsigned scale) {
  const float s = f8_scale_value(scale & 255u);
  ExactOperand o;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    bf16x2 lo, hi;
    if constexpr (F == kE4M3) { lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[i], s, false); hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)c[i], s, true); }
    else { lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((unsigned)c[i], s, false); hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((unsigned)c[i], s, true); }
    o.v[i >> 1][(i & 1) * 2] = __builtin_bit_cast(unsigned, lo); o.v[i >> 1][(i & 1) * 2 + 1] = __builtin_bit_cast(unsigned, hi);
  }
  return o;
}
__device__ __attribute__((always_inline)) inline void mfma_exact(floatx4& acc, const ExactOperand& w, const ExactOperand& x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.v[i]), __builtin_bit_cast(bf16x8, x.v[i]), acc, 0, 0, 0);
}
template <class T> constexpr bool kExact = sizeof(T) == 4;

// Four consecutive values of a row of y, at most `left` of them.
typedef float floatx4_el4 __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4_el2 __attribute__((ext_vector_type(4), aligned(2)));
template <class T> __device__ __attribute__((always_inline)) inline void store4(T* p, int left, const floatx4& v) {
  if (left >= 4) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<floatx4_el4*>(p) = v;
    else *reinterpret_cast<bf16x4_el2*>(p) = bf16x4_el2{(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i) if (i < left) p[i] = (T)v[i];
  }
}

template <class T> struct F8Product {
  F8Operand x, w;
  T* y; int64_t ldy;
  int M, N, nk;                      // nk: blocks of k
  int slices, per;                   // cut along K: slices of `per` blocks (a multiple of four), whose sums go to part [slices][M][Np] instead of y
  float* part; int Np;
};

// S stages of a slab: S - 1 slabs are on their way while one is multiplied (more of them: no faster, even where a CU has one workgroup).  A stage holds the slab of x, that of w and a word of scales for each of their rows (four slabs'
// bytes: fetched with every slab, so that each has as many loads).
template <int BM, int BN> constexpr int f8_stage_bytes() { return (BM + BN) * kSlabBytes + 1024; }
template <int FX, int FW, class T, int BM, int BN, int S>
__global__ __launch_bounds__(256, 2) void f8_gemm_kernel(F8Product<T> j) {
  constexpr int MB = BM / 32, NB = BN / 32, STAGE = f8_stage_bytes<BM, BN>(), ROWS = (BM + BN) / 4, LOADS = ROWS / 8;      // of a wavefront and slab: rows, loads of eight rows
  constexpr int WAIT = (S - 2) * (LOADS + 1);
  static_assert(ROWS <= 64 && ROWS % 8 == 0 && WAIT < 64, "tile");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S * STAGE];
  const int tiles_m = (j.M + BM - 1) / BM, tiles_n = (j.N + BN - 1) / BN;
  int t;
  if (!run_of_block(blockIdx.x, tiles_m * tiles_n * j.slices, t)) return;
  const int slice = t / (tiles_m * tiles_n);
  t -= slice * (tiles_m * tiles_n);
  const int tn = t / tiles_m, tm = t - tn * tiles_m;
  const int k0 = slice * j.per, nk = j.nk - k0 < j.per ? j.nk - k0 : j.per;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;

  // row lr of a stage: x rows, then w rows
  auto row_of = [&](int lr, bool& is_x) __attribute__((always_inline)) {
    is_x = lr < BM;
    const int r = is_x ? tm * BM + lr : tn * BN + lr - BM, last = (is_x ? j.M : j.N) - 1;
    return r < last ? r : last;
  };
  const uint8_t* src[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int lr = wave * ROWS + i * 8 + (lane >> 3), c = (lane & 7) ^ ((lr >> 1) & 7);
    bool is_x;
    const int r = row_of(lr, is_x);
    src[i] = (is_x ? j.x.codes + (int64_t)r * j.x.Kp : j.w.codes + (int64_t)r * j.w.Kp) + (int64_t)k0 * 128 + c * 16;
  }
  const uint8_t* scales;
  {
    bool is_x;
    const int r = row_of(wave * ROWS + (lane < ROWS ? lane : ROWS - 1), is_x);
    scales = (is_x ? j.x.scales + (int64_t)r * j.x.Ks : j.w.scales + (int64_t)r * j.w.Ks) + k0;          // (k0 is a multiple of four)
  }
  auto issue = [&](int kt, int stage, int i) __attribute__((always_inline)) {      // load i of LOADS + 1
    unsigned char* to = smem + stage * STAGE;
    if (i < LOADS) load16_to_lds_lanes(src[i] + (int64_t)kt * 128, to + (wave * LOADS + i) * 1024);
    else load4_to_lds_lanes(scales + (kt & ~3), to + (BM + BN) * kSlabBytes + wave * 256);
  };
  const int frow = lane & 15, g = lane >> 4;
  floatx4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[i][b] = floatx4{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int i = 0; i < S - 1; ++i)
    if (i < nk) {
#pragma unroll
      for (int l = 0; l <= LOADS; ++l) issue(i, i, l);
    }
  int at = 0, next = S - 1;                                          // stage of slab kt, and of slab kt + S - 1
  for (int kt = 0; kt < nk; ++kt) {
    if (kt + S - 2 < nk) __builtin_amdgcn_s_waitcnt(0x0F70 | (WAIT & 15) | (WAIT >> 4) << 14);          // this slab has landed ...
    else __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();                                                 // ... everybody's, and nobody reads the stage of the slab before it any more
    const unsigned char* xa = smem + at * STAGE;
    const unsigned* words = reinterpret_cast<const unsigned*>(xa + (BM + BN) * kSlabBytes);
    const int shift = (kt & 3) * 8;
    auto scale = [&](int r) __attribute__((always_inline)) { return words[r / ROWS * 64 + r % ROWS] >> shift; };
    auto codes = [&](int r) __attribute__((always_inline)) {
      const i32x4_t lo = *reinterpret_cast<const i32x4_t*>(xa + lds_off(r, g)), hi = *reinterpret_cast<const i32x4_t*>(xa + lds_off(r, g + 4));
      return (i32x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // fragments first, then the MFMAs with the loads of the slab S - 1 ahead between them: all four wavefronts issue theirs at the same time, and in one burst ahead
    // of the fragments they held up both (128 x 128, 2000 rows of 3584 columns, 3584 rows of w 33.9 -> 31.8 us; reading the next slab's fragments between the MFMAs as well: slower)
    i32x8_t cx[MB], cw[NB];
    unsigned sx[MB], sw[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) { const int r = wm * (BM / 2) + i * 16 + frow; cx[i] = codes(r); sx[i] = scale(r); }
#pragma unroll
    for (int b = 0; b < NB; ++b) { const int r = BM + wn * (BN / 2) + b * 16 + frow; cw[b] = codes(r); sw[b] = scale(r); }
    std::conditional_t<kExact<T>, ExactOperand, i32x8_t> fx[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) { if constexpr (kExact<T>) fx[i] = exact_operand<FX>(cx[i], sx[i]); else fx[i] = cx[i]; }
    const bool more = kt + S - 1 < nk;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if constexpr (kExact<T>) {
        const ExactOperand ew = exact_operand<FW>(cw[b], sw[b]);
#pragma unroll
        for (int i = 0; i < MB; ++i) mfma_exact(acc[i][b], ew, fx[i]);
      } else {
#pragma unroll
        for (int i = 0; i < MB; ++i) mfma_f8<FX, FW>(acc[i][b], cw[b], fx[i], sw[b], sx[i]);
      }
      if (more) {
#pragma unroll
        for (int l = b * (LOADS + 1) / NB; l < (b + 1) * (LOADS + 1) / NB; ++l) issue(kt + S - 1, next, l);
      }
    }
    at = at + 1 == S ? 0 : at + 1; next = next + 1 == S ? 0 : next + 1;
  }
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int m = tm * BM + wm * (BM / 2) + i * 16 + frow;
    if (m >= j.M) continue;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int n = tn * BN + wn * (BN / 2) + b * 16 + g * 4;
      if (j.slices > 1) { if (n < j.Np) *reinterpret_cast<floatx4*>(j.part + ((int64_t)slice * j.M + m) * j.Np + n) = acc[i][b]; }
      else store4(j.y + (int64_t)m * j.ldy + n, j.N - n, acc[i][b]);
    }
  }
}

// The slices of a cut product, added in order.
template <class T>
__global__ __launch_bounds__(256) void f8_slices_kernel(const float* part, int slices, int M, int N, int Np, T* y, int64_t ldy) {
  const int n4 = Np / 4;
  const int64_t all = (int64_t)M * n4, stride = (int64_t)M * Np;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < all; q += (int64_t)gridDim.x * 256) {
    const int64_t m = q / n4;
    const int n = (int)(q - m * n4) * 4;
    const float* p = part + m * Np + n;
    floatx4 s = *reinterpret_cast<const floatx4*>(p);
    for (int k0 = 1; k0 < slices; k0 += 4) {
      floatx4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = k0 + k < slices ? *reinterpret_cast<const floatx4*>(p + (k0 + k) * stride) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) s += v[k];
    }
    store4(y + m * ldy + n, N - n, s);
  }
}

// ------------------------------------------------------------------ hot kernel
// 256 x 256 tile, four wavefronts of 128 x 128 (256 accumulators a lane, in AGPRs), y in bf16.  32768 x 3584 x 3584: 316 to 330 us, 2.6 PFLOP/s (the vendor's product with one scale a
// tensor 2.42); the MFMAs are busy 69 % of the clocks, at the 1.88 GHz that the power limit leaves (nothing but these MFMAs: 2.12 GHz, 4.2 PFLOP/s; without the loads 3.3 to 3.6; eight
// wavefronts, other places for the loads, prefetches into the L2: no gain).  A slab's 64 MFMAs of 32 cycles are as long as those of a slab of the bf16
// hot kernel (gemm_nt.h), on the same bytes, so it is built like that one: slabs go straight into two LDS stages, every MFMA is fenced, fragment reads, slab
// loads are dealt out between them.  A slab is two phases: all eight blocks of x against blocks 0..3 of w, then against 4..7.  The
// workgroup meets between them, when the last fragments of the slab have been read: the second phase runs from registers, covers the first fragment reads of the next slab (an
// x block is fetched as soon as the last MFMA that reads its registers is out) and the first loads of the slab after it.
// Scales: one word a row holds four slabs' bytes, of which the MFMA picks one; the words come through LDS as well, a group of slabs ahead.
// LDS row 16 b + 4 g + e of w holds column 32 (b / 2) + 8 g + 4 (b % 2) + e of the tile's half (perm_row), so that a lane ends up with eight consecutive columns in a pair of
// blocks: 16-byte stores.
// B: which byte of sw and sx
template <int FX, int FW, int B> __device__ __attribute__((always_inline)) inline void mfma_f8_acc(floatx4& acc, const i32x8_t& w, const i32x8_t& x, unsigned sw, unsigned sx) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%7,%7,0] op_sel_hi:[%8,%8,0] cbsz:%5 blgp:%6"
               : "+a"(acc) : "v"(w), "v"(x), "v"(sw), "v"(sx), "n"(FW), "n"(FX), "n"(B & 1), "n"(B >> 1));
}
struct F8Hot { F8Operand x, w; bf16_t* y; int64_t ldy; int M, N, nk; };
constexpr int kF8Band = 8;

template <int FX, int FW>
__global__ __launch_bounds__(256) void f8_hot_kernel(F8Hot j) {
  __shared__ __attribute__((aligned(1024))) unsigned char stage0[kHotStageBytes];
  __shared__ __attribute__((aligned(1024))) unsigned char stage1[kHotStageBytes];
  __shared__ __attribute__((aligned(1024))) unsigned scales0[512];          // a word a row, x then w: the scales of four slabs
  __shared__ __attribute__((aligned(1024))) unsigned scales1[512];
  constexpr int A_BYTES = 256 * kSlabBytes;
  const int tiles_m = (j.M + 255) / 256, tiles_n = (j.N + 255) / 256;
  int tm, tn;
  if (!tile_of_block(blockIdx.x, tiles_m, tiles_n, kF8Band, false, tm, tn)) return;
  tm = __builtin_amdgcn_readfirstlane(tm); tn = __builtin_amdgcn_readfirstlane(tn);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
  const int nk = j.nk;

  // slab loads: wavefront w fills rows [64 w, 64 w + 64) of x and of w, eight rows a load; the tile's rows are within 32 bits of its first
  const uint8_t* xbase = uniform_ptr(j.x.codes + (int64_t)tm * 256 * j.x.Kp);
  const uint8_t* wbase = uniform_ptr(j.w.codes + (int64_t)tn * 256 * j.w.Kp);
  unsigned xoff[8], woff[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int lr = wave * 64 + i * 8 + (lane >> 3), c = (lane & 7) ^ ((lr >> 1) & 7);
    int m = lr, n = perm_lds_row_a(lr);
    m = tm * 256 + m < j.M ? m : j.M - 1 - tm * 256; n = tn * 256 + n < j.N ? n : j.N - 1 - tn * 256;
    xoff[i] = (unsigned)m * (unsigned)j.x.Kp + c * 16; woff[i] = (unsigned)n * (unsigned)j.w.Kp + c * 16;
  }
  auto issue = [&](int slab, unsigned char* stage, int i) __attribute__((always_inline)) {
    unsigned char* dst = stage + wave * 64 * kSlabBytes + (i & 7) * 8 * kSlabBytes + (i < 8 ? 0 : A_BYTES);
    if (i < 8) load16_to_lds_uniform(xbase + (int64_t)slab * 128, xoff[i & 7], dst);
    else load16_to_lds_uniform(wbase + (int64_t)slab * 128, woff[i & 7], dst);
  };
  const int frow = lane & 15, g = lane >> 4;
  // scales: wavefront w fetches the words of its 64 rows of x and of w
  const int groups = (nk + 3) / 4;
  const unsigned *xs, *ws;
  {
    int m = tm * 256 + wave * 64 + lane, n = tn * 256 + perm_lds_row_a(wave * 64 + lane);
    m = m < j.M ? m : j.M - 1; n = n < j.N ? n : j.N - 1;
    xs = reinterpret_cast<const unsigned*>(j.x.scales + (int64_t)m * j.x.Ks);
    ws = reinterpret_cast<const unsigned*>(j.w.scales + (int64_t)n * j.w.Ks);
  }
  auto issue_scales = [&](int group, unsigned* to) __attribute__((always_inline)) {
    group = group < groups ? group : groups - 1;
    load4_to_lds_lanes(xs + group, to + wave * 64);
    load4_to_lds_lanes(ws + group, to + 256 + wave * 64);
  };
  unsigned sx[8], sw[8];

  floatx4 acc[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int b = 0; b < 8; ++b) acc[i][b] = floatx4{0.f, 0.f, 0.f, 0.f};
  i32x8_t fx[8], fw[2][4];
  const int xrow = (wm * 128 + frow) * kSlabBytes, wrow = A_BYTES + (wn * 128 + frow) * kSlabBytes, swz = (frow >> 1) & 7;
  const int slot0 = (g ^ swz) << 4, slot1 = ((g + 4) ^ swz) << 4;
  auto read = [&](const unsigned char* p) __attribute__((always_inline)) {
    const i32x4_t lo = *reinterpret_cast<const i32x4_t*>(p + slot0), hi = *reinterpret_cast<const i32x4_t*>(p + slot1);
    return (i32x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto read_sx = [&](const unsigned* from, int i) __attribute__((always_inline)) { sx[i] = from[wm * 128 + i * 16 + frow]; };
  auto read_sw = [&](const unsigned* from, int i) __attribute__((always_inline)) { sw[i] = from[256 + wn * 128 + i * 16 + frow]; };
  // Slab kt = B modulo 4 is in `cur`; fx and fw[0] hold its x blocks and w blocks 0..3, the loads of slab kt + 1 are on their way to `nxt`.  `scales`: where the words of
  // the next group go.
  auto slab = [&](auto B, unsigned char* cur, unsigned char* nxt, int kt, unsigned* scales) __attribute__((always_inline)) {
    const int k2 = kt + 2 < nk ? kt + 2 : nk - 1;
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      const int i = q >> 2, b = i & 1 ? 3 - (q & 3) : q & 3;
      mfma_f8_acc<FX, FW, B.value>(acc[i][b], fw[0][b], fx[i], sw[b], sx[i]);
      if (q % 2 == 0 && q < 8) fw[1][q / 2] = read(cur + wrow + (4 + q / 2) * 16 * kSlabBytes);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);       // own loads have landed, own fragment reads are done
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      const int i = q >> 2, b = i & 1 ? 3 - (q & 3) : q & 3;
      mfma_f8_acc<FX, FW, B.value>(acc[i][4 + b], fw[1][b], fx[i], sw[4 + b], sx[i]);
      if ((q & 3) == 3) {
        fx[i] = read(nxt + xrow + i * 16 * kSlabBytes);
        if (B.value == 3) read_sx(scales, i);
      } else if (q % 8 == 1) {
        fw[0][q / 8] = read(nxt + wrow + (q / 8) * 16 * kSlabBytes);
        if (B.value == 3) read_sw(scales, q / 8);
      }
      if (q % 2 == 0) issue(k2, cur, q / 2);
      if (B.value == 0 && q == 0) issue_scales(kt / 4 + 1, scales);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (B.value == 3) {
#pragma unroll
      for (int i = 4; i < 8; ++i) read_sw(scales, i);
    }
  };

#pragma unroll
  for (int i = 0; i < 16; ++i) issue(0, stage0, i);
  issue_scales(0, scales0);
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int b = 0; b < 8; ++b) asm volatile("" : "+a"(acc[i][b]));
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) issue(nk > 1 ? 1 : 0, stage1, i);
#pragma unroll
  for (int i = 0; i < 8; ++i) { fx[i] = read(stage0 + xrow + i * 16 * kSlabBytes); read_sx(scales0, i); read_sw(scales0, i); }
#pragma unroll
  for (int b = 0; b < 4; ++b) fw[0][b] = read(stage0 + wrow + b * 16 * kSlabBytes);
  typedef std::integral_constant<int, 0> B0; typedef std::integral_constant<int, 1> B1; typedef std::integral_constant<int, 2> B2; typedef std::integral_constant<int, 3> B3;
  int kt = 0;
  for (; kt + 3 < nk; kt += 4) {
    slab(B0(), stage0, stage1, kt, scales1);
    slab(B1(), stage1, stage0, kt + 1, scales1);
    slab(B2(), stage0, stage1, kt + 2, scales1);
    slab(B3(), stage1, stage0, kt + 3, scales1);
  }
  if (kt < nk) slab(B0(), stage0, stage1, kt, scales1);
  if (kt + 1 < nk) slab(B1(), stage1, stage0, kt + 1, scales1);
  if (kt + 2 < nk) slab(B2(), stage0, stage1, kt + 2, scales1);
  __builtin_amdgcn_s_waitcnt(0x0070);         // the loads past the end
  mfma_drain();

  const bool edge = tm * 256 + 256 > j.M || tn * 256 + 256 > j.N;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int m = tm * 256 + wm * 128 + i * 16 + frow;
    if (edge && m >= j.M) continue;
#pragma unroll
    for (int b = 0; b < 8; b += 2) {
      const int n = tn * 256 + wn * 128 + b * 16 + g * 8;
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[e] = acc_read<true>(acc[i][b], e); v[4 + e] = acc_read<true>(acc[i][b + 1], e); }
      raw_store(j.y + (int64_t)m * j.ldy + n, edge ? j.N - n : 8, raw_make<bf16_t>(v));
    }
  }
}

// ------------------------------------------------------------------ few rows
// Up to 16 rows of x: sixteen rows of w a workgroup, whose codes go from memory straight into MFMA operands (32 consecutive bytes a lane: the lanes of a row
// have its line), four slabs of a wavefront on their way; eight wavefronts take every eighth slab and their sums are added at the end.  x comes out of the L2.
// Faster than the general kernel's tiles while a CU has one workgroup (8 rows of 3584, 3584 rows of w 5.4 us and 7.2; 14336 rows of w 15.5 and 10.9).
// RAW: x as it is: each workgroup packs all of it into LDS while its first codes of w are on their way, which takes a launch less.
constexpr int kF8FewRows = 16, kF8FewWaves = 8;

template <class T> struct F8Few {
  F8Operand x, w;                    // x: read; or, where raw is set, written by the first workgroup (codes nullptr: not wanted)
  const T* raw; int64_t ldx; int K;
  T* y; int64_t ldy;
  int M, N, nk;
};
__host__ __device__ inline int f8_raw_pitch(int Kp) { return Kp + 32; }                     // bytes of a row in LDS: rows in other banks

template <int FX, int FW, class T, bool RAW>
__global__ __launch_bounds__(kF8FewWaves * 64) void f8_few_kernel(F8Few<T> j) {
  __shared__ floatx4 sums[kF8FewWaves][64];
  extern __shared__ __attribute__((aligned(16))) uint8_t xlds[];              // RAW: codes [M][pitch], scales [M][Ks]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), frow = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, pitch = f8_raw_pitch(j.x.Kp);
  const int nr = n0 + frow < j.N ? n0 + frow : j.N - 1;
  const uint8_t* wp = j.w.codes + (int64_t)nr * j.w.Kp + g * 32;
  const uint8_t* wsp = j.w.scales + (int64_t)nr * j.w.Ks;
  const int mr = frow < j.M ? frow : j.M - 1;                        // (rows that are not there: their results are not stored)
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;                                               // slabs in flight
  i32x4_t wc[U][2];
  unsigned sw[U];
  auto fetch = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int k = k0 + u * kF8FewWaves; k = k < j.nk ? k : j.nk - 1;
      wc[u][0] = *reinterpret_cast<const i32x4_t*>(wp + (int64_t)k * 128); wc[u][1] = *reinterpret_cast<const i32x4_t*>(wp + (int64_t)k * 128 + 16);
      sw[u] = wsp[k];
    }
    asm volatile("" ::: "memory");                                   // (all of them out before anything else: the compiler would move each to where it is used)
  };
  fetch(wave);
  if constexpr (RAW) {
    uint8_t* slds = xlds + j.M * pitch;
    const int per = j.x.Kp / 8;                                      // pieces of a row: sixteen lanes have a block
    for (int p = threadIdx.x; p < j.M * per; p += kF8FewWaves * 64) {
      const int r = p / per, col = (p - r * per) * 8;
      const Raw8<T> raw = raw_load(j.raw + (int64_t)r * j.ldx + col, j.K - col);
      float v[8];
      unsigned a = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) { v[e] = raw_get(raw, e); const unsigned b = finite_bits(v[e]); a = a > b ? a : b; }
      unsigned s;
      const u32x2_t c = f8_pack8(v, a, FX, s);
      *reinterpret_cast<u32x2_t*>(xlds + r * pitch + col) = c;
      if ((threadIdx.x & 15) == 0) slds[r * j.x.Ks + col / kF8Block] = (uint8_t)s;
      if (j.x.codes && blockIdx.x == 0) {
        *reinterpret_cast<u32x2_t*>(const_cast<uint8_t*>(j.x.codes) + (int64_t)r * j.x.Kp + col) = c;
        if ((threadIdx.x & 15) == 0) {
          uint8_t* q = const_cast<uint8_t*>(j.x.scales) + (int64_t)r * j.x.Ks;
          q[col / kF8Block] = (uint8_t)s;
          if (col / kF8Block == j.nk - 1) for (int b = j.nk; b < j.x.Ks; ++b) q[b] = 127;
        }
      }
    }
    __syncthreads();
  }
  for (int k0 = wave; k0 < j.nk; k0 += kF8FewWaves * U) {
    if (k0 != wave) fetch(k0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool there = k0 + u * kF8FewWaves < j.nk;                // (no branch around the loads of x: a slab past the end is the last one, both operands zeroed)
      const int k = there ? k0 + u * kF8FewWaves : j.nk - 1;
      i32x8_t wf = __builtin_shufflevector(wc[u][0], wc[u][1], 0, 1, 2, 3, 4, 5, 6, 7);
      const uint8_t* xp = RAW ? xlds + mr * pitch + k * 128 + g * 32 : j.x.codes + (int64_t)mr * j.x.Kp + k * 128 + g * 32;
      i32x8_t xc = __builtin_shufflevector(*reinterpret_cast<const i32x4_t*>(xp), *reinterpret_cast<const i32x4_t*>(xp + 16), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int e = 0; e < 8; ++e) { wf[e] = there ? wf[e] : 0; xc[e] = there ? xc[e] : 0; }
      const unsigned sx = RAW ? xlds[j.M * pitch + mr * j.x.Ks + k] : j.x.scales[(int64_t)mr * j.x.Ks + k];
      if constexpr (kExact<T>) mfma_exact(acc, exact_operand<FW>(wf, sw[u]), exact_operand<FX>(xc, sx));
      else mfma_f8<FX, FW>(acc, wf, xc, sw[u], sx);
    }
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int i = 1; i < kF8FewWaves; ++i) acc += sums[i][lane];
  if (frow < j.M) store4(j.y + (int64_t)frow * j.ldy + n0 + g * 4, j.N - n0 - g * 4, acc);
}

}  // namespace rlk
