// f8_rows.h - activations and weights in 8 bits ("8-bit rows"): packing, restoring, packing of weights.
//
// A matrix [R, K] is held as codes [R][Kp] (one byte a value, Kp = K rounded up to 128, pads zero) and one scale byte s for 128 consecutive
// values of a row, [R][Ks], Ks = the number of blocks rounded up to 4: a value is code * 2^(s - 127).  The scale is the smallest power of two
// under which the block's largest finite magnitude is representable (448 in e4m3, 57344 in e5m2); a block of zeros has 1.
// Why powers of two: the scaled MFMA of this part multiplies them in by itself, so a block's scale costs the product nothing, and a restored value
// has at most four significant bits, so that it is exact in bf16.  A scale of full precision would use up to one bit more of the range, no more
// of the precision.
//
// All kernels here are bound by HBM.  A lane holds eight consecutive values (16 bytes in bf16), sixteen lanes a block of 128: the block's maximum takes four
// rotations inside the sixteen lanes, codes leave as 128-byte lines, the scales of four blocks as one word.  16381 rows of 5120, bf16: pack 49 us (5.1 TB/s), restore 37 (6.8).
#pragma once
#include "gemm_nt.h"

namespace rlk {

constexpr int kF8Block = 128;
enum F8Format { kE4M3 = 0, kE5M2 = 1 };                          // = rl_f8_format

__host__ __device__ inline int f8_blocks(int K) { return (K + kF8Block - 1) / kF8Block; }
__host__ __device__ inline int f8_code_pitch(int K) { return f8_blocks(K) * kF8Block; }
__host__ __device__ inline int f8_scale_pitch(int K) { return (f8_blocks(K) + 3) / 4 * 4; }

// Eight consecutive values of a row as they lie in memory, at any alignment an element has (global accesses of this part need none).
typedef unsigned u32x4_el2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u32x2_el2 __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned u32_el2 __attribute__((aligned(2)));
template <class T> struct Raw8;
template <> struct Raw8<bf16_t> { u32x4_t v; };
template <> struct Raw8<float> { u32x4_t v, w; };

template <class T> __device__ __attribute__((always_inline)) inline Raw8<T> raw_zero() {
  Raw8<T> r;
  r.v = u32x4_t{0, 0, 0, 0};
  if constexpr (sizeof(T) == 4) r.w = r.v;
  return r;
}
template <class T> __device__ __attribute__((always_inline)) inline Raw8<T> raw_load8(const T* p) {
  Raw8<T> r;
  r.v = *reinterpret_cast<const u32x4_el2*>(p);
  if constexpr (sizeof(T) == 4) r.w = *reinterpret_cast<const u32x4_el2*>(p + 4);
  return r;
}
// The first n of 8 (n < 8), by four, two and one.
template <class T> __device__ __attribute__((always_inline)) inline Raw8<T> raw_load_part(const T* p, int n) {
  Raw8<T> r = raw_zero<T>();
  const bool two = n & 2;
  if constexpr (sizeof(T) == 4) {
    u32x2_el2 b = {0, 0};
    unsigned c = 0;
    if (n & 4) r.v = *reinterpret_cast<const u32x4_el2*>(p);
    if (n & 2) b = *reinterpret_cast<const u32x2_el2*>(p + (n & 4));
    if (n & 1) c = *reinterpret_cast<const unsigned*>(p + (n & 6));
    const u32x4_t rest = {two ? b[0] : c, two ? b[1] : 0u, two ? c : 0u, 0u};
    if (n & 4) r.w = rest; else r.v = rest;
  } else {
    u32x2_el2 a = {0, 0};
    unsigned b = 0, c = 0;
    if (n & 4) a = *reinterpret_cast<const u32x2_el2*>(p);
    if (n & 2) b = *reinterpret_cast<const u32_el2*>(p + (n & 4));
    if (n & 1) c = *reinterpret_cast<const uint16_t*>(p + (n & 6));
    const unsigned r0 = two ? b : c, r1 = two ? c : 0u;
    r.v = n & 4 ? u32x4_t{a[0], a[1], r0, r1} : u32x4_t{r0, r1, 0u, 0u};
  }
  return r;
}
// r without its first d values (d < 8), zeros behind: by four, two and one.
template <class T> __device__ __attribute__((always_inline)) inline Raw8<T> raw_skip(Raw8<T> r, int d) {
  const bool four = d & 4, two = d & 2, one = d & 1;
  if constexpr (sizeof(T) == 4) {
    const u32x4_t a = four ? r.w : r.v, b = four ? u32x4_t{0, 0, 0, 0} : r.w;
    const u32x4_t e = two ? u32x4_t{a[2], a[3], b[0], b[1]} : a, f = two ? u32x4_t{b[2], b[3], 0, 0} : b;
    r.v = one ? u32x4_t{e[1], e[2], e[3], f[0]} : e;
    r.w = one ? u32x4_t{f[1], f[2], f[3], 0} : f;
  } else {
    const u32x4_t a = four ? u32x4_t{r.v[2], r.v[3], 0, 0} : r.v, b = two ? u32x4_t{a[1], a[2], a[3], 0} : a;
    r.v = one ? u32x4_t{b[0] >> 16 | b[1] << 16, b[1] >> 16 | b[2] << 16, b[2] >> 16 | b[3] << 16, b[3] >> 16} : b;
  }
  return r;
}
// By word: a choice between two pieces of an array that is left to a branch puts the array into LDS.
template <class T> __device__ __attribute__((always_inline)) inline Raw8<T> raw_pick(bool first, const Raw8<T>& a, const Raw8<T>& b) {
  Raw8<T> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o.v[i] = first ? a.v[i] : b.v[i];
    if constexpr (sizeof(T) == 4) o.w[i] = first ? a.w[i] : b.w[i];
  }
  return o;
}
// `left`: values that the row still has from p on (8 or more: all of them, none: zeros)
template <class T> __device__ __attribute__((always_inline)) inline Raw8<T> raw_load(const T* p, int left) {
  if (left >= 8) return raw_load8(p);
  return left > 0 ? raw_load_part(p, left) : raw_zero<T>();
}
template <class T> __device__ __attribute__((always_inline)) inline float raw_get(const Raw8<T>& r, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float((i < 4 ? r.v : r.w)[i & 3]);
  else return __uint_as_float(i & 1 ? r.v[i >> 1] & 0xffff0000u : r.v[i >> 1] << 16);
}
// Rounds to nearest even where T is bf16.
template <class T> __device__ __attribute__((always_inline)) inline Raw8<T> raw_make(const float (&v)[8]) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.v[i] = __float_as_uint(v[i]); r.w[i] = __float_as_uint(v[i + 4]); }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 b = {(bf16_t)v[2 * i], (bf16_t)v[2 * i + 1]};
      r.v[i] = __builtin_bit_cast(unsigned, b);
    }
  }
  return r;
}
template <class T> __device__ __attribute__((always_inline)) inline void raw_store8(T* p, const Raw8<T>& r) {
  *reinterpret_cast<u32x4_el2*>(p) = r.v;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<u32x4_el2*>(p + 4) = r.w;
}
template <class T> __device__ __attribute__((always_inline)) inline void raw_store_part(T* p, int n, const Raw8<T>& r) {
  const bool four = n & 4, two = n & 2;
  if constexpr (sizeof(T) == 4) {
    const u32x4_t rest = four ? r.w : r.v;
    if (n & 4) *reinterpret_cast<u32x4_el2*>(p) = r.v;
    if (n & 2) *reinterpret_cast<u32x2_el2*>(p + (n & 4)) = u32x2_el2{rest[0], rest[1]};
    if (n & 1) *reinterpret_cast<unsigned*>(p + (n & 6)) = two ? rest[2] : rest[0];
  } else {
    const unsigned r0 = four ? r.v[2] : r.v[0], r1 = four ? r.v[3] : r.v[1];
    if (n & 4) *reinterpret_cast<u32x2_el2*>(p) = u32x2_el2{r.v[0], r.v[1]};
    if (n & 2) *reinterpret_cast<u32_el2*>(p + (n & 4)) = r0;
    if (n & 1) *reinterpret_cast<uint16_t*>(p + (n & 6)) = (uint16_t)(two ? r1 : r0);
  }
}
template <class T> __device__ __attribute__((always_inline)) inline void raw_store(T* p, int left, const Raw8<T>& r) {
  if (left >= 8) raw_store8(p, r);
  else if (left > 0) raw_store_part(p, left, r);
}

// ------------------------------------------------------------------ codes
template <int CTRL> __device__ __attribute__((always_inline)) inline unsigned dpp_max(unsigned x) {
  const unsigned y = (unsigned)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true);
  return x > y ? x : y;
}
// The largest over the 16 lanes of a DPP row, in all of them: rotations by 8, 4, 2, 1.
__device__ __attribute__((always_inline)) inline unsigned max_of_16(unsigned x) { return dpp_max<0x121>(dpp_max<0x122>(dpp_max<0x124>(dpp_max<0x128>(x)))); }

// Bits of |v|, 0 where v is not finite: what is not finite does not set a scale.
__device__ __attribute__((always_inline)) inline unsigned finite_bits(float v) {
  const unsigned b = __float_as_uint(v) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
// Scale byte of a block whose largest finite magnitude has bits `a`: largest values 1.75 * 2^8 and 1.75 * 2^15.
__device__ __attribute__((always_inline)) inline unsigned f8_scale(unsigned a, int fmt) {
  const int e = (int)(a >> 23) - (fmt == kE4M3 ? 8 : 15) + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
  return a == 0 ? 127u : (unsigned)(e > 0 ? e : 0);
}
__device__ __attribute__((always_inline)) inline float f8_scale_value(unsigned s) { return __uint_as_float(s ? s << 23 : 0x00400000u); }   // 2^(s - 127)
__device__ __attribute__((always_inline)) inline float f8_scale_inverse(unsigned s) { return __uint_as_float((254u - s) << 23); }          // (s <= 246)

// The largest scale there is: a value next to f32's end would be rounded to 2^128, and is rounded to the largest value below it instead.
__device__ __attribute__((always_inline)) inline bool f8_scale_is_last(unsigned s, int fmt) { return s == (fmt == kE4M3 ? 247u : 240u); }
__device__ __attribute__((always_inline)) inline float f8_below_end(float v, int fmt) {
  const float most = __uint_as_float(fmt == kE4M3 ? 0x7f700000u : 0x7f600000u);          // 1.875 and 1.75 times 2^127
  return finite_bits(v) > __float_as_uint(most) ? copysignf(most, v) : v;
}

// Four scaled values to codes, nearest even; none is beyond the largest, but infinities (e4m3 has none: NaN) and NaN.
__device__ __attribute__((always_inline)) inline unsigned f8_code4(float a, float b, float c, float d, int fmt) {
  int r = 0;
  if (fmt == kE4M3) {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  }
  return (unsigned)r;
}
// Eight codes to values (unscaled).
__device__ __attribute__((always_inline)) inline void f8_values8(u32x2_t c, int fmt, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (fmt == kE4M3) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
      v[4 * i] = lo[0]; v[4 * i + 1] = lo[1]; v[4 * i + 2] = hi[0]; v[4 * i + 3] = hi[1];
    } else {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)c[i], false), hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)c[i], true);
      v[4 * i] = lo[0]; v[4 * i + 1] = lo[1]; v[4 * i + 2] = hi[0]; v[4 * i + 3] = hi[1];
    }
  }
}
__device__ __attribute__((always_inline)) inline void f8_restore8(u32x2_t c, unsigned scale, int fmt, float (&v)[8]) {
  f8_values8(c, fmt, v);
  const float s = f8_scale_value(scale);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= s;
}

struct F8Out { uint8_t* codes; uint8_t* scales; int fmt, Kp, Ks; };    // codes == nullptr: not wanted

// Eight consecutive values of a block that sixteen lanes hold, `a` being the bits of the lane's largest finite magnitude: codes and the block's scale byte.
__device__ __attribute__((always_inline)) inline u32x2_t f8_pack8(float (&v)[8], unsigned a, int fmt, unsigned& s) {
  s = f8_scale(max_of_16(a), fmt);
  const float inv = f8_scale_inverse(s);
  if (f8_scale_is_last(s, fmt)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f8_below_end(v[i], fmt);
  }
  return u32x2_t{f8_code4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv, fmt), f8_code4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv, fmt)};
}

// 512 consecutive values of a row, eight a lane starting at column `col` = first column + 8 lane (values past the row's end are zeros): codes and the word of scales.
__device__ __attribute__((always_inline)) inline void f8_pack_wave(const F8Out& o, int64_t row, int col, int lane, float (&v)[8]) {
  unsigned a = 0, s;
#pragma unroll
  for (int i = 0; i < 8; ++i) { const unsigned b = finite_bits(v[i]); a = a > b ? a : b; }
  const u32x2_t c = f8_pack8(v, a, o.fmt, s);
  const unsigned word = (unsigned)__builtin_amdgcn_readlane((int)s, 0) | (unsigned)__builtin_amdgcn_readlane((int)s, 16) << 8 |
                        (unsigned)__builtin_amdgcn_readlane((int)s, 32) << 16 | (unsigned)__builtin_amdgcn_readlane((int)s, 48) << 24;
  if (col < o.Kp) *reinterpret_cast<u32x2_t*>(o.codes + row * o.Kp + col) = c;
  if (lane == 0 && col / kF8Block < o.Ks) *reinterpret_cast<unsigned*>(o.scales + row * o.Ks + col / kF8Block) = word;
}

// ------------------------------------------------------------------ pack, restore
// A wavefront takes 2048 columns of a row at a time, four loads in flight.
constexpr int kF8Steps = 4;

template <class T>
__device__ __attribute__((always_inline)) inline void f8_pack_rows(const T* x, int64_t R, int64_t ldx, int K, const F8Out& o, int block, int blocks) {
  const int lane = threadIdx.x & 63, segs = (o.Ks / 4 + kF8Steps - 1) / kF8Steps;
  const int64_t items = R * segs;
  for (int64_t it = (int64_t)block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); it < items; it += (int64_t)blocks * 4) {
    const int64_t row = it / segs;
    const int c0 = (int)(it - row * segs) * kF8Steps * 512 + lane * 8;
    Raw8<T> r[kF8Steps];
#pragma unroll
    for (int i = 0; i < kF8Steps; ++i) r[i] = raw_load(x + row * ldx + c0 + i * 512, K - c0 - i * 512);
#pragma unroll
    for (int i = 0; i < kF8Steps; ++i) {
      if ((c0 - lane * 8 + i * 512) / kF8Block >= o.Ks) break;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = raw_get(r[i], e);
      f8_pack_wave(o, row, c0 + i * 512, lane, v);
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void f8_pack_kernel(const T* x, int64_t R, int64_t ldx, int K, F8Out o) { f8_pack_rows(x, R, ldx, K, o, blockIdx.x, gridDim.x); }

template <class T>
__global__ __launch_bounds__(256) void f8_restore_kernel(const uint8_t* codes, const uint8_t* scales, int fmt, int64_t R, int K, T* x, int64_t ldx) {
  const int lane = threadIdx.x & 63, Kp = f8_code_pitch(K), Ks = f8_scale_pitch(K), segs = (Ks / 4 + kF8Steps - 1) / kF8Steps;
  const int64_t items = R * segs;
  for (int64_t it = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); it < items; it += (int64_t)gridDim.x * 4) {
    const int64_t row = it / segs;
    const int c0 = (int)(it - row * segs) * kF8Steps * 512 + lane * 8;
    u32x2_t c[kF8Steps];
    unsigned s[kF8Steps];
#pragma unroll
    for (int i = 0; i < kF8Steps; ++i) {
      const int col = c0 + i * 512;
      c[i] = u32x2_t{0, 0}; s[i] = 127;
      if (col < Kp) { c[i] = *reinterpret_cast<const u32x2_t*>(codes + row * Kp + col); s[i] = scales[row * Ks + col / kF8Block]; }
    }
#pragma unroll
    for (int i = 0; i < kF8Steps; ++i) {
      const int col = c0 + i * 512;
      float v[8];
      f8_restore8(c[i], s[i], fmt, v);
      if (col < K) raw_store(x + row * ldx + col, K - col, raw_make<T>(v));
    }
  }
}

// A weight [N, K]: one scale for 128 x 128 values, written for each of the 128 rows, so that a weight has the form every other operand has; and, if
// wanted, the transpose [K, N] with the same values.  One workgroup a block; the transpose goes through LDS.  Bound by HBM where w is large (14336 x 3584, f32 and bf16, with the
// transpose 56 and 39 us, 5.5 and 5.3 TB/s, without 41 and 34); a weight of 784 blocks is three workgroups a CU, little more than a latency each (3584 x 3584: 16.4 and 16.7 us, 4.7 and 3.1 TB/s, without 14.5 and 12.9).
template <class T>
__global__ __launch_bounds__(256) void f8_pack_weight_kernel(const T* w, int64_t ldw, int N, int K, F8Out o, F8Out t) {
  constexpr int kPitch = 132;                                        // bytes of a transposed row in LDS: words of a row's neighbours in other banks
  __shared__ unsigned most[4];
  __shared__ __attribute__((aligned(16))) uint8_t lds[128 * kPitch];
  const int n0 = blockIdx.y * 128, k0 = blockIdx.x * 128, tid = threadIdx.x, lane = tid & 63;
  const int c = (tid & 15) * 8;
  Raw8<T> r[8];
  unsigned a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int n = n0 + i * 16 + (tid >> 4);
    r[i] = n < N ? raw_load(w + (int64_t)n * ldw + k0 + c, K - k0 - c) : raw_zero<T>();
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) { const unsigned b = finite_bits(raw_get(r[i], e)); a = a > b ? a : b; }
  for (int d = 32; d > 0; d >>= 1) { const unsigned b = (unsigned)__shfl_xor((int)a, d); a = a > b ? a : b; }
  if (lane == 0) most[tid >> 6] = a;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) a = a > most[i] ? a : most[i];
  const unsigned s = f8_scale(a, o.fmt);
  const float inv = f8_scale_inverse(s);
  const bool last = f8_scale_is_last(s, o.fmt);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int q = i * 16 + (tid >> 4);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (last ? f8_below_end(raw_get(r[i], e), o.fmt) : raw_get(r[i], e)) * inv;
    const u32x2_t x = {f8_code4(v[0], v[1], v[2], v[3], o.fmt), f8_code4(v[4], v[5], v[6], v[7], o.fmt)};
    if (n0 + q < N) *reinterpret_cast<u32x2_t*>(o.codes + (int64_t)(n0 + q) * o.Kp + k0 + c) = x;
#pragma unroll
    for (int e = 0; e < 8; ++e) lds[(c + e) * kPitch + q] = (uint8_t)(x[e >> 2] >> ((e & 3) * 8));
  }
  // scale bytes; the last block of a row writes the pads behind it as well
  if (tid < 128 && n0 + tid < N) {
    uint8_t* p = o.scales + (int64_t)(n0 + tid) * o.Ks;
    p[blockIdx.x] = (uint8_t)s;
    if (blockIdx.x == gridDim.x - 1) for (int b = blockIdx.x + 1; b < o.Ks; ++b) p[b] = 127;
  }
  if (!t.codes) return;
  if (tid < 128 && k0 + tid < K) {
    uint8_t* p = t.scales + (int64_t)(k0 + tid) * t.Ks;
    p[blockIdx.y] = (uint8_t)s;
    if (blockIdx.y == gridDim.y - 1) for (int b = blockIdx.y + 1; b < t.Ks; ++b) p[b] = 127;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int q = i * 16 + (tid >> 4);                               // row of the transpose
    u32x2_t x;
    x[0] = *reinterpret_cast<const unsigned*>(lds + q * kPitch + c); x[1] = *reinterpret_cast<const unsigned*>(lds + q * kPitch + c + 4);
    if (k0 + q < K) *reinterpret_cast<u32x2_t*>(t.codes + (int64_t)(k0 + q) * t.Kp + n0 + c) = x;
  }
}

}  // namespace rlk
