// norm_linear.h - host side and C entry points of layer norm, 8-bit rows and the 8-bit linear layer (include/rl_norm_linear.h).
#pragma once
#include "../../include/rl_norm_linear.h"
#include "f8_grad.h"
#include "f8_rows.h"
#include "gemm_f8.h"
#include "layer_norm.h"

namespace rlk {

static_assert((int)kE4M3 == (int)RL_E4M3 && (int)kE5M2 == (int)RL_E5M2 && kNormMaxH == RL_LAYER_NORM_MAX_H, "header");
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - (1 << 16);
constexpr int kMaxCols = 1 << 22;                             // columns of an 8-bit operand, and rows of a weight

static bool known(int32_t dtype) { return dtype == RL_F32 || dtype == RL_BF16; }
static bool known_f8(int32_t f) { return f == RL_E4M3 || f == RL_E5M2; }
static size_t size_of(int32_t dtype) { return dtype == RL_F32 ? 4 : 2; }
static bool off(const void* p, size_t align) { return reinterpret_cast<uintptr_t>(p) % align != 0; }
static bool bad_rows(const void* p, int64_t ld, int32_t dtype, int64_t R, int64_t cols) {
  return R < 0 || R >= kMaxRows || cols < 1 || ld < cols || ld > ((int64_t)1 << 40) / (R > 0 ? R : 1) || off(p, size_of(dtype));
}
static bool bad_ws(const void* ws, size_t bytes, size_t need) { return need && (!ws || off(ws, 256) || bytes < need); }
static rl_status launched() { return hipGetLastError() == hipSuccess ? RL_OK : RL_ERR_HIP; }
static unsigned blocks_of(int64_t n, int64_t most) { return (unsigned)(n < most ? (n > 0 ? n : 1) : most); }
static F8Out f8_out(void* codes, void* scales, int fmt, int K) { return F8Out{(uint8_t*)codes, (uint8_t*)scales, fmt, f8_code_pitch(K), f8_scale_pitch(K)}; }
static F8Operand f8_operand(const void* codes, const void* scales, int64_t rows, int K) {
  return F8Operand{(const uint8_t*)codes, (const uint8_t*)scales, (int)rows, f8_code_pitch(K), f8_scale_pitch(K)};
}

// A launch has less than 2^32 threads: that many workgroups of 256.  A product has at most half as many tiles of 128 x 128, and takes smaller ones only where they are not more (f8_plan).
constexpr int64_t kMostBlocks = ((int64_t)1 << 24) - kXcds;
static bool bad_product(int64_t M, int64_t N, int64_t K) {
  return M < 0 || M >= kMaxRows || N < 1 || N > kMaxCols || K < 1 || K > kMaxCols || ((M + 127) / 128) * ((N + 127) / 128) > (1 << 23);
}

// ------------------------------------------------------------------ layer norm
// Calls f with the team of a row of H columns: wavefronts and pieces a lane as constants.  One wavefront exchanges nothing and takes its sums once, but is alone with the row's
// latency: up to 1536 columns it has the row to itself, beyond 1024 of them only where there are rows enough (bf16, 1157 columns, one wavefront of three pieces / four of one, us: forward with the
// checkpoint 64 rows 5.4 / 4.0, 1000 5.9 / 5.4, 5003 11.5 / 13.7, 20000 30.6 / 37.8; backward with its sum 600 9.5 / 9.3, 1000 9.8 / 10.5, 5003 15.2 / 18.3, 20000 32 / 37; f32: the same
// or up to 10 % less).
constexpr int kNormWideRows = 1024;
template <class F> static void with_team(int64_t R, int H, F f) {
  typedef std::integral_constant<int, 1> I1; typedef std::integral_constant<int, 2> I2;
  if (H <= 512) f(I1(), I1());
  else if (H <= 1024) f(I1(), I2());
  else if (H <= 1536 && R > kNormWideRows) f(I1(), std::integral_constant<int, 3>());
  else if (H <= 2048) f(std::integral_constant<int, 4>(), I1());
  else if (H <= 4096) f(std::integral_constant<int, 4>(), I2());
  else if (H <= 8192) f(std::integral_constant<int, 8>(), I2());
  else f(std::integral_constant<int, 16>(), I2());
}

// Workgroups: five a CU, each walking rows.  us, bf16, 768 / 1024 / 1280 workgroups: 32749 rows of 3584 89 / 88 / 87, with the checkpoint 124 / 117 / 118 (2048: 124, one a row: 162);
// 5003 rows of 2048 at 512 / 1024 / 1280 13.2 / 10.9 / 10.8 and 17.4 / 14.1 / 14.1; 3000 rows of 3584 11.3 / 10.5 / 9.9 and 14.8 / 14.2 / 13.1; 16000 rows of 5120 66 / 65 / 65 and 102 / 94 / 98.
constexpr int kNormBlocks = 1280;
template <class T>
static void run_norm_forward(const NormFwd<T>& j, hipStream_t s) {
  with_team(j.R, j.H, [&](auto tw, auto ch) {
    constexpr int TW = tw.value, CH = ch.value, NT = norm_threads(TW), TEAMS = NT / (TW * 64);
    const int64_t blocks = (j.R + TEAMS - 1) / TEAMS;
    ln_forward_kernel<T, TW, CH><<<blocks_of(blocks, kNormBlocks), NT, 0, s>>>(j);
  });
}

// Backward: one launch up to kNormFewRows rows.  us, 3584 columns, one launch / two: 128 rows 3.8 / 4.3 + 2.7, 256 5.6 / 5.3 + 3.0, 512 8.9 / 7.3 + 3.4, 1024 21.3 / 8.8 + 3.5;
// 768 columns, 512 rows 8.0 / 3.9 + 3.4; the host takes 3.5 for a launch.
// Beyond, the workgroups' sums cost 8 bytes a column and workgroup, twice: time goes as rows / workgroups and as workgroups, and is least at a multiple of the root of the rows,
// 10 sqrt(R) (192 cases of 600 to 20000 rows of 768 to 3584 columns in both types, from x and from a checkpoint, with the sum: 5.5 % behind the best of nine launches in the mean, 22 % at worst: 2175
// rows of 1024, f32, 466 workgroups 12.9, 256 10.5, a number that the sum's launch has no tail for; 1000 rows of 2048: 12.5 us, a workgroup a row 16.3).
// At most as many workgroups as keep the loads going: by the registers of a lane, four a CU up to 2048 columns, two up to 4096 (32749 rows of 3584, 512 / 768 / 1024 workgroups
// 125 / 134 / 138 us), three from a checkpoint, whose loads are shorter (133 / 114 / 141), two up to 8192 (16000 rows of 5120 93 / 107 / 101 and 95 / 112 / 98), one beyond (6000 rows of
// 12000, 256 / 512 92 / 98); two where a wavefront has a row to itself (20000 rows of 1000 22.4 / 23.3 / 24.4, of 1157 32.0 / 38.2 / 35.5).
constexpr int kNormFewRows = 512;
static int norm_pitch(int H) { return (H + 7) / 8 * 8; }
// 0: one launch
static int norm_blocks(int64_t R, int H, bool codes) {
  int blocks = 0;
  if (R > kNormFewRows) with_team(R, H, [&](auto tw, auto ch) {
    constexpr int TW = tw.value, TEAMS = norm_threads(TW) / (TW * 64), MOST = TW == 16 ? 256 : TW != 4 ? 512 : ch.value == 1 ? 1024 : 0;
    const int64_t most = MOST ? MOST : codes ? 768 : 512, root = (int64_t)(10.f * sqrtf((float)R));
    blocks = (int)blocks_of((R + TEAMS - 1) / TEAMS, root < most ? root : most);
  });
  return blocks;
}
static size_t norm_part_bytes(int64_t R, int H) { return up256((size_t)norm_blocks(R, H, true) * 2 * norm_pitch(H) * 4); }

// dx has bytes of dy or of x
template <class T>
static bool norm_in_place(const NormBwd<T>& j) {
  auto meet = [&](const T* p, int64_t ld) {
    return p && j.R && p < j.dx + (j.R - 1) * j.lddx + j.H && j.dx < p + (j.R - 1) * ld + j.H;
  };
  return meet(j.dy, j.lddy) || meet(j.x, j.ldx);
}

template <class T, bool CK>
static void run_norm_backward(NormBwd<T> j, hipStream_t s) {
  const int blocks = norm_blocks(j.R, j.H, CK && sizeof(T) == 2);
  with_team(j.R, j.H, [&](auto tw, auto ch) {
    constexpr int TW = tw.value, CH = ch.value, NT = norm_threads(TW), TEAMS = NT / (TW * 64);
    if (blocks) {
      ln_backward_kernel<T, CK, TW, CH><<<blocks, NT, 0, s>>>(j);
      ln_sum_kernel<<<(2 * j.Hp + 31) / 32, 256, 0, s>>>(j.part, blocks, j.Hp, j.H, j.dgamma, j.dbeta);
    } else if constexpr (TW > 1 || CH < 3) {                        // (three pieces a lane: only with more rows)
      static_assert(kNormFewRows <= kNormWideRows, "three pieces");
      const int rows = (int)((j.R + TEAMS - 1) / TEAMS), columns = f8_blocks(j.H);
      // the workgroups of a column read what those of a row may overwrite: then one after the other (the column's, of which there are always some, first)
      if (!norm_in_place(j)) {
        j.row_blocks = rows;
        ln_backward_few_kernel<T, CK, TW, CH><<<rows + columns, NT, 0, s>>>(j);
      } else {
        j.row_blocks = 0;
        ln_backward_few_kernel<T, CK, TW, CH><<<columns, NT, 0, s>>>(j);
        j.row_blocks = rows;
        if (rows) ln_backward_few_kernel<T, CK, TW, CH><<<rows, NT, 0, s>>>(j);
      }
    }
  });
}

// ------------------------------------------------------------------ products
// Tile and cut along K of a product.  A workgroup takes `start` us and `one` us a slab, `two` where a CU has two of them (measured, in rounds that fill the chip or part of it;
// bf16 outputs and f32 ones, whose MFMAs run at half the rate); a cut product takes a second launch and a pass over the slices.  The cheapest by that account is
// taken: 1 % behind the fastest of all tiles and cuts in the mean of 91 products of 48 to 4000 rows and seven weights of 300 x 5000 to 14336 x 3584, at most 15 % behind but for one
// of 8 us (us, by tiles of 32 x 32 / 64 x 64 / 64 x 128 / 128 x 128 / 256 x 256, each with its best cut, 3584 columns and rows of w: 48 rows 7.9 / 8.4 / - / - / -;
// 250 16.7 / 11.7 / 15.3 / 18.2 / 32.5; 1000 - / 27.1 / 23.0 / 26.7 / 35.2; 2000 - / 53.0 / 43.4 / 31.3 / 36.1; 4000 - / - / - / 61.9 / 37.0).
struct F8Tile { int bm, bn; float start[2], one[2], two[2]; };
constexpr F8Tile kF8Tiles[] = {
    {32, 32, {2.7f, 3.2f}, {0.17f, 0.23f}, {0.20f, 0.31f}},
    {64, 64, {3.2f, 3.4f}, {0.28f, 0.47f}, {0.39f, 0.65f}},
    {64, 128, {3.9f, 4.4f}, {0.43f, 0.70f}, {0.67f, 1.06f}},
    {128, 128, {4.4f, 4.7f}, {0.68f, 1.15f}, {0.95f, 1.69f}},
    {256, 256, {7.0f, 0.f}, {1.15f, 0.f}, {0.f, 0.f}},               // hot kernel: bf16 outputs, one workgroup a CU, not cut
};
constexpr int kF8Hot = 4;
struct F8Plan { int tile, slices, per; size_t part; int Np; };
static F8Plan f8_plan(int64_t M, int N, int K, bool exact) {
  const int nk = f8_blocks(K), whole = (nk + 3) / 4 * 4;
  F8Plan best{0, 1, whole, 0, (N + 3) / 4 * 4};
  float least = 3e38f;
  for (int t = 0; t <= kF8Hot - (exact ? 1 : 0); ++t) {
    const F8Tile& c = kF8Tiles[t];
    const int64_t tiles = ((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
    if (tiles > kMostBlocks) continue;
    for (int slices = 1; slices <= 16 && slices <= (nk + 3) / 4; ++slices) {
      if (slices > 1 && (t == kF8Hot || tiles * slices > 512)) break;
      const int per = slices > 1 ? ((nk + slices - 1) / slices + 3) / 4 * 4 : whole;          // whole words of scales
      if ((nk + per - 1) / per != slices) continue;
      const int64_t n = tiles * slices;
      const float len = (float)(slices > 1 ? per : nk), one = c.start[exact] + c.one[exact] * len, two = c.start[exact] + c.two[exact] * len;
      float us;
      if (t == kF8Hot) us = (float)((n + 255) / 256) * one;
      else { const int64_t left = n % 512; us = (float)(n / 512) * two + (left == 0 ? 0.f : left <= 256 ? one : two); }
      if (slices > 1) us += 2.4f + (float)M * (float)N * (float)(slices + 1) * 1e-6f;
      if (us < least) { least = us; best.tile = t; best.slices = slices; best.per = per; }
    }
  }
  if (best.slices > 1) best.part = up256((size_t)best.slices * M * best.Np * 4);
  return best;
}

template <int FX, int FW, class T>
static void run_f8_tiles(const F8Operand& x, const F8Operand& w, int K, T* y, int64_t ldy, void* ws, hipStream_t s) {
  const F8Plan p = f8_plan(x.rows, w.rows, K, kExact<T>);
  if constexpr (!kExact<T>)
    if (p.tile == kF8Hot) {
      f8_hot_kernel<FX, FW><<<launch_tiles((x.rows + 255) / 256, (w.rows + 255) / 256), 256, 0, s>>>(F8Hot{x, w, y, ldy, x.rows, w.rows, f8_blocks(K)});
      return;
    }
  const F8Product<T> j{x, w, y, ldy, x.rows, w.rows, f8_blocks(K), p.slices, p.per, (float*)ws, p.Np};
  const F8Tile& c = kF8Tiles[p.tile];
  const int64_t n = (int64_t)((x.rows + c.bm - 1) / c.bm) * ((w.rows + c.bn - 1) / c.bn) * p.slices;
  const unsigned blocks = (unsigned)((n + kXcds - 1) / kXcds * kXcds);
  if (p.tile == 0) f8_gemm_kernel<FX, FW, T, 32, 32, 6><<<blocks, 256, 0, s>>>(j);
  else if (p.tile == 1) f8_gemm_kernel<FX, FW, T, 64, 64, 4><<<blocks, 256, 0, s>>>(j);
  else if (p.tile == 2) f8_gemm_kernel<FX, FW, T, 64, 128, 3><<<blocks, 256, 0, s>>>(j);
  else f8_gemm_kernel<FX, FW, T, 128, 128, 2><<<blocks, 256, 0, s>>>(j);
  if (p.slices > 1) f8_slices_kernel<T><<<blocks_of(((int64_t)x.rows * p.Np / 4 + 255) / 256, 4096), 256, 0, s>>>(j.part, p.slices, j.M, j.N, p.Np, y, ldy);
}
// One workgroup of the few-rows kernel a CU; with more slabs than its wavefronts have on their way the tiles do better.
static bool f8_few(int64_t M, int N, int K) { return M <= kF8FewRows && N <= 16 * 256 && f8_blocks(K) <= 32; }
// Packing x in every workgroup instead of a launch ahead: up to so many bytes of codes, times the rounds of workgroups (3584 columns; 3584 rows of w: 4 rows of x 6.2 us and 5.2 + 3.3,
// 8 rows 8.4 and 5.4 + 3.3; 14336: 1 row 12.3 and 10.9 + 3.3, 4 rows 15.7).
static bool f8_takes_raw(int64_t M, int N, int K) { return M <= kF8FewRows && M * f8_raw_pitch(f8_code_pitch(K)) * ((N + 4095) / 4096) <= 28800; }
template <int FX, int FW, class T>
static void run_f8_few_of(const F8Operand& x, const F8Operand& w, const T* raw, int64_t ldx, int K, T* y, int64_t ldy, hipStream_t s) {
  const F8Few<T> j{x, w, raw, ldx, K, y, ldy, x.rows, w.rows, f8_blocks(K)};
  const int blocks = (w.rows + 15) / 16, nt = kF8FewWaves * 64;
  if (raw) f8_few_kernel<FX, FW, T, true><<<blocks, nt, x.rows * (f8_raw_pitch(x.Kp) + x.Ks), s>>>(j);
  else f8_few_kernel<FX, FW, T, false><<<blocks, nt, 0, s>>>(j);
}
// raw: x as it is (f8_takes_raw), or nullptr
template <class T>
static void run_f8_product(const F8Operand& x, int fx, const F8Operand& w, int fw, const T* raw, int64_t ldx, int K, T* y, int64_t ldy, void* ws, hipStream_t s) {
  auto go = [&](auto FX, auto FW) {
    if (raw || f8_few(x.rows, w.rows, K)) run_f8_few_of<FX.value, FW.value, T>(x, w, raw, ldx, K, y, ldy, s);
    else run_f8_tiles<FX.value, FW.value, T>(x, w, K, y, ldy, ws, s);
  };
  typedef std::integral_constant<int, 0> E4;
  typedef std::integral_constant<int, 1> E5;
  if (fx == RL_E4M3) { if (fw == RL_E4M3) go(E4(), E4()); else go(E4(), E5()); }
  else { if (fw == RL_E4M3) go(E5(), E4()); else go(E5(), E5()); }
}
// (either type of y: the larger of the two)
static size_t f8_product_bytes(int64_t M, int N, int K) {
  if (f8_few(M, N, K)) return 0;
  const size_t a = f8_plan(M, N, K, false).part, b = f8_plan(M, N, K, true).part;
  return a > b ? a : b;
}
struct F8ForwardPlan { size_t codes, scales, mm, total; bool raw; };
static F8ForwardPlan f8_forward_plan(int64_t M, int N, int K, bool keep) {
  F8ForwardPlan p{};
  p.raw = f8_takes_raw(M, N, K);
  if (!keep && !p.raw) { p.scales = up256((size_t)M * f8_code_pitch(K)); p.mm = p.scales + up256((size_t)M * f8_scale_pitch(K)); }
  p.total = p.mm + (p.raw ? 0 : f8_product_bytes(M, N, K));
  return p;
}

template <class T> static void run_f8_pack(const T* x, int64_t ldx, int64_t R, int K, const F8Out& o, hipStream_t s) {
  const int segs = (o.Ks / 4 + kF8Steps - 1) / kF8Steps;
  f8_pack_kernel<T><<<blocks_of((R * segs + 3) / 4, 1 << 16), 256, 0, s>>>(x, R, ldx, K, o);
}

// ------------------------------------------------------------------ backward of the linear layer
// The launch that prepares the contractions has a workgroup for 64 tokens of a chunk and 128 k, and those that pack and copy dy; the weight gradient's one for 256 x 256 values
// (with K's tiles rounded up to the XCDs).
constexpr int kPackBlocks = 1 << 16, kCopyBlocks = 1 << 13;
static bool bad_gradient(int64_t M, int64_t N, int64_t K) {
  if (bad_product(M, N, K) || bad_product(M, K, N)) return true;
  const int64_t tokens = M < kGradChunk ? (M + 127) / 128 * 128 : kGradChunk;
  return tokens / 64 * f8_blocks((int)K) > kMostBlocks - kPackBlocks - kCopyBlocks || ((K + 255) / 256 + kXcds) * ((N + 255) / 256) > kMostBlocks;
}

// bf16 rows of dy that lie on 16 bytes are read where they are, others and f32 go through the workspace.
static bool f8_grad_direct(int32_t dtype, int N, int64_t lddy, bool aligned) { return dtype == RL_BF16 && N % 8 == 0 && lddy % 8 == 0 && aligned && lddy < (1 << 23); }
// slices: of the weight gradient's contraction over a whole chunk, and over the tokens that are left
struct F8GradPlan { size_t codes, scales, mm, xt, terms, part, total; int chunk, copies, Np; bool raw, direct; SplitK slices[2]; };
// Only what a call for these outputs touches: at 32749 x 3584 x 3584, bf16, 353 MB, and 235 more where dy has to be copied; 118 for dx alone (3001 x 1157 x 1163, f32: 97).
static F8GradPlan f8_grad_plan(int64_t M, int N, int K, int32_t dtype, bool dx, bool dW, bool direct) {
  F8GradPlan p{};
  size_t o = 0;
  auto take = [&](size_t n) { const size_t at = o; o += up256(n); return at; };
  p.raw = dx && f8_takes_raw(M, K, N);                             // (packed where it is multiplied)
  p.direct = direct;
  if (dx && !p.raw) {
    p.codes = take((size_t)M * f8_code_pitch(N));
    p.scales = take((size_t)M * f8_scale_pitch(N));
    p.mm = take(f8_product_bytes(M, K, N));
  }
  p.copies = dtype == RL_F32 ? kGradTerms : 1;
  const int most = kGradChunk / p.copies / 128 * 128;
  p.chunk = (int)(M < most ? (M + 127) / 128 * 128 : most);
  p.Np = (N + 7) / 8 * 8;
  if (dW && M) {
    p.xt = take((size_t)p.copies * p.chunk * ((K + 255) / 256 * 256) * 2);
    if (!direct) p.terms = take((size_t)p.copies * p.chunk * p.Np * 2);
    const int tiles = ((K + kBM - 1) / kBM) * ((p.Np + kBN - 1) / kBN);
    auto cut = [&](int64_t tokens) { return split_k_host(tiles, (int)((tokens + 127) / 128) * p.copies, kHotSlots, 0); };
    if (M >= p.chunk) p.slices[0] = cut(p.chunk);
    if (M % p.chunk) p.slices[1] = cut(M % p.chunk);
    const int slices = p.slices[0].slices > p.slices[1].slices ? p.slices[0].slices : p.slices[1].slices;
    p.part = take(slices > 1 ? (size_t)slices * N * ((K + 3) / 4 * 4) * 4 : 0);
  }
  p.total = o;
  return p;
}

// One launch prepares both contractions of the first chunk; a chunk that follows has its x^T and dy prepared ahead of its contraction.
template <class T>
static void run_f8_backward(const T* dy, int64_t lddy, int64_t M, int N, int K, int fdy, const F8Operand& x, int fx, const F8Operand& wt, int fw, T* dx, int64_t lddx,
                            float* dW, int64_t lddw, bool accumulate, unsigned char* ws, const F8GradPlan& p, hipStream_t s) {
  bf16_t* xt = (bf16_t*)(ws + p.xt);
  bf16_t* terms = (bf16_t*)(ws + p.terms);
  const bool direct = p.direct, raw = p.raw;
  for (int64_t t0 = 0; t0 < M; t0 += p.chunk) {
    const int tokens = (int)(M - t0 < p.chunk ? M - t0 : p.chunk), pad = (tokens + 127) / 128 * 128;
    F8GradPrep<T> j{};
    j.dy = dy; j.lddy = lddy; j.M = M; j.N = N; j.packed = f8_out(ws + p.codes, ws + p.scales, fdy, N);
    if (dx && t0 == 0 && !raw) j.pack_blocks = (int)blocks_of((M * ((j.packed.Ks / 4 + kF8Steps - 1) / kF8Steps) + 3) / 4, kPackBlocks);
    int copy_blocks = 0;
    if (dW) {
      j.codes = x.codes + t0 * x.Kp; j.scales = x.scales + t0 * x.Ks; j.fmt = fx; j.tokens = tokens; j.Kp = x.Kp; j.Ks = x.Ks;
      j.xt = xt; j.pad = pad; j.copies = p.copies; j.restore_blocks = pad / 64 * f8_blocks(K);
      j.chunk = dy + t0 * lddy; j.Np = p.Np; j.terms = terms;
      if (!direct) copy_blocks = (int)blocks_of(((int64_t)pad * p.Np / 8 + 255) / 256, kCopyBlocks);
    }
    const int blocks = j.pack_blocks + j.restore_blocks + copy_blocks;
    if (blocks) f8_grad_prep_kernel<T><<<blocks, 256, 0, s>>>(j);
    if (dx && t0 == 0) run_f8_product<T>(f8_operand(raw ? nullptr : ws + p.codes, raw ? nullptr : ws + p.scales, M, N), fdy, wt, fw, raw ? dy : nullptr, lddy, N, dx, lddx, ws + p.mm, s);
    if (!dW) return;
    GemmDims d{};
    d.M = K; d.N = direct ? N : p.Np; d.K = p.copies * pad; d.lda = d.K; d.ldb = direct ? lddy : p.Np;
    d.group_m = 8; d.split_slots = kHotSlots; d.b_k_rows = direct ? tokens : d.K;
    const bool add = accumulate || t0 > 0;
    const int tm = (d.M + kBM - 1) / kBM, tn = (d.N + kBN - 1) / kBN;
    const SplitK sk = p.slices[tokens == p.chunk ? 0 : 1];          // (a step is 128 tokens, two slabs)
    const int64_t ldp = (K + 3) / 4 * 4;
    const EpiF8Grad e{dW, lddw, N, K, add, (float*)(ws + p.part), ldp};
    f8_grad_kernel<TuneDX><<<split_launch(tm, tn, kHotSlots), 256, 0, s>>>(xt, direct ? (const bf16_t*)(dy + t0 * lddy) : terms, d, e);
    if (sk.slices > 1) f8_grad_slices_kernel<<<blocks_of(((int64_t)N * (ldp / 4) + 255) / 256, 4096), 256, 0, s>>>(e.part, sk.slices, N, K, ldp, dW, lddw, add);
  }
}

__global__ __launch_bounds__(256) void f8_zero_kernel(float* dW, int64_t ld, int N, int K) {
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < (int64_t)N * K; q += (int64_t)gridDim.x * 256) dW[q / K * ld + q % K] = 0.f;
}

}  // namespace rlk

// ------------------------------------------------------------------ C entry points
using namespace rlk;

extern "C" {

int64_t rl_f8_code_pitch(int32_t K) { return K > 0 && K <= kMaxCols ? f8_code_pitch(K) : 0; }
int64_t rl_f8_scale_pitch(int32_t K) { return K > 0 && K <= kMaxCols ? f8_scale_pitch(K) : 0; }

rl_status rl_layer_norm_forward(const void* x, int64_t ldx, int32_t dtype, int64_t R, int32_t H, const void* gamma, const void* beta,
                                int32_t param_dtype, float eps, void* y, int64_t ldy, float* stats, void* codes, void* scales,
                                int32_t format, void* stream) {
  if (!gamma || (R != 0 && (!x || !y)) || !codes != !scales) return RL_ERR_NULL;
  if (!known(dtype) || !known(param_dtype) || (codes && !known_f8(format))) return RL_ERR_DTYPE;
  if (H > kNormMaxH || bad_rows(x, ldx, dtype, R, H) || bad_rows(y, ldy, dtype, R, H) || off(gamma, size_of(param_dtype)) ||
      off(beta, size_of(param_dtype)) || off(codes, 16) || off(scales, 16) || off(stats, 8)) return RL_ERR_SHAPE;
  if (!(eps >= 0.f) || !__builtin_isfinite(eps)) return RL_ERR_RANGE;
  if (R == 0) return RL_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const NormParams p{gamma, beta, param_dtype == RL_BF16};
  const F8Out o = f8_out(codes, scales, format, H);
  if (dtype == RL_BF16) run_norm_forward(NormFwd<bf16_t>{(const bf16_t*)x, (bf16_t*)y, R, ldx, ldy, H, eps, p, (float2*)stats, o}, s);
  else run_norm_forward(NormFwd<float>{(const float*)x, (float*)y, R, ldx, ldy, H, eps, p, (float2*)stats, o}, s);
  return launched();
}

rl_status rl_layer_norm_backward_workspace_bytes(int64_t R, int32_t H, size_t* bytes) {
  if (!bytes) return RL_ERR_NULL;
  if (R < 0 || R >= kMaxRows || H < 1 || H > kNormMaxH) return RL_ERR_SHAPE;
  *bytes = norm_part_bytes(R, H);
  return RL_OK;
}

rl_status rl_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* codes, const void* scales, int32_t format,
                                 int32_t dtype, int64_t R, int32_t H, const void* gamma, int32_t param_dtype, const float* stats,
                                 void* dx, int64_t lddx, float* dgamma, float* dbeta, void* ws, size_t ws_bytes, void* stream) {
  if (!gamma || !dgamma || (R != 0 && (!dy || !dx || !stats || (!x && (!codes || !scales))))) return RL_ERR_NULL;
  if (x && (codes || scales)) return RL_ERR_NULL;                  // one of the two
  if (!known(dtype) || !known(param_dtype) || (codes && !known_f8(format))) return RL_ERR_DTYPE;
  if (H > kNormMaxH || bad_rows(dy, lddy, dtype, R, H) || bad_rows(dx, lddx, dtype, R, H) || (x && bad_rows(x, ldx, dtype, R, H)) ||
      off(gamma, size_of(param_dtype)) || off(codes, 16) || off(scales, 16) || off(stats, 8) || off(dgamma, 16) || off(dbeta, 16)) return RL_ERR_SHAPE;
  if (bad_ws(ws, ws_bytes, norm_part_bytes(R, H))) return RL_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  auto go = [&](auto zero) {
    typedef decltype(zero) T;
    const NormBwd<T> j{(const T*)dy, (const T*)x, (T*)dx, R, lddy, ldx, lddx, H, (const uint8_t*)codes, (const uint8_t*)scales, format,
                       f8_code_pitch(H), f8_scale_pitch(H), NormParams{gamma, nullptr, param_dtype == RL_BF16}, (const float2*)stats, (float*)ws, norm_pitch(H), dgamma, dbeta, 0};
    if (codes) run_norm_backward<T, true>(j, s); else run_norm_backward<T, false>(j, s);
  };
  if (dtype == RL_BF16) go(bf16_t()); else go(float());
  return launched();
}

rl_status rl_f8_pack(const void* x, int64_t ldx, int32_t dtype, int64_t R, int32_t K, int32_t format, void* codes, void* scales, void* stream) {
  if (R != 0 && (!x || !codes || !scales)) return RL_ERR_NULL;
  if (!known(dtype) || !known_f8(format)) return RL_ERR_DTYPE;
  if (K > kMaxCols || bad_rows(x, ldx, dtype, R, K) || off(codes, 16) || off(scales, 16)) return RL_ERR_SHAPE;
  if (R == 0) return RL_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const F8Out o = f8_out(codes, scales, format, K);
  if (dtype == RL_BF16) run_f8_pack((const bf16_t*)x, ldx, R, K, o, s); else run_f8_pack((const float*)x, ldx, R, K, o, s);
  return launched();
}

rl_status rl_f8_unpack(const void* codes, const void* scales, int32_t format, int64_t R, int32_t K, void* x, int64_t ldx, int32_t dtype, void* stream) {
  if (R != 0 && (!x || !codes || !scales)) return RL_ERR_NULL;
  if (!known(dtype) || !known_f8(format)) return RL_ERR_DTYPE;
  if (K > kMaxCols || bad_rows(x, ldx, dtype, R, K) || off(codes, 16) || off(scales, 16)) return RL_ERR_SHAPE;
  if (R == 0) return RL_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const int segs = (f8_scale_pitch(K) / 4 + kF8Steps - 1) / kF8Steps;
  const unsigned blocks = blocks_of((R * segs + 3) / 4, 1 << 16);
  if (dtype == RL_BF16) f8_restore_kernel<bf16_t><<<blocks, 256, 0, s>>>((const uint8_t*)codes, (const uint8_t*)scales, format, R, K, (bf16_t*)x, ldx);
  else f8_restore_kernel<float><<<blocks, 256, 0, s>>>((const uint8_t*)codes, (const uint8_t*)scales, format, R, K, (float*)x, ldx);
  return launched();
}

rl_status rl_f8_pack_weight(const void* w, int64_t ldw, int32_t dtype, int32_t N, int32_t K, int32_t format, void* codes, void* scales,
                            void* codes_t, void* scales_t, void* stream) {
  if (!w || !codes || !scales || !codes_t != !scales_t) return RL_ERR_NULL;
  if (!known(dtype) || !known_f8(format)) return RL_ERR_DTYPE;
  if (N < 1 || N > kMaxCols || K > kMaxCols || bad_rows(w, ldw, dtype, N, K) || off(codes, 16) || off(scales, 16) || off(codes_t, 16) || off(scales_t, 16)) return RL_ERR_SHAPE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const dim3 grid(f8_blocks(K), f8_blocks(N));
  const F8Out o = f8_out(codes, scales, format, K), t = f8_out(codes_t, scales_t, format, N);
  if (dtype == RL_BF16) f8_pack_weight_kernel<bf16_t><<<grid, 256, 0, s>>>((const bf16_t*)w, ldw, N, K, o, t);
  else f8_pack_weight_kernel<float><<<grid, 256, 0, s>>>((const float*)w, ldw, N, K, o, t);
  return launched();
}

rl_status rl_f8_matmul_workspace_bytes(int64_t M, int32_t N, int32_t K, size_t* bytes) {
  if (!bytes) return RL_ERR_NULL;
  if (bad_product(M, N, K)) return RL_ERR_SHAPE;
  *bytes = f8_product_bytes(M, N, K);
  return RL_OK;
}

rl_status rl_f8_matmul(const void* x_codes, const void* x_scales, int32_t x_format, const void* w_codes, const void* w_scales, int32_t w_format,
                       int64_t M, int32_t N, int32_t K, void* y, int64_t ldy, int32_t dtype, void* ws, size_t ws_bytes, void* stream) {
  if (!w_codes || !w_scales || (M != 0 && (!x_codes || !x_scales || !y))) return RL_ERR_NULL;
  if (!known(dtype) || !known_f8(x_format) || !known_f8(w_format)) return RL_ERR_DTYPE;
  size_t need = 0;
  if (rl_f8_matmul_workspace_bytes(M, N, K, &need) != RL_OK || bad_rows(y, ldy, dtype, M, N) || off(x_codes, 16) || off(x_scales, 16) || off(w_codes, 16) || off(w_scales, 16))
    return RL_ERR_SHAPE;
  if (bad_ws(ws, ws_bytes, need)) return RL_ERR_WORKSPACE;
  if (M == 0) return RL_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const F8Operand x = f8_operand(x_codes, x_scales, M, K), w = f8_operand(w_codes, w_scales, N, K);
  if (dtype == RL_BF16) run_f8_product<bf16_t>(x, x_format, w, w_format, nullptr, 0, K, (bf16_t*)y, ldy, ws, s);
  else run_f8_product<float>(x, x_format, w, w_format, nullptr, 0, K, (float*)y, ldy, ws, s);
  return launched();
}

rl_status rl_f8_linear_forward_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t keep, size_t* bytes) {
  if (!bytes) return RL_ERR_NULL;
  if (bad_product(M, N, K)) return RL_ERR_SHAPE;
  *bytes = f8_forward_plan(M, N, K, keep != 0).total;
  return RL_OK;
}

rl_status rl_f8_linear_forward(const void* x, int64_t ldx, int32_t dtype, int64_t M, int32_t K, int32_t x_format, const void* w_codes,
                               const void* w_scales, int32_t w_format, int32_t N, void* y, int64_t ldy, void* x_codes, void* x_scales,
                               void* ws, size_t ws_bytes, void* stream) {
  if (!w_codes || !w_scales || (M != 0 && (!x || !y)) || !x_codes != !x_scales) return RL_ERR_NULL;
  if (!known(dtype) || !known_f8(x_format) || !known_f8(w_format)) return RL_ERR_DTYPE;
  if (bad_product(M, N, K) || bad_rows(x, ldx, dtype, M, K) || bad_rows(y, ldy, dtype, M, N) || off(x_codes, 16) || off(x_scales, 16) ||
      off(w_codes, 16) || off(w_scales, 16)) return RL_ERR_SHAPE;
  const F8ForwardPlan p = f8_forward_plan(M, N, K, x_codes != nullptr);
  if (bad_ws(ws, ws_bytes, p.total)) return RL_ERR_WORKSPACE;
  if (M == 0) return RL_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  unsigned char* o = static_cast<unsigned char*>(ws);
  if (!x_codes && !p.raw) { x_codes = o + p.codes; x_scales = o + p.scales; }
  const F8Operand xo = f8_operand(x_codes, x_scales, M, K), w = f8_operand(w_codes, w_scales, N, K);
  auto go = [&](auto zero) {
    typedef decltype(zero) T;
    if (!p.raw) run_f8_pack((const T*)x, ldx, M, K, f8_out(x_codes, x_scales, x_format, K), s);
    run_f8_product<T>(xo, x_format, w, w_format, p.raw ? (const T*)x : nullptr, ldx, K, (T*)y, ldy, o + p.mm, s);
  };
  if (dtype == RL_BF16) go(bf16_t()); else go(float());
  return launched();
}

rl_status rl_f8_linear_backward_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t dtype, size_t* bytes) {
  if (!bytes) return RL_ERR_NULL;
  if (!known(dtype)) return RL_ERR_DTYPE;
  if (bad_gradient(M, N, K)) return RL_ERR_SHAPE;
  *bytes = f8_grad_plan(M, N, K, dtype, true, true, false).total;
  return RL_OK;
}

rl_status rl_f8_linear_backward_workspace_bytes_for(int64_t M, int32_t N, int32_t K, int32_t dtype, int64_t lddy, int32_t dy_aligned, int32_t want_dx, int32_t want_dW, size_t* bytes) {
  if (!bytes) return RL_ERR_NULL;
  if (!known(dtype)) return RL_ERR_DTYPE;
  if (bad_gradient(M, N, K) || lddy < N) return RL_ERR_SHAPE;
  *bytes = f8_grad_plan(M, N, K, dtype, want_dx != 0, want_dW != 0, f8_grad_direct(dtype, N, lddy, dy_aligned != 0)).total;
  return RL_OK;
}

rl_status rl_f8_linear_backward(const void* dy, int64_t lddy, int32_t dtype, int64_t M, int32_t N, int32_t K, int32_t dy_format,
                                const void* x_codes, const void* x_scales, int32_t x_format, const void* wt_codes, const void* wt_scales, int32_t w_format,
                                void* dx, int64_t lddx, float* dW, int64_t lddw, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  if ((!dx && !dW && M != 0) || (M != 0 && !dy) || (dx && (!wt_codes || !wt_scales)) || (dW && M != 0 && (!x_codes || !x_scales))) return RL_ERR_NULL;
  if (!known(dtype) || (dx && (!known_f8(dy_format) || !known_f8(w_format))) || (dW && !known_f8(x_format))) return RL_ERR_DTYPE;
  if (bad_gradient(M, N, K) || bad_rows(dy, lddy, dtype, M, N) || (dx && bad_rows(dx, lddx, dtype, M, K)) ||
      (dW && (lddw < K || off(dW, 4))) || off(x_codes, 16) || off(x_scales, 16) || off(wt_codes, 16) || off(wt_scales, 16)) return RL_ERR_SHAPE;
  const F8GradPlan p = f8_grad_plan(M, N, K, dtype, dx != nullptr, dW != nullptr, f8_grad_direct(dtype, N, lddy, !off(dy, 16)));
  if (bad_ws(ws, ws_bytes, p.total)) return RL_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (M == 0) {
    if (dW && !accumulate) f8_zero_kernel<<<blocks_of(((int64_t)N * K + 255) / 256, 4096), 256, 0, s>>>(dW, lddw, N, K);
    return launched();
  }
  unsigned char* w = static_cast<unsigned char*>(ws);
  auto go = [&](auto zero) {
    typedef decltype(zero) T;
    run_f8_backward((const T*)dy, lddy, M, N, K, dy_format, f8_operand(x_codes, x_scales, M, K), x_format, f8_operand(wt_codes, wt_scales, K, N), w_format, (T*)dx, lddx,
                    dW, lddw, accumulate != 0, w, p, s);
  };
  if (dtype == RL_BF16) go(bf16_t()); else go(float());
  return launched();
}

}  // extern "C"
