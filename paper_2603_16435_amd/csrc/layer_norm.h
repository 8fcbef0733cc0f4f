// layer_norm.h - layer norm over the rows of a matrix, forward and backward, with an 8-bit checkpoint of its input.
//
//   mean = sum x / H,  rstd = (sum (x - mean)^2 / H + eps)^(-1/2),  xh = (x - mean) rstd,  y = xh gamma + beta
//   g = dy gamma,  dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum_rows dy xh,  dbeta = sum_rows dy
//
// Bound by HBM: forward x and y, backward x (or its codes), dy and dx, each once (32768 rows of 3584, bf16: 82 us, 5.7 TB/s, and 139, 5.1; with the checkpoint 114 and 125).  A row is held by a team of TW wavefronts, in registers, eight
// consecutive values a lane and CH such pieces a lane (three at most: four made registers of 300, and 5120 columns ran at 3.9 TB/s); a team walks rows far apart with the
// parameters of its columns in registers.  Sums are f32.  (Two or four rows at a time: no faster, fewer wavefronts fit a CU.)
//
// Mean and variance: a wavefront's own values give its sum and the sum of squares about its own mean, which are joined exactly
// (sum_w [q_w + n_w (mean_w - mean)^2]): no difference of large sums, and one exchange instead of two.
//
// A row of x that is not finite (a masked token's) has statistics that are not; where its dy is zero it counts as nothing and its dx is 0, because products
// of zero are zeros here (asking once a row whether its statistics are finite: 32749 rows of 3584 and their checkpoint, both ways, 328 us
// and 245).
//
// Backward: a team keeps its columns' sums of dgamma and dbeta in registers the whole way; they go to the workspace and ln_sum_kernel adds the teams' in
// order (no atomics: same bits every run).  Few rows: one launch, in which further workgroups form those sums column by column out of a second read of x and dy.
#pragma once
#include "f8_rows.h"

namespace rlk {

constexpr int kNormMaxH = 16384;

template <int CTRL, int RM> __device__ __attribute__((always_inline)) inline float dpp_add(float x) {
  return x + __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, RM, 0xF, false));
}
// Sum over the wavefront, in a scalar register: shifts by 1, 2, 4, 8 inside rows of 16 lanes, then row to row; lane 63 has it.
__device__ __attribute__((always_inline)) inline float wave_sum(float x) {
  x = dpp_add<0x111, 0xF>(x); x = dpp_add<0x112, 0xF>(x); x = dpp_add<0x114, 0xF>(x); x = dpp_add<0x118, 0xF>(x);
  x = dpp_add<0x142, 0xA>(x); x = dpp_add<0x143, 0xC>(x);
  return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
}

// Which columns of a row a lane holds: pieces of eight from c0 + c * TW * 512 on.  Where H is no multiple of eight, one lane of one wavefront has a piece
// that is not whole: its load ends with the row and is shifted in registers (bf16, 10000 rows of 1157, four wavefronts a row, forward 17.9 us, backward 26; by element 20.7 and 39).
template <int TW, int CH> struct Pieces {
  int c0, H, part;                   // part: columns of the lane's piece that is not whole, 0 if it has none
  int part_c;                        // that piece
  bool part_here;                    // it is in this wavefront (uniform)
  int held;                          // pieces of the wavefront that hold any column (uniform); the others are left out where that pays
  __device__ Pieces(int w, int lane, int H_) : c0((w * 64 + lane) * 8), H(H_) {
    const int p = H / 8;
    held = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) held += (c * TW + w) * 512 < H ? 1 : 0;
    part_c = p / (TW * 64);
    part = p % (TW * 64) == w * 64 + lane ? H % 8 : 0;
    part_here = H % 8 && p % (TW * 64) / 64 == w;
  }
  __device__ __attribute__((always_inline)) int col(int c) const { return c0 + c * TW * 512; }
  __device__ __attribute__((always_inline)) bool whole(int c) const { return col(c) + 8 <= H; }
  // Eight wavefronts a team: with 5120 columns six of them have one piece (16000 rows, forward 72 -> 66 us).  Fewer: the branch costs more than it saves (3584 columns, backward from
  // a checkpoint 114 -> 128).
  __device__ __attribute__((always_inline)) bool has(int c) const { return TW < 8 || c < held; }
  template <class T> __device__ __attribute__((always_inline)) void load(const T* row, bool there, Raw8<T> (&r)[CH]) const {
    if (H < 8) {                                     // (a row shorter than the load)
#pragma unroll
      for (int c = 0; c < CH; ++c) r[c] = c == 0 && there && part ? raw_load_part(row, part) : raw_zero<T>();
      return;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      r[c] = raw_zero<T>();
      if (there && col(c) < H) r[c] = raw_load8(row + (whole(c) ? col(c) : H - 8));
    }
    if (part_here) {
      const Raw8<T> t = raw_skip(last(r), part ? 8 - part : 0);
#pragma unroll
      for (int c = 0; c < CH; ++c) r[c] = raw_pick(c == part_c, t, r[c]);
    }
  }
  // the wavefront's pieces that hold the one that is not whole
  template <class T> __device__ __attribute__((always_inline)) Raw8<T> last(const Raw8<T> (&r)[CH]) const {
    Raw8<T> t = r[0];
#pragma unroll
    for (int c = 1; c < CH; ++c) t = raw_pick(c == part_c, r[c], t);
    return t;
  }
  template <class T> __device__ __attribute__((always_inline)) void store(T* row, const Raw8<T> (&r)[CH]) const {
#pragma unroll
    for (int c = 0; c < CH; ++c) if (whole(c)) raw_store8(row + col(c), r[c]);
    if (part_here) {
      const Raw8<T> t = last(r);
      if (part) raw_store_part(row + col(part_c), part, t);
    }
  }
  // parameters of the lane's columns, zeros past the end
  __device__ __attribute__((always_inline)) void params(const void* p, int bf16, float (&v)[CH][8]) const {
    if (bf16) {
      Raw8<bf16_t> r[CH];
      load((const bf16_t*)p, p != nullptr, r);
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = raw_get(r[c], e);
    } else {
      Raw8<float> r[CH];
      load((const float*)p, p != nullptr, r);
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = raw_get(r[c], e);
    }
  }
};

constexpr int norm_threads(int tw) { return tw > 1 ? tw * 64 : 256; }

struct NormParams { const void* gamma; const void* beta; int bf16; };
template <class T> struct NormFwd {
  const T* x; T* y; int64_t R, ldx, ldy; int H; float eps;
  NormParams p; float2* stats; F8Out ckpt;
};

template <class T, int TW, int CH>
__global__ __launch_bounds__(norm_threads(TW)) void ln_forward_kernel(NormFwd<T> j) {
  constexpr int TEAMS = norm_threads(TW) / (TW * 64);
  __shared__ float2 red[2][TW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = wave % TW, team = blockIdx.x * TEAMS + wave / TW, teams = gridDim.x * TEAMS;
  const Pieces<TW, CH> at(w, lane, j.H);
  const float inv_h = 1.f / (float)j.H;
  // columns that wavefront i of the team holds: of every run of TW * 512 its 512
  auto columns = [&](int i) __attribute__((always_inline)) {
    int n = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) { const int left = j.H - (c * TW + i) * 512; n += left < 0 ? 0 : left < 512 ? left : 512; }
    return n;
  };
  const int mine = columns(w);
  const float inv_mine = mine > 0 ? 1.f / (float)mine : 0.f;
  const int peer = lane < TW ? columns(lane) : 0;    // lane i joins what wavefront i found
  const float peer_n = (float)peer, inv_peer = peer > 0 ? 1.f / peer_n : 0.f;
  float gamma[CH][8], beta[CH][8];
  at.params(j.p.gamma, j.p.bf16, gamma);
  at.params(j.p.beta, j.p.bf16, beta);
  int flip = 0;
  constexpr bool AHEAD = TW == 8;                    // the next row on its way while one is worked on: 16000 rows of 5120 72 -> 65 us; 32749 of 3584 88 -> 93
  Raw8<T> ahead[AHEAD ? CH : 1];
  if constexpr (AHEAD) at.load(j.x + (int64_t)(team < j.R ? team : 0) * j.ldx, true, ahead);
  for (int64_t row = team; row < j.R; row += teams) {
    Raw8<T> r[CH];
    if constexpr (AHEAD) {
#pragma unroll
      for (int c = 0; c < CH; ++c) r[c] = ahead[c];
      if (row + teams < j.R) at.load(j.x + (row + teams) * j.ldx, true, ahead);
    } else at.load(j.x + row * j.ldx, true, r);
    float a = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.has(c)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) a += raw_get(r[c], e);
      }
    const float sum = wave_sum(a), m = sum * inv_mine;
    a = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.has(c)) {
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) { const float d = raw_get(r[c], e) - m; t += d * d; }
        a += at.whole(c) ? t : 0.f;
      }
    if (at.part_here) {
      const Raw8<T> t = at.last(r);
#pragma unroll
      for (int e = 0; e < 7; ++e) { const float d = raw_get(t, e) - m; a += e < at.part ? d * d : 0.f; }
    }
    float mean = m, sq = wave_sum(a);
    if constexpr (TW > 1) {
      if (lane == 0) red[flip][w] = make_float2(sum, sq);
      __syncthreads();
      const float2 p = red[flip][lane < TW ? lane : 0];
      mean = wave_sum(lane < TW ? p.x : 0.f) * inv_h;
      const float d = p.x * inv_peer - mean;
      sq = wave_sum(peer > 0 ? p.y + peer_n * d * d : 0.f);
      flip ^= 1;                                     // two sets: a wavefront that is ahead writes the other one
    }
    const float rstd = 1.f / sqrtf(sq * inv_h + j.eps);
    if (j.stats && w == 0 && lane == 0) j.stats[row] = make_float2(mean, rstd);
    if (j.ckpt.codes) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (at.has(c)) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = raw_get(r[c], e);
          f8_pack_wave(j.ckpt, row, at.col(c), lane, x);
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.has(c)) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (raw_get(r[c], e) - mean) * rstd * gamma[c][e] + beta[c][e];
        r[c] = raw_make<T>(v);
      }
    at.store(j.y + row * j.ldy, r);
  }
}

template <class T> struct NormBwd {
  const T* dy; const T* x; T* dx; int64_t R, lddy, ldx, lddx; int H;
  const uint8_t *codes, *scales; int fmt, Kp, Ks;
  NormParams p; const float2* stats;
  float* part; int Hp;            // [workgroups][2][Hp]: sums of dgamma and dbeta
  float *dgamma, *dbeta; int row_blocks;          // few rows
};

// a b, 0 where one of them is 0, whatever the other is (v_mul_legacy_f32).
__device__ __attribute__((always_inline)) inline float mul_zero(float a, float b) {
  float r;
  asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
// Team `team` of `teams`.  SUMS: dgamma, dbeta of its rows to sums [2][Hp].
template <class T, bool CK, int TW, int CH, bool SUMS>
__device__ __attribute__((always_inline)) inline void ln_backward_rows(const NormBwd<T>& j, int team, int teams, int w, int lane, float2 (&red)[2][TW], float* sums) {
  const Pieces<TW, CH> at(w, lane, j.H);
  const float inv_h = 1.f / (float)j.H;
  float gamma[CH][8], dg[SUMS ? CH : 1][8], db[SUMS ? CH : 1][8];
  at.params(j.p.gamma, j.p.bf16, gamma);
#pragma unroll
  for (int c = 0; c < (SUMS ? CH : 1); ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[c][e] = db[c][e] = 0.f;
  int flip = 0;
  for (int64_t row = team; row < j.R; row += teams) {
    Raw8<T> rx[CH], ry[CH];
    u32x2_t code[CK ? CH : 1];
    unsigned scale[CK ? CH : 1];
    const float2 st = j.stats[row];
    at.load(j.dy + row * j.lddy, true, ry);
    if constexpr (CK) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = at.col(c);
        code[c] = u32x2_t{0, 0}; scale[c] = 127;
        if (col < j.Kp) {
          code[c] = *reinterpret_cast<const u32x2_t*>(j.codes + row * j.Kp + col);
          scale[c] = j.scales[row * j.Ks + col / kF8Block];
        }
      }
    } else at.load(j.x + row * j.ldx, true, rx);
    auto normal = [&](int c, float (&xh)[8]) __attribute__((always_inline)) {
      if constexpr (CK) f8_restore8(code[c], scale[c], j.fmt, xh);
      else {
#pragma unroll
        for (int e = 0; e < 8; ++e) xh[e] = raw_get(rx[c], e);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) xh[e] = (xh[e] - st.x) * st.y;
    };
    float a = 0.f, b = 0.f;                          // mean(g), mean(g xh)
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.has(c)) {
        float xh[8];
        normal(c, xh);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = raw_get(ry[c], e), g = d * gamma[c][e];
          a += g; b += mul_zero(g, xh[e]);
          if constexpr (SUMS) { dg[c][e] += mul_zero(d, xh[e]); db[c][e] += d; }
        }
      }
    a = wave_sum(a); b = wave_sum(b);
    if constexpr (TW > 1) {
      if (lane == 0) red[flip][w] = make_float2(a, b);
      __syncthreads();
      a = red[flip][0].x; b = red[flip][0].y;
#pragma unroll
      for (int i = 1; i < TW; ++i) { a += red[flip][i].x; b += red[flip][i].y; }
      flip ^= 1;
    }
    const float ma = a * inv_h, mb = b * inv_h;
    Raw8<T> out[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (at.has(c)) {
        float xh[8], v[8];
        normal(c, xh);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = mul_zero(st.y, raw_get(ry[c], e) * gamma[c][e] - ma - mul_zero(xh[e], mb));
        out[c] = raw_make<T>(v);
      }
    at.store(j.dx + row * j.lddx, out);
  }
  if constexpr (SUMS) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = at.col(c);
      if (col >= j.Hp) continue;
      float* p = sums + col;
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        *reinterpret_cast<floatx4*>(p + e) = floatx4{dg[c][e], dg[c][e + 1], dg[c][e + 2], dg[c][e + 3]};
        *reinterpret_cast<floatx4*>(p + j.Hp + e) = floatx4{db[c][e], db[c][e + 1], db[c][e + 2], db[c][e + 3]};
      }
    }
  }
}

template <class T, bool CK, int TW, int CH>
__global__ __launch_bounds__(norm_threads(TW)) void ln_backward_kernel(NormBwd<T> j) {
  constexpr int TEAMS = norm_threads(TW) / (TW * 64);
  __shared__ float2 red[2][TW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* const out = j.part + (int64_t)blockIdx.x * 2 * j.Hp;
  if constexpr (TEAMS == 1) ln_backward_rows<T, CK, TW, CH, true>(j, blockIdx.x, gridDim.x, wave, lane, red, out);
  else {                                             // (5003 rows of 768, bf16, the teams' sums joined here 10.6 us with the sum, each to the workspace 16.0)
    __shared__ __attribute__((aligned(16))) float sums[TEAMS][2 * TW * CH * 512];
    ln_backward_rows<T, CK, TW, CH, true>(j, blockIdx.x * TEAMS + wave / TW, gridDim.x * TEAMS, wave % TW, lane, red, sums[wave / TW]);
    __syncthreads();
    for (int i = threadIdx.x * 4; i < 2 * j.Hp; i += 1024) {
      floatx4 v = *reinterpret_cast<const floatx4*>(sums[0] + i);
#pragma unroll
      for (int t = 1; t < TEAMS; ++t) v += *reinterpret_cast<const floatx4*>(sums[t] + i);
      *reinterpret_cast<floatx4*>(out + i) = v;
    }
  }
}

// dgamma, dbeta of 128 columns: sixteen lanes of eight columns, the rows dealt out among groups of such lanes.
template <class T, bool CK, int NT>
__device__ __attribute__((always_inline)) inline void ln_backward_columns(const NormBwd<T>& j, int block, float (&sums)[NT / 16][2][128]) {
  constexpr int GROUPS = NT / 16, U = 4;
  const int q = threadIdx.x & 15, grp = threadIdx.x >> 4, col = block * 128 + q * 8, left = j.H - col;
  float dg[8], db[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dg[e] = db[e] = 0.f;
  for (int64_t r0 = grp; r0 < j.R; r0 += GROUPS * U) {
    Raw8<T> ry[U], rx[U];
    u32x2_t code[U];
    unsigned scale[U];
    float2 st[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = r0 + u * GROUPS, row = r < j.R ? r : r0;
      st[u] = j.stats[row];
      ry[u] = raw_load(j.dy + row * j.lddy + col, left);
      if constexpr (CK) { code[u] = *reinterpret_cast<const u32x2_t*>(j.codes + row * j.Kp + col); scale[u] = j.scales[row * j.Ks + block]; }
      else rx[u] = raw_load(j.x + row * j.ldx + col, left);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r0 + u * GROUPS >= j.R) break;
      float xh[8];
      if constexpr (CK) f8_restore8(code[u], scale[u], j.fmt, xh);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (!CK) xh[e] = raw_get(rx[u], e);
        const float d = raw_get(ry[u], e);
        dg[e] += mul_zero(d, (xh[e] - st[u].x) * st[u].y); db[e] += d;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) { sums[grp][0][q * 8 + e] = dg[e]; sums[grp][1][q * 8 + e] = db[e]; }
  __syncthreads();
  for (int i = threadIdx.x; i < 256; i += NT) {
    const int k = i >> 7, h = block * 128 + (i & 127);
    float v = sums[0][k][i & 127];
    for (int g = 1; g < GROUPS; ++g) v += sums[g][k][i & 127];
    float* o = k ? j.dbeta : j.dgamma;
    if (o && h < j.H) o[h] = v;
  }
}

template <class T, bool CK, int TW, int CH>
__global__ __launch_bounds__(norm_threads(TW)) void ln_backward_few_kernel(NormBwd<T> j) {
  constexpr int NT = norm_threads(TW), TEAMS = NT / (TW * 64);
  __shared__ float2 red[2][TW];
  __shared__ float sums[NT / 16][2][128];
  if ((int)blockIdx.x < j.row_blocks) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    ln_backward_rows<T, CK, TW, CH, false>(j, blockIdx.x * TEAMS + wave / TW, j.row_blocks * TEAMS, wave % TW, lane, red, nullptr);
  } else ln_backward_columns<T, CK, NT>(j, (int)blockIdx.x - j.row_blocks, sums);
}

// Sums over the workgroups: one takes 32 columns of [parts][2 Hp], a line of each part, in 32 slices of the parts.
__global__ __launch_bounds__(256) void ln_sum_kernel(const float* part, int parts, int Hp, int H, float* dgamma, float* dbeta) {
  __shared__ floatx4 lds[32][8];
  const int q = threadIdx.x & 7, s = threadIdx.x >> 3, col = blockIdx.x * 32 + q * 4;
  floatx4 v = {0.f, 0.f, 0.f, 0.f};
  if (col < 2 * Hp) {
    const int per = (parts + 31) / 32, end = (s + 1) * per < parts ? (s + 1) * per : parts;
    int t = s * per;
    for (; t + 8 <= end; t += 8) {
      floatx4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const floatx4*>(part + (int64_t)(t + i) * 2 * Hp + col);
#pragma unroll
      for (int i = 0; i < 8; ++i) v += x[i];
    }
    for (; t < end; ++t) v += *reinterpret_cast<const floatx4*>(part + (int64_t)t * 2 * Hp + col);
  }
  lds[s][q] = v;
  __syncthreads();
  if (s > 0 || col >= 2 * Hp) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) v += lds[i][q];
  const bool second = col >= Hp;                     // (Hp is a multiple of 8: four columns are of one kind)
  float* o = second ? dbeta : dgamma;
  const int h = col - (second ? Hp : 0);
  if (!o) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) if (h + e < H) o[h + e] = v[e];
}

}  // namespace rlk
