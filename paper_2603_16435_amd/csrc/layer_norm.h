// layer_norm.h - layer norm over the rows of a matrix, forward and backward, with an 8-bit checkpoint of its input.
//
//   mean = sum x / H,  rstd = (sum (x - mean)^2 / H + eps)^(-1/2),  xh = (x - mean) rstd,  y = xh gamma + beta
//   g = dy gamma,  dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum_rows dy xh,  dbeta = sum_rows dy
//
// Bound by HBM: forward x and y, backward x (or its codes), dy and dx, each once.  A row is held by a team of TW wavefronts, in registers, eight
// consecutive values a lane and CH such pieces a lane, so that mean and variance are taken one after the other (no sum of squares whose difference would
// cancel) without a second read.  Statistics and sums are f32.
//
// Backward: a team walks rows far apart and keeps its columns' sums of dgamma and dbeta in registers the whole way; ROWS rows at a time, so that their
// loads are all in flight and one exchange between the wavefronts serves them all.  Each team's sums go to the workspace and ln_sum_kernel adds
// the teams' in order (no atomics: same bits every run).
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

struct NormParams { const void* gamma; const void* beta; int bf16; };
// eight parameters from column `col` on, zeros past the end
__device__ __attribute__((always_inline)) inline void norm_params(const void* p, int bf16, int col, int H, float (&v)[8]) {
  if (bf16) {
    const Raw8<bf16_t> r = raw_load((const bf16_t*)p + col, H - col);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = raw_get(r, i);
  } else {
    const Raw8<float> r = raw_load((const float*)p + col, H - col);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = raw_get(r, i);
  }
}

template <class T> struct NormFwd {
  const T* x; T* y; int64_t R, ldx, ldy; int H; float eps;
  NormParams p; float2* stats; F8Out ckpt;
};

template <class T, int TW, int CH>
__global__ __launch_bounds__(TW > 4 ? TW * 64 : 256) void ln_forward_kernel(NormFwd<T> j) {
  constexpr int NT = TW > 4 ? TW * 64 : 256, TEAMS = NT / (TW * 64);
  __shared__ float red[2][TW > 1 ? TW : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = wave % TW, team = wave / TW;
  const int c0 = (w * 64 + lane) * 8;
  const float inv_h = 1.f / (float)j.H;
  auto team_sum = [&](float s, int slot) __attribute__((always_inline)) {
    s = wave_sum(s);
    if constexpr (TW > 1) {
      if (lane == 0) red[slot][w] = s;
      __syncthreads();
      s = red[slot][0];
#pragma unroll
      for (int i = 1; i < TW; ++i) s += red[slot][i];
    }
    return s;
  };
  for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < j.R; row += (int64_t)gridDim.x * TEAMS) {
    Raw8<T> r[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) r[c] = raw_load(j.x + row * j.ldx + c0 + c * TW * 512, j.H - c0 - c * TW * 512);
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += raw_get(r[c], e);
    const float mean = team_sum(s, 0) * inv_h;
    s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int left = j.H - c0 - c * TW * 512;
#pragma unroll
      for (int e = 0; e < 8; ++e) { const float d = raw_get(r[c], e) - mean; s += e < left ? d * d : 0.f; }
    }
    const float var = team_sum(s, 1) * inv_h;
    const float rstd = 1.f / sqrtf(var + j.eps);
    if (j.stats && w == 0 && lane == 0) j.stats[row] = make_float2(mean, rstd);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = c0 + c * TW * 512, left = j.H - col;
      float g[8], b[8], v[8];
      norm_params(j.p.gamma, j.p.bf16, col, j.H, g);
      if (j.p.beta) norm_params(j.p.beta, j.p.bf16, col, j.H, b);
      else {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (raw_get(r[c], e) - mean) * rstd * g[e] + b[e];
      if (j.ckpt.codes) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = raw_get(r[c], e);
        f8_pack_wave(j.ckpt, row, col, lane, x);
      }
      raw_store(j.y + row * j.ldy + col, left, raw_make<T>(v));
    }
    // (the next row's first sum is in another slot than this row's last, and one barrier lies between a slot's reads and its next writes)
  }
}

template <class T> struct NormBwd {
  const T* dy; const T* x; T* dx; int64_t R, lddy, ldx, lddx; int H;
  const uint8_t *codes, *scales; int fmt, Kp, Ks;
  NormParams p; const float2* stats;
  float* part; int Hp;            // [teams][2][Hp]: sums of dgamma and dbeta
};

template <class T, bool CK, int TW, int CH, int ROWS>
__global__ __launch_bounds__(TW > 4 ? TW * 64 : 256) void ln_backward_kernel(NormBwd<T> j) {
  constexpr int NT = TW > 4 ? TW * 64 : 256, TEAMS = NT / (TW * 64);
  __shared__ float red[2][2 * ROWS][TW > 1 ? TW : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = wave % TW, team = blockIdx.x * TEAMS + wave / TW, teams = gridDim.x * TEAMS;
  const int c0 = (w * 64 + lane) * 8;
  const float inv_h = 1.f / (float)j.H;
  float gamma[CH][8], dg[CH][8], db[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    norm_params(j.p.gamma, j.p.bf16, c0 + c * TW * 512, j.H, gamma[c]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[c][e] = db[c][e] = 0.f;
  }
  int flip = 0;
  for (int64_t first = (int64_t)team * ROWS; first < j.R; first += (int64_t)teams * ROWS) {
    Raw8<T> rx[CK ? 1 : ROWS][CK ? 1 : CH], ry[ROWS][CH];
    u32x2_t code[CK ? ROWS : 1][CK ? CH : 1];
    unsigned scale[CK ? ROWS : 1][CK ? CH : 1];
    float2 st[ROWS];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      const bool there = first + q < j.R;
      const int64_t row = there ? first + q : first;
      st[q] = j.stats[row];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = c0 + c * TW * 512, left = j.H - col;
        ry[q][c] = raw_load(j.dy + row * j.lddy + col, there ? left : 0);
        if constexpr (CK) {
          code[q][c] = u32x2_t{0, 0}; scale[q][c] = 127;
          if (col < j.Kp) {
            code[q][c] = *reinterpret_cast<const u32x2_t*>(j.codes + row * j.Kp + col);
            scale[q][c] = j.scales[row * j.Ks + col / kF8Block];
          }
        } else rx[q][c] = raw_load(j.x + row * j.ldx + col, left);
      }
    }
    auto values = [&](int q, int c, float (&xh)[8]) __attribute__((always_inline)) {
      if constexpr (CK) f8_restore8(code[q][c], scale[q][c], j.fmt, xh);
      else {
#pragma unroll
        for (int e = 0; e < 8; ++e) xh[e] = raw_get(rx[q][c], e);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) xh[e] = (xh[e] - st[q].x) * st[q].y;
    };
    float a[ROWS], b[ROWS];                          // mean(g), mean(g xh)
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      a[q] = b[q] = 0.f;
      if (first + q < j.R) {                         // (a row that is read in the place of one that is not there adds nothing, whatever it holds)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float xh[8];
          values(q, c, xh);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float d = raw_get(ry[q][c], e), g = d * gamma[c][e];
            const float p = xh[e];
            a[q] += g; b[q] += g * p;
            dg[c][e] += d * p; db[c][e] += d;
          }
        }
      }
      a[q] = wave_sum(a[q]); b[q] = wave_sum(b[q]);
    }
    if constexpr (TW > 1) {
      if (lane == 0) {
#pragma unroll
        for (int q = 0; q < ROWS; ++q) { red[flip][2 * q][w] = a[q]; red[flip][2 * q + 1][w] = b[q]; }
      }
      __syncthreads();
#pragma unroll
      for (int q = 0; q < ROWS; ++q) {
        a[q] = red[flip][2 * q][0]; b[q] = red[flip][2 * q + 1][0];
#pragma unroll
        for (int i = 1; i < TW; ++i) { a[q] += red[flip][2 * q][i]; b[q] += red[flip][2 * q + 1][i]; }
      }
      flip ^= 1;                                     // two sets: a wavefront that is ahead writes the other one
    }
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      if (first + q >= j.R) break;
      const float ma = a[q] * inv_h, mb = b[q] * inv_h;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = c0 + c * TW * 512;
        float xh[8], v[8];
        values(q, c, xh);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = st[q].y * (raw_get(ry[q][c], e) * gamma[c][e] - ma - xh[e] * mb);
        raw_store(j.dx + (first + q) * j.lddx + col, j.H - col, raw_make<T>(v));
      }
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = c0 + c * TW * 512;
    if (col >= j.Hp) continue;
    float* p = j.part + (int64_t)team * 2 * j.Hp + col;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      *reinterpret_cast<floatx4*>(p + e) = floatx4{dg[c][e], dg[c][e + 1], dg[c][e + 2], dg[c][e + 3]};
      *reinterpret_cast<floatx4*>(p + j.Hp + e) = floatx4{db[c][e], db[c][e + 1], db[c][e + 2], db[c][e + 3]};
    }
  }
}

// Sums over the teams: a workgroup takes 64 columns of [teams][2 Hp], sixteen slices of the teams each.
__global__ __launch_bounds__(256) void ln_sum_kernel(const float* part, int teams, int Hp, int H, float* dgamma, float* dbeta) {
  __shared__ floatx4 lds[16][16];
  const int q = threadIdx.x & 15, s = threadIdx.x >> 4, col = blockIdx.x * 64 + q * 4;
  floatx4 v = {0.f, 0.f, 0.f, 0.f};
  if (col < 2 * Hp) {
    const int per = (teams + 15) / 16, end = (s + 1) * per < teams ? (s + 1) * per : teams;
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
  for (int i = 1; i < 16; ++i) v += lds[i][q];
  const bool second = col >= Hp;                     // (Hp is a multiple of 8: four columns are of one kind)
  float* o = second ? dbeta : dgamma;
  const int h = col - (second ? Hp : 0);
  if (!o) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) if (h + e < H) o[h + e] = v[e];
}

}  // namespace rlk
