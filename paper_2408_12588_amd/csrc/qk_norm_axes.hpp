// Norm of queries and keys per head, and their rotation by the token's place on up to three axes (frame, row, column), in one pass.
//
//   y = (x - mean) / sqrt(var + eps) * gamma + beta      layernorm over the head dimension (biased variance), or
//   y = x / sqrt(mean(x^2) + eps) * gamma + beta         root mean square, or  y = x * gamma + beta
//   neighbouring pairs (y[2i], y[2i+1]) turned by the angle of pair i: the features of a head are cut into one section per axis and
//   a remainder that is not turned; (cos, sin) of every place and pair of an axis come from a table that the caller keeps.
//
// The table instead of angles computed here: it is (T dt + Y dy + X dx) / 2 pairs, a few KB that stay in L1, where the angle of a far place
// needs fp64 to be right.  Bound by HBM, q and k read and written once.  LPR neighbouring lanes share a (token, head) row, 8 features each,
// so that every load and store of a wavefront is one contiguous stretch; a lane has the same features of the same token's q and k,
// whose factors it therefore loads once.  25440 tokens of 16 heads of 72 (234 MB): 48 us, 4.9 TB/s, where a copy reaches 5.1; with one group of rows per
// wavefront, gamma and beta unpacked each time, 65; an earlier form with three lanes per row, 24 features each, which read 16 bytes in every 48, took 71.
#pragma once
#include "q8_common.hpp"
#include "rope_table.hpp"

namespace pab {

enum { NORM_NONE = 0, NORM_LAYER = 1, NORM_RMS = 2 };

struct QkAxesParams {
  const void *q, *k;                 // token pitches ld_q, ld_k elements
  void *q_out, *k_out;
  const void *gq, *bq, *gk, *bk;     // [D] or nullptr
  const f32x2 *factors;              // axis by axis, place by place, pair by pair
  long long ld_q, ld_k, ld_q_out, ld_k_out;
  int heads_q, heads_k;
  unsigned n_row;                    // tokens * max(heads_q, heads_k)
  Divisor heads, tokens, YX, X;      // rows per token, tokens per batch, tokens per frame, tokens per row
  int end_t, end_y, end_x;           // first pair behind each axis's section
  int first_y, first_x;              // where the axes' tables start, in pairs
  int whole;                         // every section is a multiple of 8 features
  float eps;
};

// sum over the LPR lanes of a row, in all of them
template <int LPR>
__device__ __forceinline__ float row_sum(float s, int first) {
  auto moved = [](float x, auto ctrl) {
    return __uint_as_float((unsigned)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  if constexpr (LPR == 4 || LPR == 8 || LPR == 16) {
    s += moved(s, std::integral_constant<int, 0xB1>{});
    s += moved(s, std::integral_constant<int, 0x4E>{});
    if constexpr (LPR >= 8) s += moved(s, std::integral_constant<int, 0x141>{});
    if constexpr (LPR >= 16) s += moved(s, std::integral_constant<int, 0x140>{});
    return s;
  } else {   // the sums of the lanes behind, one lane at a time (moves over the whole wavefront), then the first lane's for all
    float t = s;
#pragma unroll
    for (int l = 1; l < LPR; ++l) t = s + moved(t, std::integral_constant<int, 0x130>{});
    return __shfl(t, first);
  }
}

template <typename T, int LPR, int NORM>
__global__ __launch_bounds__(256) void qk_norm_axes_kernel(const QkAxesParams p) {
  constexpr int D = 8 * LPR, RPW = 64 / LPR;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int in_wave = lane / LPR, part = lane % LPR, first = lane - part;

  float weight[2][2][8];               // gamma and beta of q and of k
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const T *gamma = static_cast<const T *>(w ? p.gk : p.gq), *beta = static_cast<const T *>(w ? p.bk : p.bq);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      weight[w][0][e] = 1.0f;
      weight[w][1][e] = 0.0f;
    }
    if (gamma) load_row8(gamma + 8 * part, weight[w][0]);
    if (beta) load_row8(beta + 8 * part, weight[w][1]);
  }

  // the wavefront's rows, RPW at a time
  for (unsigned row0 = (blockIdx.x * 4 + wave) * RPW; row0 < p.n_row; row0 += gridDim.x * 4 * RPW) {
    const unsigned row = row0 + in_wave;
    const bool live = in_wave < RPW && row < p.n_row;
    const unsigned tok = quotient(live ? row : 0, p.heads);
    const int head = (int)((live ? row : 0) - tok * p.heads.d);
    const bool has[2] = {live && head < p.heads_q, live && head < p.heads_k};
    float v[2][8];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[w][e] = 0.0f;
      if (has[w]) load_row8(static_cast<const T *>(w ? p.k : p.q) + (w ? tok * p.ld_k : tok * p.ld_q) + head * D + 8 * part, v[w]);
    }

    // factors of the lane's four pairs
    f32x2 f[4];
    const bool turn = p.factors != nullptr;
    if (turn) {
      const unsigned g = tok - quotient(tok, p.tokens) * p.tokens.d;   // token of its batch entry
      const unsigned t = quotient(g, p.YX), r = g - t * p.YX.d, y = quotient(r, p.X), x = r - y * p.X.d;
      const int dt = p.end_t, dy = p.end_y - p.end_t, dx = p.end_x - p.end_y;
      const f32x2 *ft = p.factors + (long long)t * dt, *fy = p.factors + p.first_y + (long long)y * dy - p.end_t,
                  *fx = p.factors + p.first_x + (long long)x * dx - p.end_y;
      if (p.whole) {   // sections of whole fours of pairs: the lane's lie in one, 32 bytes
        const int j = 4 * part;
        f32x4 lo = {1.0f, 0.0f, 1.0f, 0.0f}, hi = lo;
        if (j < p.end_x) {
          const f32x4 *src = reinterpret_cast<const f32x4 *>((j < p.end_t ? ft : j < p.end_y ? fy : fx) + j);
          lo = src[0];
          hi = src[1];
        }
        f[0] = f32x2{lo[0], lo[1]}; f[1] = f32x2{lo[2], lo[3]}; f[2] = f32x2{hi[0], hi[1]}; f[3] = f32x2{hi[2], hi[3]};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = 4 * part + e;
          const f32x2 *src = j < p.end_t ? ft : j < p.end_y ? fy : fx;
          f[e] = f32x2{1.0f, 0.0f};
          if (j < p.end_x) f[e] = src[j];
        }
      }
    }

#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float mean = 0.0f, rstd = 1.0f;
      if constexpr (NORM == NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[w][e];
        mean = row_sum<LPR>(s, first) * (1.0f / D);
      }
      if constexpr (NORM != NORM_NONE) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[w][e] -= mean;
          ss += v[w][e] * v[w][e];
        }
        rstd = 1.0f / sqrtf(row_sum<LPR>(ss, first) * (1.0f / D) + p.eps);
      }
      if (has[w]) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = v[w][e] * rstd * weight[w][0][e] + weight[w][1][e];
        // What lies behind the last section is left alone, by selection: (1, 0) would make a NaN of an infinity's neighbour.  Costs 1 % (47.9 -> 48.4);
        // with a branch for lanes that turn all of their pairs nothing, but 5 % where sections are not whole fours of pairs.
        if (turn) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float c = f[e][0], s = f[e][1], x = o[2 * e], y = o[2 * e + 1];
            const bool turned = 4 * part + e < p.end_x;
            o[2 * e] = turned ? x * c - y * s : x;
            o[2 * e + 1] = turned ? x * s + y * c : y;
          }
        }
        store_row8(static_cast<T *>(w ? p.k_out : p.q_out) + (w ? tok * p.ld_k_out : tok * p.ld_q_out) + head * D + 8 * part, o);
      }
    }
  }
}

// ---- the table: (cos, sin)((origin + place * step) * theta^(-2 i / d)) of one axis, in fp64 because the angle of a far place has no
//      bits left behind the point in fp32; a few thousand pairs, once per video shape ----
struct RopeFactorsParams {
  f32x2 *out;
  int n[3], half[3];                 // places and pairs of each axis
  double origin[3], step[3], log_theta;
  unsigned n_pair;
};

__global__ __launch_bounds__(256) void rope_factors_kernel(const RopeFactorsParams p) {
  const unsigned id = blockIdx.x * 256 + threadIdx.x;
  if (id >= p.n_pair) return;
  unsigned r = id;
  int a = 0;
  while (r >= (unsigned)p.n[a] * p.half[a]) {    // id < n_pair: ends at the third axis at the latest
    r -= (unsigned)p.n[a] * p.half[a];
    ++a;
  }
  const int place = (int)(r / p.half[a]), i = (int)(r % p.half[a]);
  const double angle = (p.origin[a] + place * p.step[a]) * exp(-p.log_theta * i / p.half[a]);
  double s, c;
  sincos(angle, &s, &c);
  p.out[id] = f32x2{(float)c, (float)s};
}

}  // namespace pab
