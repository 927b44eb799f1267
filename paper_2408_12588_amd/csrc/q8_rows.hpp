// Passes over 8-bit rows (q8_common.hpp): values -> rows, layernorm + modulate -> rows, rows -> values with the gated residual.
// Each touches every element once: large ones are bound by memory.  25440 rows of 1152 / 2048, us, over four sets of buffers in turn: quantise bf16
// (88 / 156 MB) 18.4 / 29.6, fp32 (147 / 261 MB) 26.5 / 45.6, read back with gate and residual (147 / 261 MB) 29.5 / 48.4: 4.8 to 5.7 TB/s where a copy of
// 1 GiB reaches 5.1, because they read more than they write and find some of it in the last-level cache of 256 MB.  An output that takes the same
// memory in every call stays there (quantise 14.9).  Layernorm + modulate, one set of buffers: 22.1 / 29.3.  Looking at each value for infinities by
// itself costs 4, 12 and 13 % (quantise bf16 of 1152 columns 15.9 -> 16.5, layernorm 24.8, 33.1): block_max looks at the largest only.
#pragma once
#include "module_rowwise.hpp"
#include "q8_common.hpp"

namespace pab {

struct QuantizeParams {
  const void *x;            // [rows, K], row pitch ldx elements
  unsigned char *data, *scale;
  long long ldx, ld, ld_scale;
  int K;
  unsigned n_item;          // rows * blocks per row
  Divisor nb;               // blocks per row
};

// 16 lanes take a block of 128 values, 8 each.
template <typename T>
__global__ __launch_bounds__(256) void quantize_kernel(const QuantizeParams p) {
  const unsigned item = blockIdx.x * 16 + (threadIdx.x >> 4);
  const int part = threadIdx.x & 15;
  const bool live = item < p.n_item;
  const unsigned row = quotient(live ? item : 0, p.nb), b = (live ? item : 0) - row * p.nb.d;
  const int c = 128 * (int)b + 8 * part;
  float v[1][8] = {{0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f}};
  if (live && c < p.K) load_row8(static_cast<const T *>(p.x) + row * p.ldx + c, v[0]);
  const int byte = q8_scale_byte(max16(block_max(v)));
  const float inv = q8_inverse(byte);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[0][e] *= inv;
  if (!live) return;
  *reinterpret_cast<u32x2 *>(p.data + row * p.ld + c) = u32x2{pack_e4m3(v[0][0], v[0][1], v[0][2], v[0][3]), pack_e4m3(v[0][4], v[0][5], v[0][6], v[0][7])};
  if (part == 0) p.scale[row * p.ld_scale + b] = (unsigned char)byte;
}

struct DequantizeParams {
  const unsigned char *data, *scale;
  const void *x;            // [rows, K] or nullptr: out = x + gate * value
  const void *gate;         // [K] or nullptr: 1
  void *out;
  long long ld, ld_scale, ldx, ldo;
  int K;
  unsigned n_item;          // rows * chunks of 8 columns
  Divisor nc;               // chunks per row
};

// A lane takes 8 columns.
template <typename T>
__global__ __launch_bounds__(256) void dequantize_kernel(const DequantizeParams p) {
  const unsigned item = blockIdx.x * 256 + threadIdx.x;
  if (item >= p.n_item) return;
  const unsigned row = quotient(item, p.nc);
  const int c = 8 * (int)(item - row * p.nc.d);
  const u32x2 d = *reinterpret_cast<const u32x2 *>(p.data + row * p.ld + c);
  const float s = q8_scale(p.scale[row * p.ld_scale + (c >> 7)]);
  float v[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)d[h], true);
    v[4 * h] = lo[0] * s; v[4 * h + 1] = lo[1] * s; v[4 * h + 2] = hi[0] * s; v[4 * h + 3] = hi[1] * s;
  }
  if (p.gate) {
    float g[8];
    load_row8(static_cast<const T *>(p.gate) + c, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= g[e];
  }
  if (p.x) {
    float x[8];
    load_row8(static_cast<const T *>(p.x) + row * p.ldx + c, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
  store_row8(static_cast<T *>(p.out) + row * p.ldo + c, v);
}

struct LnQ8Params {
  const bf16_t *x, *shift, *scale;   // [n_tok, C], [C], [C]
  unsigned char *data, *scales;
  long long ld, ld_scale;
  int n_tok, C;
  float eps;
};

// ln_modulate_kernel (module_rowwise.hpp) that leaves 8-bit rows: a lane's chunks of 8 columns are 64 apart, so 16 neighbouring lanes
// hold a block of 128.  The normed row is quantised from fp32, without the rounding to bf16 in between.  A wavefront per token, although 1152 columns
// leave three quarters of the third chunk idle: 16 lanes per token, four tokens per wavefront, take 23.8 us instead of 22.1 and at 2048 columns 52.6
// instead of 29.3 (registers); wavefronts that go through many tokens and keep shift and scale take 26.2 where this took 24.8.
template <int NCH>
__global__ __launch_bounds__(256) void ln_modulate_q8_kernel(const LnQ8Params p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tok = blockIdx.x * 4 + wave;
  if (tok >= p.n_tok) return;
  const int C = p.C, nchunk = C >> 3, npad = (C + 127) / 128 * 16;
  const bf16_t *xr = p.x + (long long)tok * C;
  bf16x8 x[NCH], sh[NCH], sc[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) x[i] = lane + 64 * i < nchunk ? *reinterpret_cast<const bf16x8 *>(xr + 8 * (lane + 64 * i)) : zero8();
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    sh[i] = sc[i] = zero8();
    if (lane + 64 * i < nchunk) {
      sh[i] = *reinterpret_cast<const bf16x8 *>(p.shift + 8 * (lane + 64 * i));
      sc[i] = *reinterpret_cast<const bf16x8 *>(p.scale + 8 * (lane + 64 * i));
    }
  }
  float v[NCH][8];
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[i][e] = (float)x[i][e];
      s += v[i][e];
    }
  const float mean = wave_sum(s) / (float)C;
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
    if (lane + 64 * i < nchunk) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = v[i][e] - mean;
        ss += d * d;
      }
    }
  const float rstd = 1.0f / sqrtf(wave_sum(ss) / (float)C + p.eps);
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = lane + 64 * i;
    float y[1][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[0][e] = (v[i][e] - mean) * rstd * (1.0f + (float)sc[i][e]) + (float)sh[i][e];
    if (c >= nchunk) {   // padding columns
#pragma unroll
      for (int e = 0; e < 8; ++e) y[0][e] = 0.0f;
    }
    const int byte = q8_scale_byte(max16(block_max(y)));
    const float inv = q8_inverse(byte);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[0][e] *= inv;
    if (c < npad) {
      *reinterpret_cast<u32x2 *>(p.data + tok * p.ld + 8 * c) =
          u32x2{pack_e4m3(y[0][0], y[0][1], y[0][2], y[0][3]), pack_e4m3(y[0][4], y[0][5], y[0][6], y[0][7])};
      if ((lane & 15) == 0) p.scales[tok * p.ld_scale + (c >> 4)] = (unsigned char)byte;
    }
  }
}

}  // namespace pab
