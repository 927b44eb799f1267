// Products of 8-bit rows for few tokens (a timestep's modulation, single tokens): one workgroup per 16 features, its 8 wavefronts take every
// eighth K slice each, for up to 16 MS tokens.
//
// What bounds it: the way of the weights from memory to the registers, once.  Nothing is shared between wavefronts but the sums, so operands
// go from memory straight into the instruction's layout (16 rows of 64 bytes per load), those of three slices at a time requested before
// the first product, and there is no LDS stage and no barrier in the K loop.  The sums are added through LDS, group by group in order.
// 1 x 6912 x 1152 (8 MB of weights): 4.1 us, 5.6 with 64 x 64 tiles and K groups; 3 x 3256 x 4440 5.9, 10.4.  Slices deeper than three ahead
// change nothing.
#pragma once
#include "gemm_q8.hpp"

namespace pab {

template <int MS, int ACT>
__global__ __launch_bounds__(512) void gemm_q8_few_kernel(const GemmQ8Params p) {
  constexpr int KG = 8, DEEP = 3;
  __shared__ f32x4 sums[KG][MS][64];
  const int lane = threadIdx.x & 63, l16 = lane & 15, q16 = lane >> 4;
  const int kg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = 16 * blockIdx.x, nk = p.nk;
  const int feature = min(n0 + l16, p.N - 1);          // rows past either matrix re-read its last one; nothing of them is stored
  const unsigned char *w = p.W + feature * p.ldw + 16 * q16, *sw = p.sw + feature * p.lsw;
  const unsigned char *t[MS], *st[MS];
#pragma unroll
  for (int a = 0; a < MS; ++a) {
    const int token = min(16 * a + l16, p.M - 1);
    t[a] = p.A + token * p.lda + 16 * q16;
    st[a] = p.sa + token * p.lsa;
  }
  auto rd = [](const unsigned char *row, int kt) {
    typedef __attribute__((ext_vector_type(4))) int i32x4;
    const i32x4 lo = *reinterpret_cast<const i32x4 *>(row + 128LL * kt), hi = *reinterpret_cast<const i32x4 *>(row + 128LL * kt + 64);
    return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  };
  f32x4 acc[MS];
#pragma unroll
  for (int a = 0; a < MS; ++a) acc[a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int k0 = kg; k0 < nk; k0 += DEEP * KG) {
    i32x8 wf[DEEP], tf[DEEP][MS];
    int ws[DEEP], ts[DEEP][MS];
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      const int kt = k0 + d * KG;
      if (kt < nk) {
        wf[d] = rd(w, kt);
        ws[d] = sw[kt];
#pragma unroll
        for (int a = 0; a < MS; ++a) {
          tf[d][a] = rd(t[a], kt);
          ts[d][a] = st[a][kt];
        }
      }
    }
#pragma unroll
    for (int d = 0; d < DEEP; ++d)
      if (k0 + d * KG < nk) {
#pragma unroll
        for (int a = 0; a < MS; ++a) acc[a] = mfma_q8(wf[d], tf[d][a], acc[a], ws[d], ts[d][a]);
      }
  }
#pragma unroll
  for (int a = 0; a < MS; ++a) sums[kg][a][lane] = acc[a];
  __syncthreads();
  if (kg >= MS) return;                                // wavefront a finishes token sub-tile a
  const int n = n0 + 4 * q16, m = 16 * kg + l16;
  if (n >= p.N || m >= p.M) return;
  f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
  if (p.bias) {
    const bf16x4 b4 = *reinterpret_cast<const bf16x4 *>(p.bias + n);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (float)b4[e];
  }
#pragma unroll
  for (int g = 0; g < KG; ++g) y += sums[g][kg][lane];
  bf16x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (bf16_t)(ACT == Q8_GELU ? gelu_q8(y[e]) : y[e]);
  *reinterpret_cast<bf16x4 *>(p.C + m * p.ldc + n) = o;
}

}  // namespace pab
