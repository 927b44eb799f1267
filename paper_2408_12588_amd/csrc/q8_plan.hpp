// Which tiles a product of 8-bit rows takes: estimates as for the bf16 projections (launch_plan.hpp, with its kernel numbers), with constants of
// their own, in us, at so many slices of 128.  A few tiles are bound by the latency of their K loop, more than one per CU by L2 and by their
// stores.  Both sides of the lines, measured in us:
//   16, 32, 48: gemm_q8_few for up to 16, 32, 64 tokens, against 64 x 64 tiles with K groups, by kernel trace: 1 x 6912 x 1152 4.1 / 5.6, 3 x 3256 x 4440
//   5.9 / 10.4, 17 x 1152 x 1152 4.0 / 5.4, 64 x 1152 x 1152 5.6 / 5.5, but 64 x 1152 x 4608 13.4 / 10.8, 20 x 4608 x 4608 13.6 / 10.7
//   64 x 64 tiles, three K groups / one: 1 x 6912 x 1152 4.9 / 5.4, 1260 x 576 x 2304 7.4 / 8.5, but 1260 x 576 x 576 4.5 / 4.4
//   96 x 128, two K groups / 128 x 128: 1260 x 2304 x 576 7.0 / 7.4, 2600 x 1152 x 4608 21.7 / 27.8
//   160 x 128, two K groups / 128 x 128 / large tiles: 4413 x 1152 x 4608 27.3 / 31.3 / 41.7, 4413 x 1152 x 1152 10.5 / 11.4 / 15.5
//   128 x 128 / large: 1260 x 3456 x 1152 11.1 / 14.5, 8000 x 1152 x 1152 18.9 / 18.4, 4413 x 4608 x 1152 33.5 / 30.2
//   64 x 128 / 128 x 128, 8-bit outputs with GELU: 1260 x 1152 x 576 6.2 / 8.5, 1260 x 3456 x 1152 16.3 / 13.4
//   large tiles, 256 / 288 features: 25440 x 3456 x 1152 98.8 / 99.2, 25440 x 1152 x 4608 128 / 133, 57600 x 1152 x 4608 294 / 273
//   the same with GELU, whose 288-feature kernel spills three registers: where the plan takes 288, the choice without it / with it 8000 x 2304 x 4608 95 / 72,
//   57600 x 1152 x 4608 308 / 288, but 25440 x 576 x 576 20.2 / 22.2; 10 % for it in the mean of 52 shapes
// Against the best kernel of each of 1200 random shapes, those of the fit among them, the choice loses 0.7 % in the mean; on others 1.0 % (219 into rows, with
// their stores as they are now) and 1.2 % (218 into bf16).
#pragma once
#include <algorithm>
#include <cstdint>

#include "launch_plan.hpp"

namespace pab {

// GELU with K groups, one of which applies it to all sums: 501 x 2816 x 640 into rows, 64 x 128 tiles, two groups / one 6.9 / 6.4
constexpr double GELU_US = 0.8;

// Sizes that a launch and the kernels' 32-bit indexes hold.  A grid has fewer than 2^32 threads: 12.5 million workgroups of 512 (1 token, 200 million features
// in kernel 16) are too many, where a quarter of them of 256 (kernel 64) are not.  The last tile's indexes end less than 512 past the matrix.
constexpr int Q8_MOST = 0x7fffffff - 511;
inline int q8_threads(int kernel) {
  return kernel == 97 ? 1024 : kernel == 65 ? 768 : kernel == 64 || kernel == 128 ? 256 : 512;
}
inline bool q8_fits(int kernel, long long units) { return (units + 7) / 8 * 8 * q8_threads(kernel) < 1LL << 32; }   // grids are multiples of 8

// base: launch, first copies, K groups' sums; latency: a slice of a lone tile; l2, out: a slice and the stores where every CU has a tile
inline void q8_tile(int kernel, bool gelu, double base, double latency, double l2, double out, int M, int N, int slices, GemmPlan *best) {
  const int bm = tile_tokens(kernel), bn = tile_features(kernel);
  const long long n_mt = ((long long)M + bm - 1) / bm, n_nt = ((long long)N + bn - 1) / bn, all = n_mt * n_nt;
  if (((kernel & 1) && all > GEMM_CUS) || !q8_fits(kernel, all)) return;   // K groups: one workgroup per CU
  const double load = all / (double)GEMM_CUS + 0.25, us = base + (gelu && (kernel & 1) ? GELU_US : 0.0) + slices * std::max(latency, load * l2) + load * out;
  if (us < best->us) *best = GemmPlan{kernel, (int)n_mt, (int)n_nt, 0, (int)all, us, tile_order(bm, bn, n_mt, n_nt)};
}

// kernel 0: no launch holds the problem
inline GemmPlan plan_q8(int M, int N, int nk, bool out8, bool gelu) {
  GemmPlan best{0, 0, 0, 0, 0, 1e30, 0};
  if (M > Q8_MOST || N > Q8_MOST) return best;
  if (!out8 && M <= 64 && q8_fits(16, (N + 15) / 16)) {   // few tokens: 16 features per workgroup, which reads them and every token at about 38 KB / us
    const int units = (N + 15) / 16;
    best = GemmPlan{M <= 16 ? 16 : M <= 32 ? 32 : 48, 1, units, 0, units, 2.9 + (units + GEMM_CUS - 1) / GEMM_CUS * (16 + M) * 128.0 * nk / 38000.0, 0};
  }
  if (out8) {    // tiles are whole blocks of 128 features
    q8_tile(96, gelu, 2.06, 0.51, 0.4, 0.85, M, N, nk, &best);
  } else {
    q8_tile(64, gelu, 2.03, 0.376, 0.3, 0.56, M, N, nk, &best);
    q8_tile(65, gelu, 3.1, 0.157, 0.177, 0.65, M, N, nk, &best);
  }
  q8_tile(97, gelu, 3.1, 0.28, 0.3, 0.87, M, N, nk, &best);
  q8_tile(113, gelu, 2.5, 0.51, 0.436, 1.4, M, N, nk, &best);
  q8_tile(128, gelu, 2.13, 0.88, 0.514, 1.6, M, N, nk, &best);
  q8_tile(129, gelu, 2.93, 0.66, 0.51, 2.24, M, N, nk, &best);
  q8_tile(161, gelu, 3.1, 0.7, 0.586, 2.35, M, N, nk, &best);
  if (!out8 || N % 128 == 0) plan_stream(8, M, N, nk, 1.58 * nk + 4.7, 0.46, &best);   // tiles moved back to the edge start at whole blocks
  if (!out8) plan_stream(9, M, N, nk, 1.70 * nk + 8.0, 0.34, &best);
  if (best.n_units > Q8_MOST) best.kernel = 0;
  return best;
}

// Whether an output of M rows of `width` bytes, `pitch` apart, is written past the caches.  Only where rows start at whole pieces of 64 bytes, or memory
// reads what it keeps of them (53536 x 3544 x 200: 138 -> 252 us).  In us, through the caches / past them, alone and with the pass or product that reads it:
//   a tile per workgroup, bf16: gains (4413 x 1152 x 1152 12.2 / 11.2 and 16.5 / 16.1, 2600 x 2304 x 1152 12.5 / 11.2 and 17.3 / 16.7)
//   a tile per workgroup, 8-bit rows: the next product reads them, many times over, and two of the kernels (96, 97) write them 32 bytes at a time: through
//   the caches (1260 x 3456 x 576 9.1 / 8.9 but 22.1 / 25.3, 2600 x 2304 x 2304 20.3 / 20.3 and 32.9 / 35.4, MLP of 501 x 1152 / 4608 25.6 / 28.8;
//   6249 x 576 x 1152 19.7 / 19.1 is the largest loss)
//   large tiles, whose operands wait in L2 while a tile is stored: large outputs gain (25440 x 3456 x 1152, 176 MB, 116 / 95 and 157 / 151; in rows
//   40000 x 4608 x 1152 207 / 189 and 425 / 427), of a small one the reader finds more in the last-level cache of 256 MB (25440 x 1152 x 1152, 59 MB, 41.4 / 40.2
//   but 56.9 / 58.1; in rows 25440 x 4608 x 1152, 117 MB, 134 / 124 but 275 / 279); bf16 between 100 and 150 MB would gain (19000 x 3456 x 1152 89 / 72 and 117 / 115)
inline bool q8_past_caches(int kernel, bool out8, long long M, const void *to, long long width, long long pitch) {
  if ((reinterpret_cast<uintptr_t>(to) | (unsigned long long)width | (unsigned long long)pitch) % 64) return false;
  return kernel >= 64 ? !out8 : M * width > (150LL << 20);
}

}  // namespace pab
