// Products of 8-bit rows that fill the chip: one persistent workgroup of 4 wavefronts per CU works through tiles of 256 tokens x 32 NS features,
// 2 wavefronts along the tokens x 2 along the features, 8 x NS sub-tiles each (layouts and the instruction: gemm_q8.hpp).  The
// division of the work, the stream of copies through two LDS stages across tile borders, the tail tiles and the tiles moved back to end at
// the matrix edge (rows that two tiles compute are written twice with the same bits) are those of gemm_stream.hpp; a slice of
// 128 bytes is twice its multiply-adds.
//
// One wavefront per SIMD with all 512 registers (256 or 288 of sums) reads half the operands from LDS that eight wavefronts of half its tile
// read, and waits for nobody but the copies.  To keep the matrix core fed by itself, it goes through a slice in an order that
// leaves every load time: weight sub-tiles 0 .. NS - 3 one after the other, each with all token sub-tiles, operands two steps (16
// products) ahead; then the barrier, when everything of the slice has been read: it frees its stage and publishes the other; then
// token by token with the last two weight sub-tiles, after which the token's registers take the next slice's operand.  The
// copies of the slice after that go out one by one between the products behind the barrier.
// There is no branch inside a slice: the compiler sinks products past one, and then holds their operands.  The copies of a tile of fewer than 256
// tokens repeat its last rows, and those behind the last tile repeat that tile; nobody reads either.
#pragma once
#include "gemm_q8.hpp"

namespace pab {

template <int NS, int ACT, bool OUT8>
__global__ __launch_bounds__(256, 1) void gemm_q8_stream_kernel(const GemmQ8Params p) {
  constexpr int BM = 256, BN = 32 * NS, ROWS = BM + BN;
  // bytes: token rows, pair rows of the weights, odd sub-tiles; a dword of scales for each (copied by 64)
  constexpr int STAGE = 128 * ROWS + 4 * ((ROWS + 63) / 64 * 64);
  constexpr int NPAIR = NS / 2;
  constexpr bool ODD = NS % 2 != 0;
  constexpr int W0 = 128 * BM, W1 = W0 + 128 * 64 * NPAIR, SC = 128 * ROWS;   // byte offsets in a stage
  constexpr int SHIFT1 = ODD ? 16 : 0;           // features of wave column 1 before its pairs
  constexpr int NDMA = 8 + 2 * NPAIR + (ODD ? 1 : 0) + 1;   // copies of a wavefront per slice: 32 rows each, and the scales
  static_assert(NPAIR == 4, "scales are copied by two pairs, outputs stored by two pairs");
  static_assert(!OUT8 || NS == 8, "a wavefront's features are one block");
  constexpr int BIAS = 2 * STAGE, XPOSE = BIAS + 2048;   // byte offsets: two bias rows, 2 KB per wavefront

  __shared__ __attribute__((aligned(16))) unsigned char smem[XPOSE + 4 * 2048];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, q16 = lane >> 4;
  const int wm = wave >> 1, wn = wave & 1;
  const unsigned lds0 = (unsigned)(size_t)((__attribute__((address_space(3))) unsigned char *)smem);
  const int M = p.M, N = p.N, nk = p.nk;

  // ---- the workgroup's tiles: unit i of it is number wg + i * gridDim.x; a round of a full grid gives each XCD 32
  //      consecutive units, which are 4 token tiles x 8 feature tiles ----
  struct Tile { int m0, n0, ms; };
  constexpr int GM = 4;
  const int n_full = p.n_mt * p.n_nt;
  auto unit = [&](int u) __attribute__((always_inline)) {
    Tile t;
    if (u < n_full) {
      const int g = u / (GM * p.n_nt), r = u % (GM * p.n_nt), gm = min(GM, p.n_mt - g * GM);   // the last group may be smaller
      t.m0 = (g * GM + r % gm) * BM; t.n0 = (r / gm) * BN; t.ms = 4;
    } else {
      const int r = u - n_full;
      t.ms = p.ms_tail;
      t.m0 = min(p.n_mt * BM + (r / p.n_nt) * 64 * t.ms, M - 64 * t.ms); t.n0 = (r % p.n_nt) * BN;
    }
    t.n0 = min(t.n0, N - BN);
    t.m0 = __builtin_amdgcn_readfirstlane(t.m0);
    t.n0 = __builtin_amdgcn_readfirstlane(t.n0);
    t.ms = __builtin_amdgcn_readfirstlane(t.ms);
    return t;
  };
  const int wg = gridDim.x == 256 ? (blockIdx.x & 7) * 32 + (blockIdx.x >> 3) : blockIdx.x;
  const int n_mine = (p.n_units - wg + (int)gridDim.x - 1) / (int)gridDim.x;

  // ---- copies: wavefront w moves rows 8 w .. 8 w + 7 of every 32 rows; its lane row lane >> 3, position lane & 7.  Weight rows lie by
  //      wave column, pair, sub-tile, operand row; row i of a pair is its feature 8 ((i & 15) >> 2) + 4 (i >> 4) + (i & 3) ----
  const int crow = 8 * wave + (lane >> 3);
  const int cq = (lane & 7) ^ gemm_swizzle(crow);
  auto in_pair = [](int i) { return 8 * ((i & 15) >> 2) + 4 * (i >> 4) + (i & 3); };
  constexpr int COL1 = 16 * NS + SHIFT1;         // first paired feature of wave column 1
  // odd sub-tiles: the last 16 features of wave column 0, the first 16 of column 1
  auto odd_feature = [](int i) { return (i >> 4 ? 16 * NS : 32 * NPAIR) + (i & 15); };
  const unsigned voff_a = (unsigned)(crow * p.lda + 16 * cq), voff_w = (unsigned)(in_pair(crow) * p.ldw + 16 * cq),
                 voff_s = (unsigned)(odd_feature(crow) * p.ldw + 16 * cq);
  // scales: wavefront w those of 64 tokens and of two pairs, and all of them (the same) those of the odd rows
  const unsigned soff_a = (unsigned)(lane * p.lsa), soff_w = (unsigned)((32 * (lane >> 5) + in_pair(lane & 31)) * p.lsw),
                 soff_s = (unsigned)(odd_feature(lane & 31) * p.lsw);
  struct Source {                                // where a tile's slices come from
    const unsigned char *a, *w, *sa, *sw, *so;
    int last;                                    // last of its rounds of 32 tokens
  };
  auto source = [&](int i) __attribute__((always_inline)) {
    const Tile t = unit(wg + i * (int)gridDim.x);
    Source s;
    s.last = 2 * t.ms - 1;
    s.a = p.A + t.m0 * p.lda;
    s.w = p.W + t.n0 * p.ldw;
    s.so = p.sw + t.n0 * p.lsw;
    s.sa = p.sa + (t.m0 + 64 * min(wave, t.ms - 1)) * p.lsa;
    s.sw = s.so + ((wave >> 1) * COL1 + 64 * (wave & 1)) * p.lsw;
    return s;
  };
  auto copy_round = [&](const Source &s, int kt, int stage, int i) __attribute__((always_inline)) {   // copy i of slice kt
    const unsigned lds = lds0 + STAGE * stage + 1024 * wave;
    if (i == 0) {
      const unsigned sc = lds0 + STAGE * stage + SC;
      const int k = kt & ~3;
      dma4_to_lds(s.sa + k, soff_a, sc + 256 * wave);
      dma4_to_lds(s.sw + k, soff_w, sc + 4 * BM + 256 * wave);
      if (ODD) dma4_to_lds(s.so + k, soff_s, sc + 4 * (BM + 64 * NPAIR));
      return;
    }
    --i;
    if (i < 8) dma16_to_lds(s.a + 128LL * kt + 32LL * min(i, s.last) * p.lda, voff_a, lds + 4096 * i);
    else if (i < 8 + 2 * NPAIR)
      dma16_to_lds(s.w + 128LL * kt + ((i - 8) / NPAIR * COL1 + 32 * ((i - 8) % NPAIR)) * p.ldw, voff_w, lds + W0 + 4096 * (i - 8));
    else dma16_to_lds(s.w + 128LL * kt, voff_s, lds + W1);
  };

  Source cur = source(0), nxt = cur;
  for (int stage = 0; stage < 2; ++stage) {      // the first two slices (there are two or more)
#pragma unroll
    for (int i = 0; i < NDMA; ++i) copy_round(cur, stage, stage, i);
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  const int sw = gemm_swizzle(l16);
  const unsigned op = 128 * l16 + 16 * (q16 ^ sw);        // operand address inside 16 rows
  int stage = 0;

  auto run_tile = [&](auto ms_tag, const Tile t, int parity) __attribute__((always_inline)) {
    constexpr int MS = 2 * decltype(ms_tag)::value;        // token sub-tiles of a wavefront
    constexpr int LAST = NS - 2;                           // the last two weight sub-tiles go token by token
    f32x4 acc[MS][NS];
    i32x8 tf[MS], wf[3], hf[2];                            // tokens, ring of weights, last two weights
    int ts[MS], tn[MS], ws[3], hs[2];                      // their scales; tn: the next slice's
    unsigned tb, tb4, wb, wb4, tsb, wsb;
    auto use_stage = [&](int s, int k) __attribute__((always_inline)) {
      const unsigned st = lds0 + STAGE * s;
      tb = st + 2048 * MS * wm + op;
      wb = st + W0 + 4096 * NPAIR * wn + op;
      tb4 = tb ^ 64;
      wb4 = wb ^ 64;
      tsb = st + SC + 4 * (16 * MS * wm + l16) + (k & 3);
      wsb = st + SC + 4 * (BM + 32 * NPAIR * wn + l16) + (k & 3);
    };
    auto rd_t = [&](int a) __attribute__((always_inline)) { tf[a] = lds_read32(tb + 2048 * a, tb4 + 2048 * a); };
    auto rd_w = [&](int b, i32x8 &w, int &scale) __attribute__((always_inline)) {
      const bool pair = b < 2 * NPAIR;
      scale = lds_read_byte(wsb + (pair ? 64 * b : 4 * 64 * NPAIR - 4 * (32 * NPAIR - 16) * wn));
      const unsigned off = pair ? 2048 * b : W1 - W0 - (4096 * NPAIR - 2048) * wn;
      w = lds_read32(wb + off, wb4 + off);
    };
    use_stage(stage, 0);
#pragma unroll
    for (int a = 0; a < MS; ++a) {
      ts[a] = lds_read_byte(tsb + 64 * a);
      rd_t(a);
    }
    rd_w(0, wf[0], ws[0]);
    rd_w(1, wf[1], ws[1]);
#pragma unroll
    for (int a = 0; a < MS; ++a)
#pragma unroll
      for (int b = 0; b < NS; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[a][b][e] = 0.0f;

    // the copies of slice kt + 2: PER behind the barrier of slice kt with every token sub-tile, the others in the first part of slice
    // kt + 1, every EACH products
    constexpr int PER = MS == 8 ? 1 : MS == 2 ? 4 : 2, EACH = MS == 8 ? 2 : 1;
    static_assert(PER * MS + LAST * MS / EACH >= NDMA, "all copies have a place");
    for (int kt = 0; kt < nk; ++kt) {
      const bool last = kt + 1 >= nk;
      const Source &before = last ? nxt : cur;
      const int k1 = last ? 0 : kt + 1;
#pragma unroll
      for (int j = 0; j < LAST; ++j) {
        if (j + 2 < LAST) rd_w(j + 2, wf[(j + 2) % 3], ws[(j + 2) % 3]);
        else rd_w(j + 2, hf[j + 2 - LAST], hs[j + 2 - LAST]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int a = 0; a < MS; ++a) {
          const int i = PER * MS + (j * MS + a) / EACH;
          if ((j * MS + a) % EACH == 0 && i < NDMA) copy_round(before, k1, stage ^ 1, i);
          acc[a][j] = mfma_q8(wf[j % 3], tf[a], acc[a][j], ws[j % 3], ts[a]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // this slice has been read, the next one has arrived
      stage ^= 1;
      use_stage(stage, kt + 1 == nk ? 0 : kt + 1);
      const int ks = kt + 2;
      const bool over = ks >= nk;
      const Source &from = over ? nxt : cur;
      const int k = over ? ks - nk : ks;
#pragma unroll
      for (int a = 0; a < MS; ++a) {
#pragma unroll
        for (int i = PER * a; i < PER * a + PER; ++i)
          if (i < NDMA) copy_round(from, k, stage ^ 1, i);
        acc[a][LAST] = mfma_q8(hf[0], tf[a], acc[a][LAST], hs[0], ts[a]);
        __builtin_amdgcn_sched_barrier(0);
        if (a == 0) rd_w(0, wf[0], ws[0]);
        if (a == 1) rd_w(1, wf[1], ws[1]);
        tn[a] = lds_read_byte(tsb + 64 * a);
        acc[a][LAST + 1] = mfma_q8(hf[1], tf[a], acc[a][LAST + 1], hs[1], ts[a]);
        __builtin_amdgcn_sched_barrier(0);
        rd_t(a);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int a = 0; a < MS; ++a) ts[a] = tn[a];
    }

    const int shift = wn ? SHIFT1 : 0, odd = wn ? 0 : 32 * NPAIR;   // where the pairs / the odd sub-tile start
    const bf16_t *bs = reinterpret_cast<const bf16_t *>(smem + BIAS + 1024 * parity) + wn * 16 * NS;
    const int f0 = t.n0 + wn * 16 * NS, m0 = t.m0 + wm * 16 * MS;
    const unsigned xs = lds0 + XPOSE + 2048 * wave;
    auto finish = [](float x) { return ACT == Q8_GELU ? gelu(x) : x; };
    if constexpr (OUT8) {
      // a wavefront's 128 features are a block: bias and activation, the largest magnitude over a lane's 32 and its token's four
      // lanes, then 16 tokens x 128 bytes at a time
      float bv[4][8];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        bf16x8 b8 = zero8();
        if (p.bias) b8 = *reinterpret_cast<const bf16x8 *>(bs + 32 * u + 8 * q16);
#pragma unroll
        for (int e = 0; e < 8; ++e) bv[u][e] = (float)b8[e];
      }
#pragma unroll
      for (int a = 0; a < MS; ++a) {
        unsigned big = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = finish(acc[a][2 * u + (e >> 2)][e & 3] + bv[u][e]);
            acc[a][2 * u + (e >> 2)][e & 3] = x;
            big = max(big, finite_bits(x));
          }
        const int byte = q8_scale_byte(max_across(big));
        const float inv = q8_inverse(byte);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = q8_scaled(acc[a][2 * u + (e >> 2)][e & 3], inv);
          // chunk 2 u + (q16 >> 1) of the row, swizzled as everywhere
          *(__attribute__((address_space(3))) u32x2 *)(size_t)(xs + 128 * l16 + 16 * ((2 * u + (q16 >> 1)) ^ sw) + 8 * (q16 & 1)) =
              u32x2{pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7])};
        }
        if (q16 == 0) p.s8[(m0 + 16 * a + l16) * p.ls8 + (f0 >> 7)] = (unsigned char)byte;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const unsigned xr = xs + 128 * (lane >> 3) + 16 * ((lane & 7) ^ gemm_swizzle(lane >> 3));
        typedef const __attribute__((address_space(3))) u32x4 *ptr;
        const u32x4 r0 = *(ptr)(size_t)xr, r1 = *(ptr)(size_t)((xr ^ 64) + 1024);   // rows 8 further: swizzle ^ 4
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        unsigned char *dst = p.C8 + (m0 + 16 * a + (lane >> 3)) * p.ld8 + f0 + 16 * (lane & 7);
        *reinterpret_cast<u32x4 *>(dst) = r0;
        *reinterpret_cast<u32x4 *>(dst + 8 * p.ld8) = r1;
      }
    } else {
      // ---- bias, activation, stores: 16 tokens x 64 features at a time through the wavefront's 2 KB ----
      const unsigned xw = xs + 128 * l16, xr = xs + 128 * (lane >> 3) + 16 * ((lane & 7) ^ gemm_swizzle(lane >> 3));
#pragma unroll
      for (int h = 0; h < NPAIR / 2; ++h) {
        float bv[2][8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          bf16x8 b8 = zero8();
          if (p.bias) b8 = *reinterpret_cast<const bf16x8 *>(bs + shift + 64 * h + 32 * u + 8 * q16);
#pragma unroll
          for (int e = 0; e < 8; ++e) bv[u][e] = (float)b8[e];
        }
        bf16_t *dst = p.C + f0 + shift + 64 * h + 8 * (lane & 7) + (long long)(m0 + (lane >> 3)) * p.ldc;
#pragma unroll
        for (int a = 0; a < MS; ++a) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            bf16x8 y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (bf16_t)finish(acc[a][4 * h + 2 * u + (e >> 2)][e & 3] + bv[u][e]);
            lds_write8(xw + 16 * ((4 * u + q16) ^ sw), y);
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          const bf16x8 r0 = lds_read8(xr), r1 = lds_read8((xr ^ 64) + 1024);   // rows 8 further: swizzle ^ 4
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          *reinterpret_cast<bf16x8 *>(dst) = r0;
          *reinterpret_cast<bf16x8 *>(dst + 8 * p.ldc) = r1;
          dst += 16 * p.ldc;
        }
      }
      if (ODD) {
        bf16x4 b4;
#pragma unroll
        for (int e = 0; e < 4; ++e) b4[e] = (bf16_t)0.0f;
        if (p.bias) b4 = *reinterpret_cast<const bf16x4 *>(bs + odd + 4 * q16);
        bf16_t *dst = p.C + f0 + odd + 8 * (lane & 1) + (long long)(m0 + (lane >> 1)) * p.ldc;
#pragma unroll
        for (int a0 = 0; a0 < MS; a0 += 4) {               // four sub-tiles are the wavefront's 2 KB
#pragma unroll
          for (int a = a0; a < MS && a < a0 + 4; ++a) {
            bf16x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (bf16_t)finish(acc[a][NS - 1][e] + (float)b4[e]);
            lds_write4(xs + 32 * (16 * (a - a0) + l16) + 8 * q16, y);
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
          for (int a = 0; a < (MS - a0 < 4 ? MS - a0 : 4) / 2; ++a)
            *reinterpret_cast<bf16x8 *>(dst + (16 * a0 + 32 * a) * p.ldc) = lds_read8(xs + 1024 * a + 16 * lane);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
      }
    }
  };

  for (int i = 0; i < n_mine; ++i) {
    const Tile t = unit(wg + i * (int)gridDim.x);
    nxt = source(min(i + 1, n_mine - 1));
    if (p.bias && wave == 3) dma16_to_lds(p.bias + t.n0, 16 * min(lane, BN / 8 - 1), lds0 + BIAS + 1024 * (i & 1));
    if (t.ms == 4) run_tile(std::integral_constant<int, 4>{}, t, i & 1);
    else if (t.ms == 3) run_tile(std::integral_constant<int, 3>{}, t, i & 1);
    else if (t.ms == 2) run_tile(std::integral_constant<int, 2>{}, t, i & 1);
    else run_tile(std::integral_constant<int, 1>{}, t, i & 1);
    cur = nxt;
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);            // the last copies
}

}  // namespace pab
