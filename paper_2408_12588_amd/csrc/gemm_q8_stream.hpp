// Products of 8-bit rows that fill the chip: one persistent workgroup of 8 wavefronts per CU works through tiles of 256 tokens x 32 NS features,
// 4 wavefronts along the tokens x 2 along the features, 4 x NS sub-tiles each (layouts and the instruction: gemm_q8.hpp).  The
// division of the work, the stream of copies through two LDS stages across tile borders, the tail tiles and the tiles moved back to end at
// the matrix edge (rows that two tiles compute are written twice with the same bits) are those of gemm_stream.hpp; a slice of
// 128 bytes is twice its multiply-adds.
//
// Inside a slice: NS steps of one weight sub-tile (32 bytes a lane, one instruction deep) x the token sub-tiles.  Weight operands are read
// RING - 1 steps ahead.  Token operands, 8 registers each, have no second set: the last step reads the next slice's behind each
// product that used the old one.  One barrier per slice, RING - 1 steps before its end, when everything of it has been read: it frees its
// stage and publishes the other, and the copies of the slice after that go out two per step, so that they have half a slice to arrive.
// There is no branch inside a slice: the compiler sinks products past one, and then holds their operands.  The copies of a tile of fewer than 256
// tokens repeat its last rows, and those behind the last tile repeat that tile; nobody reads either.
//
// Between tiles: the first slice of a tile, written out by itself, starts the sums from the bias, which was copied a tile ahead; its barrier does not
// wait for the stores of the tile before (memory operations of a wavefront end in order, so leaving as many of the last ones open as
// there were stores is enough); and the stores of a step of the epilogue go out behind the arithmetic of the next.  Large outputs are written past
// the caches (q8_plan.hpp says when): what all workgroups of an XCD store at once is as large as its L2, and drives out the operands.  The 32-byte
// pieces of odd sub-tiles never are: memory would read what it keeps of them (288-feature tiles, 53536 x 3584 x 200: 92 -> 135).
//
// Measured, us: a slice of 256 x 256 x 128 takes 1.53 to 1.57 (1024 tiles, 9 to 36 slices deep), of 256 x 288 1.65 to 1.78, and a tile 3 (8-bit or
// large outputs) to 6 and 8 more, with GELU 3 to 4 more.  The products of a slice alone, from registers, take 1.22 on random values, where power holds them to
// 3.5 PF, and 0.99 on zeros (4.3 PF); its 66 KB take 1.10 at the 60 GB/s that L2 gives a CU when all ask.  Neither bounds the loop by itself: it takes
// 1.37 with all operands in L2, 1.08 without the copies (the same values each time), and the barrier waits for every copy of a slice before the
// first of the slice after next is sent, so that the way from L2 empties once in each.  Tried: two copies per step are best (all at
// once 2.12; in the second half 1.8; one or three per step slower), tile orders that share operands within an XCD (groups of 2 to 16 token tiles) are
// the same.  Four wavefronts of 128 x 128 with 512 registers run the loop as fast and leave a tile more slowly; touching the slice after next for
// L2 gains 3 % at K = 1152 and loses 9 % at 4608.  Not tried: token copies that stay in flight across the barrier.  Whole products: 25440 x 3456 x
// 1152 98 (2.06 PF), 57600 x 1152 x 4608 271 (2.26 PF), 16384 x 4096 x 1152 into 8-bit rows 73 (2.1 PF), with GELU 90.
#pragma once
#include "gemm_q8.hpp"

namespace pab {

template <int NS, int RING, int ACT, bool OUT8>
__global__ __launch_bounds__(512, 2) void gemm_q8_stream_kernel(const GemmQ8Params p) {
  constexpr int BM = 256, BN = 32 * NS, ROWS = BM + BN;
  // bytes: token rows, pair rows of the weights, odd sub-tiles; a dword of scales for each (copied by 64)
  constexpr int STAGE = 128 * ROWS + 4 * ((ROWS + 63) / 64 * 64);
  constexpr int NPAIR = NS / 2;
  constexpr bool ODD = NS % 2 != 0;
  constexpr int W0 = 128 * BM, W1 = W0 + 128 * 64 * NPAIR, SC = 128 * ROWS;   // byte offsets in a stage
  constexpr int SHIFT1 = ODD ? 16 : 0;           // features of wave column 1 before its pairs
  constexpr int NDMA = 4 + NPAIR + (ODD ? 1 : 0);   // copy rounds of a wavefront per slice
  constexpr int AHEAD = RING - 1, JB = NS - AHEAD;  // operand distance, barrier step
  constexpr int PER = 2;                         // copy rounds per step
  static_assert(NPAIR % 2 == 0, "pairs are stored two at a time");
  static_assert(NS % RING == 0 && NDMA <= PER * NS, "the operand ring continues across slices");
  static_assert(!OUT8 || NS == 8, "a wavefront's features are one block");
  constexpr int BIAS = 2 * STAGE, XPOSE = BIAS + 2048;   // byte offsets: two bias rows, 2 KB per wavefront

  __shared__ __attribute__((aligned(16))) unsigned char smem[XPOSE + 8 * 2048];
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

  // ---- copies: wavefront w moves rows 8 w .. 8 w + 7 of every 64 rows; its lane row lane >> 3, position lane & 7 ----
  const int crow = 8 * wave + (lane >> 3);
  const int cq = (lane & 7) ^ gemm_swizzle(crow);
  // row i of a round of pair rows, 32 of each wave column: sub-tile (i >> 4) & 1, operand row i & 15
  auto pair_feature = [](int i) { return (i >> 5) * (16 * NS + SHIFT1) + 8 * ((i & 15) >> 2) + 4 * ((i >> 4) & 1) + (i & 3); };
  // odd sub-tiles: the last 16 features of wave column 0, the first 16 of column 1
  auto odd_feature = [](int i) { return (i >> 4 ? 16 * NS : 32 * NPAIR) + (i & 15); };
  const unsigned voff_a = (unsigned)(crow * p.lda + 16 * cq), voff_w = (unsigned)(pair_feature(crow) * p.ldw + 16 * cq),
                 voff_s = (unsigned)(odd_feature(crow & 31) * p.ldw + 16 * cq);
  // scales: wavefronts 0-3 those of 64 tokens each, 4-7 of a round of pair rows each, and all of them (the same) those of the odd rows
  const bool tok_wave = wave < 4;
  const unsigned soff = (unsigned)(tok_wave ? lane * p.lsa : pair_feature(lane) * p.lsw), soff_s = (unsigned)(odd_feature(lane & 31) * p.lsw);
  struct Source {                                // where a tile's slices come from
    const unsigned char *a, *w, *sc, *so;
    int last;                                    // last of its rounds of 64 tokens
  };
  auto source = [&](int i) __attribute__((always_inline)) {
    const Tile t = unit(wg + i * (int)gridDim.x);
    const unsigned char *so = p.sw + t.n0 * p.lsw;
    return Source{p.A + t.m0 * p.lda, p.W + t.n0 * p.ldw,
                  tok_wave ? p.sa + (t.m0 + 64 * min(wave, t.ms - 1)) * p.lsa : so + 32 * (wave - 4) * p.lsw, so, t.ms - 1};
  };
  // The slice that is being copied: pointers that run from round to round
  struct Window {
    const unsigned char *a, *w;
    int last;
  };
  const unsigned step_a = (unsigned)(64 * p.lda), step_w = (unsigned)(32 * p.ldw);
  auto open = [&](const Source &s, int kt, int stage) __attribute__((always_inline)) {   // copies the scales
    const unsigned sc = lds0 + STAGE * stage + SC;
    const int k = kt & ~3;
    dma4_to_lds(s.sc + k, soff, sc + 256 * wave);
    if (ODD) dma4_to_lds(s.so + k, soff_s, sc + 4 * (BM + 64 * NPAIR));
    return Window{s.a + 128LL * kt, s.w + 128LL * kt, s.last};
  };
  auto copy_round = [&](Window &v, int stage, int i) __attribute__((always_inline)) {   // round i, in order
    const unsigned lds = lds0 + STAGE * stage + 1024 * wave;
    if (i < 4) {
      dma16_to_lds(v.a, voff_a, lds + 8192 * i);
      v.a += i < v.last ? step_a : 0u;
    } else if (ODD && i == 4) {
      dma16_to_lds(v.w, voff_s, lds0 + STAGE * stage + W1 + 1024 * (wave & 3));   // wavefronts 4-7: the same once more
    } else {
      dma16_to_lds(v.w, voff_w, lds + W0 + 8192 * (i - 4 - (ODD ? 1 : 0)));
      v.w += step_w;
    }
  };

  auto copy_bias = [&](int i) __attribute__((always_inline)) {
    if (p.bias && wave == 7) dma16_to_lds(p.bias + unit(wg + i * (int)gridDim.x).n0, 16 * min(lane, BN / 8 - 1), lds0 + BIAS + 1024 * (i & 1));
  };

  Source cur = source(0), nxt = cur;
  Window win;
  for (int stage = 0; stage < 2; ++stage) {      // the first two slices (there are two or more)
    win = open(cur, stage, stage);
#pragma unroll
    for (int i = 0; i < NDMA; ++i) copy_round(win, stage, i);
  }
  copy_bias(0);
  if (!p.bias) lds_write8(lds0 + BIAS + 16 * (tid & 127), zero8());
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  const int sw = gemm_swizzle(l16);
  const unsigned op = 128 * l16 + 16 * (q16 ^ sw);        // operand address inside 16 rows
  int stage = 0;

  auto run_tile = [&](auto ms_tag, const Tile t, int parity) __attribute__((always_inline)) {
    constexpr int MS = decltype(ms_tag)::value;            // token sub-tiles of a wavefront
    f32x4 acc[MS][NS];
    i32x8 tf[MS], wf[RING];                                // token operands, ring of weight operands
    int ts[MS], ws[RING];                                  // their scales
    unsigned tb, tb4, wb, wb4, tsb, wsb;
    auto use_stage = [&](int s, int k) __attribute__((always_inline)) {
      const unsigned st = lds0 + STAGE * s;
      tb = st + 2048 * MS * wm + op;
      wb = st + W0 + 4096 * wn + op;
      tb4 = tb ^ 64;
      wb4 = wb ^ 64;
      tsb = st + SC + 4 * (16 * MS * wm + l16) + (k & 3);
      wsb = st + SC + 4 * (BM + 32 * wn + l16) + (k & 3);
    };
    auto rd_t = [&](int a) __attribute__((always_inline)) {
      ts[a] = lds_read_byte(tsb + 64 * a);
      tf[a] = lds_read32(tb + 2048 * a, tb4 + 2048 * a);
    };
    auto rd_w = [&](int b, int slot) __attribute__((always_inline)) {
      const bool pair = b < 2 * NPAIR;
      ws[slot] = lds_read_byte(wsb + (pair ? 256 * (b >> 1) + 64 * (b & 1) : 4 * (64 * NPAIR) - 64 * wn));
      const unsigned off = pair ? 8192 * (b >> 1) + 2048 * (b & 1) : W1 - W0 - 2048 * wn;
      wf[slot] = lds_read32(wb + off, wb4 + off);
    };
    use_stage(stage, 0);
#pragma unroll
    for (int a = 0; a < MS; ++a) rd_t(a);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) rd_w(j, j);
    const int shift = wn ? SHIFT1 : 0, odd = wn ? 0 : 32 * NPAIR;   // where the pairs / the odd sub-tile start
    // the sums start from the bias: a lane's features of sub-tile b are four from here on
    const unsigned bias_at = lds0 + BIAS + 1024 * parity + 2 * (wn * 16 * NS);
    auto bias_of = [&](int b) __attribute__((always_inline)) {
      const unsigned f = b < 2 * NPAIR ? shift + 32 * (b >> 1) + 4 * (b & 1) + 8 * q16 : odd + 4 * q16;
      const bf16x4 v = *(const __attribute__((address_space(3))) bf16x4 *)(size_t)(bias_at + 2 * f);
      return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
    };

    // The stores of a tile are not waited for at the first barrier of the next one: all copies that it publishes were issued before them.  Stores of
    // a wavefront behind its last copy, at least (the tile before had as many tokens or more):
    constexpr int STORES = OUT8 ? 3 * MS : 4 * MS + (ODD ? (MS + 1) / 2 : 0);
    auto either = [&](bool next) __attribute__((always_inline)) {   // field by field: a selection, no branch
      return Source{next ? nxt.a : cur.a, next ? nxt.w : cur.w, next ? nxt.sc : cur.sc, next ? nxt.so : cur.so, next ? nxt.last : cur.last};
    };
    auto slice = [&](auto first_tag, int kt) __attribute__((always_inline)) {
      constexpr bool FIRST = decltype(first_tag)::value;
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        f32x4 b4;
        if (FIRST) b4 = bias_of(j);
        if (j == JB) {   // this slice has been read, the next one has arrived
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(FIRST ? STORES : 0) : "memory");
          stage ^= 1;
          use_stage(stage, kt + 1 == nk ? 0 : kt + 1);
          const bool over = kt + 2 >= nk;
          win = open(either(over), kt + 2 - (over ? nk : 0), stage ^ 1);
        }
        const int d = (j - JB + NS) % NS;   // steps since the barrier; the copies of slice kt + 2 go into the free stage
        if (!FIRST || j >= JB) {
#pragma unroll
          for (int r = PER * d; r < PER * d + PER; ++r)
            if (r < NDMA) copy_round(win, stage ^ 1, r);
        }
        rd_w((j + AHEAD) % NS, (j + AHEAD) % RING);
#pragma unroll
        for (int a = 0; a < MS; ++a) {
          acc[a][j] = mfma_q8(wf[j % RING], tf[a], FIRST ? b4 : acc[a][j], ws[j % RING], ts[a]);
          if (j == NS - 1) {
            __builtin_amdgcn_sched_barrier(0);   // not before the product that reads the registers
            rd_t(a);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    slice(std::true_type{}, 0);
    for (int kt = 1; kt < nk; ++kt) slice(std::false_type{}, kt);
#pragma unroll
    for (int r = PER * (NS - JB); r < NDMA; ++r) copy_round(win, stage ^ 1, r);   // the rest of the next tile's second slice

    // ---- activation, stores: what a step reads back from the wavefront's 2 KB is stored behind the arithmetic of the next one ----
    const int f0 = t.n0 + wn * 16 * NS, m0 = t.m0 + wm * 16 * MS;
    const unsigned xs = lds0 + XPOSE + 2048 * wave, xr = xs + 128 * (lane >> 3) + 16 * ((lane & 7) ^ gemm_swizzle(lane >> 3));
    typedef const __attribute__((address_space(3))) u32x4 *lds_cptr_u;
    auto finish = [](float x) { return ACT == Q8_GELU ? gelu_q8(x) : x; };
    if constexpr (OUT8) {
      // a wavefront's 128 features are a block: the largest magnitude over a lane's 32 and its token's four lanes, then 16 tokens x 128 bytes
      unsigned char *dst = p.C8 + (m0 + (lane >> 3)) * p.ld8 + f0 + 16 * (lane & 7);
      u32x4 r0, r1;
      auto store = [&]() __attribute__((always_inline)) {
        put16(dst, r0, p.past);
        put16(dst + 8 * p.ld8, r1, p.past);
        dst += 16 * p.ld8;
      };
#pragma unroll
      for (int a = 0; a < MS; ++a) {
        float x[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[u][e] = finish(acc[a][2 * u + (e >> 2)][e & 3]);
        const int byte = q8_scale_byte(max_across(block_max(x)));
        const float inv = q8_inverse(byte);
        u32x2 y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[u][e] *= inv;
          y[u] = u32x2{pack_e4m3(x[u][0], x[u][1], x[u][2], x[u][3]), pack_e4m3(x[u][4], x[u][5], x[u][6], x[u][7])};
        }
        if (a) store();
        if (q16 == 0) p.s8[(m0 + 16 * a + l16) * p.ls8 + (f0 >> 7)] = (unsigned char)byte;
#pragma unroll
        for (int u = 0; u < 4; ++u)   // chunk 2 u + (q16 >> 1) of the row, swizzled as everywhere
          *(__attribute__((address_space(3))) u32x2 *)(size_t)(xs + 128 * l16 + 16 * ((2 * u + (q16 >> 1)) ^ sw) + 8 * (q16 & 1)) = y[u];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        r0 = *(lds_cptr_u)(size_t)xr;
        r1 = *(lds_cptr_u)(size_t)((xr ^ 64) + 1024);   // rows 8 further: swizzle ^ 4
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      store();
    } else {
      // 16 tokens x 64 features at a time
      const unsigned xw = xs + 128 * l16;
      bf16_t *dst = p.C + f0 + shift + 8 * (lane & 7) + (m0 + (lane >> 3)) * p.ldc;
      u32x4 r0, r1;
      auto store = [&](int i) __attribute__((always_inline)) {   // of step i: sub-tile i % MS, features 64 (i / MS)
        put16(dst, r0, p.past);
        put16(dst + 8 * p.ldc, r1, p.past);
        dst += i % MS == MS - 1 ? 64 - (MS - 1) * 16 * p.ldc : 16 * p.ldc;
      };
#pragma unroll
      for (int i = 0; i < NPAIR / 2 * MS; ++i) {
        const int h = i / MS, a = i % MS;
        bf16x8 y[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) y[u][e] = (bf16_t)finish(acc[a][4 * h + 2 * u + (e >> 2)][e & 3]);
        if (i) store(i - 1);
#pragma unroll
        for (int u = 0; u < 2; ++u) lds_write8(xw + 16 * ((4 * u + q16) ^ sw), y[u]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        r0 = *(lds_cptr_u)(size_t)xr;
        r1 = *(lds_cptr_u)(size_t)((xr ^ 64) + 1024);   // rows 8 further: swizzle ^ 4
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      store(NPAIR / 2 * MS - 1);
      if (ODD) {
        bf16_t *to = p.C + f0 + odd + 8 * (lane & 1) + (m0 + (lane >> 1)) * p.ldc;
#pragma unroll
        for (int a = 0; a < MS; ++a) {
          bf16x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = (bf16_t)finish(acc[a][NS - 1][e]);
          lds_write4(xs + 32 * (16 * a + l16) + 8 * q16, y);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int a = 0; a < (MS + 1) / 2; ++a) {
          const u32x4 r = *(lds_cptr_u)(size_t)(xs + 1024 * a + 16 * lane);
          if (2 * a + 1 < MS || lane < 32) *reinterpret_cast<u32x4 *>(to + 32 * a * p.ldc) = r;   // 32 bytes: half of what memory takes at once
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
  };

  for (int i = 0; i < n_mine; ++i) {
    const Tile t = unit(wg + i * (int)gridDim.x);
    nxt = source(min(i + 1, n_mine - 1));
    copy_bias(min(i + 1, n_mine - 1));
    if (t.ms == 4) run_tile(std::integral_constant<int, 4>{}, t, i & 1);
    else if (t.ms == 3) run_tile(std::integral_constant<int, 3>{}, t, i & 1);
    else if (t.ms == 2) run_tile(std::integral_constant<int, 2>{}, t, i & 1);
    else run_tile(std::integral_constant<int, 1>{}, t, i & 1);
    cur = nxt;
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);            // the last copies
}

}  // namespace pab
