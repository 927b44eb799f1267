// Products of 8-bit rows (q8_common.hpp): C[M, N] = act(A W^T + bias), A [M, K] tokens, W [N, K] weights, fp32 sums on the matrix core, one
// rounding on the way out: to bf16, or to 8-bit rows again (the scale of 128 features of a token is found on the sums themselves).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 rows of 128 e4m3 bytes of either operand, 32 bytes a lane, and a scale byte per lane; both
// scales go into the products.  A K slice is 128 bytes of a row, one cache line, which is one block of the format: every slice has
// one scale per row.  Bytes, LDS reads and clocks of a slice are those of a 64-column slice of the bf16 projections (gemm_common.hpp), at twice the
// work; the layouts below are theirs: chunk q of stage row r at position q ^ ((r >> 1) & 7), weight rows of a pair of sub-tiles in
// the order 8 (i >> 2) + 4 u + (i & 3), results through LDS into row order.  A lane takes chunks q16 and q16 + 4 of its row as its 32 bytes:
// which columns meet which does not matter as long as it is the same in both operands.
#pragma once
#include <type_traits>
#include "gemm_common.hpp"
#include "q8_common.hpp"

namespace pab {

typedef __attribute__((ext_vector_type(8))) int i32x8;

struct GemmQ8Params {
  const unsigned char *A, *W;        // e4m3, row pitches lda, ldw bytes
  const unsigned char *sa, *sw;      // exponent bytes, row pitches lsa, lsw (multiples of 4)
  const bf16_t *bias;                // [N] or nullptr
  bf16_t *C;                         // bf16 output, row pitch ldc elements, or
  unsigned char *C8, *s8;            // 8-bit rows, row pitches ld8, ls8 bytes
  long long lda, ldw, lsa, lsw, ldc, ld8, ls8;
  int M, N, nk;                      // nk: K slices of 128
  int n_mt, n_nt;                    // token / feature tiles
  int by_feature, n_inner;           // consecutive tiles share their features (1) or their tokens (0), n_inner of them
  int ms_tail, n_units;              // large tiles: see gemm_q8_stream.hpp
  int past;                          // the output goes past the caches (8-bit rows: of large tiles only)
};

enum { Q8_NONE = 0, Q8_GELU = 1 };

__device__ __forceinline__ i32x8 lds_read32(unsigned addr, unsigned addr4) {   // chunks q16 and q16 + 4 of a row: addresses 64 ^ apart
  typedef __attribute__((ext_vector_type(4))) int i32x4;
  typedef const __attribute__((address_space(3))) i32x4 *ptr;
  const i32x4 lo = *(ptr)(size_t)addr, hi = *(ptr)(size_t)addr4;
  return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}
__device__ __forceinline__ int lds_read_byte(unsigned addr) {
  return *(const __attribute__((address_space(3))) unsigned char *)(size_t)addr;
}
__device__ __forceinline__ f32x4 mfma_q8(i32x8 w, i32x8 t, f32x4 c, int sw, int st) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, t, c, 0, 0, 0, sw, 0, st);   // both e4m3, byte 0 of the scales
}

// A wavefront-wide copy of 4 bytes per lane straight into LDS: lane i's at LDS byte address lds_addr + 4 i (lds_addr uniform).  Lanes that are
// switched off copy nothing.  Completion as for dma16_to_lds.
__device__ __forceinline__ void dma4_to_lds(const void *from, unsigned lds_addr) {
  lds_addr = __builtin_amdgcn_readfirstlane(lds_addr);
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off"
               :
               : "v"(from), "{m0}"(lds_addr)
               : "memory");
}

// ... from base + voff (base uniform)
__device__ __forceinline__ void dma4_to_lds(const void *base, unsigned voff, unsigned lds_addr) {
  lds_addr = __builtin_amdgcn_readfirstlane(lds_addr);
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(voff), "s"(base), "{m0}"(lds_addr)
               : "memory");
}

// 16 bytes of the output, past the caches or not.  In asm: the compiler makes one store of two to the same address and drops the hint.  The two cycles
// behind it are the instruction's, before its data registers may be written again.
__device__ __forceinline__ void put16(void *to, u32x4 v, int past) {
  if (past) asm volatile("global_store_dwordx4 %0, %1, off nt\n\ts_nop 1" ::"v"(to), "v"(v) : "memory");
  else *reinterpret_cast<u32x4 *>(to) = v;
}

// Largest finite magnitude of a token over the four lanes (lane bits 4 and 5) that hold its features
__device__ __forceinline__ unsigned max_across(unsigned x) {
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(b[0], b[1]);
}

// GELU in its tanh form, x / (1 + exp(-2 u)), u = sqrt(2 / pi) (x + 0.044715 x^3) (products written out: the same bits wherever it is inlined)
__device__ __forceinline__ float gelu_q8(float x) {
#pragma clang fp contract(off)
  const float s = __builtin_fmaf(x * x, -0.102943236f, -2.302208198f);   // -2 sqrt(2 / pi) log2(e) (0.044715 x^2 + 1)
  return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * s));
}

// ---- everything that does not fill the chip with large tiles: one workgroup per tile, WM x WN wavefronts of MS x NS sub-tiles, K slices
//      through a ring of NST stages; KG groups of such wavefronts take every KG-th slice through rings of their own, their sums
//      are added through LDS.  OUT8: a tile's features are whole blocks of 128. ----
template <int WM, int WN, int MS, int NS, int NST, int KG, int ACT, bool OUT8>
__global__ __launch_bounds__(64 * WM * WN * KG, KG > 1 ? WM * WN * KG / 4 : 2) void gemm_q8_tile_kernel(const GemmQ8Params p) {
  constexpr int NW = WM * WN, BM = 16 * MS * WM, BN = 16 * NS * WN;
  constexpr int ROWS = BM + BN, STAGE = 132 * ROWS;      // bytes: rows, then a dword of scales for each
  constexpr int ROUNDS = ROWS / 8, MYR = ROUNDS / NW, TOKR = BM / 8 / NW;   // copy rounds: all, per wavefront, of token rows
  constexpr int SPW = ROWS / NW, SCN = (SPW + 63) / 64;  // scale dwords a wavefront copies, in copies of 64
  static_assert(ROUNDS % NW == 0 && (BM / 8) % NW == 0 && ROWS % NW == 0, "copies must deal evenly to the wavefronts");
  static_assert(NS % 2 == 0 && (NS == 2 || NS % 4 == 0) && STAGE % 16 == 0, "sub-tiles come in pairs");
  static_assert(NST >= 2 && NST <= 3 && (NST - 2) * (MYR + SCN) < 16, "vmcnt immediates");
  constexpr int PART = 1024 * MS * NS * NW;              // bytes of a group's sums
  constexpr int MAXIMA = OUT8 ? 4 * BM * WN : 0;         // a token's largest magnitude, by wavefront column
  static_assert(NW * 2048 + MAXIMA + (KG - 1) * PART <= KG * NST * STAGE, "output staging must fit the rings");
  static_assert(!OUT8 || (BN % 128 == 0 && 128 % (16 * NS) == 0), "tiles are whole blocks");

  __shared__ __attribute__((aligned(16))) unsigned char smem[KG * NST * STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int kg = __builtin_amdgcn_readfirstlane(tid >> 6) / NW, wave = __builtin_amdgcn_readfirstlane(tid >> 6) % NW;
  const int l16 = lane & 15, q16 = lane >> 4;
  const int wm = wave / WN, wn = wave % WN;
  const unsigned lds_all = (unsigned)(size_t)((__attribute__((address_space(3))) unsigned char *)smem);
  const unsigned lds0 = lds_all + NST * STAGE * kg;      // the group's ring

  // every XCD takes a contiguous run of tiles
  const int n_tiles = p.n_mt * p.n_nt, per = (n_tiles + 7) >> 3;
  const int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= n_tiles) return;
  const int outer = id / p.n_inner, in = id - outer * p.n_inner;
  const int m0 = (p.by_feature ? in : outer) * BM, n0 = (p.by_feature ? outer : in) * BN;
  const int M = p.M, N = p.N, nk = p.nk;

  // round r = wave + NW i: stage rows 8 r .. 8 r + 7, token rows first.  Rows past the matrix re-read its last row; what
  // they produce is never stored.  LDS row i of a 32-row weight pair: sub-tile i >> 4, operand row i & 15.
  auto feature_of = [](int w) { return (w & ~31) + 8 * ((w & 15) >> 2) + 4 * ((w >> 4) & 1) + (w & 3); };
  auto source = [&](int row) { return row < BM ? min(row, M - 1 - m0) : min(feature_of(row - BM), N - 1 - n0); };   // in the tile
  const unsigned char *A = p.A + m0 * p.lda, *W = p.W + n0 * p.ldw;
  unsigned voff[MYR];
  const int cq = (lane & 7) ^ gemm_swizzle(8 * wave + (lane >> 3));   // 8 NW rows further the swizzle is the same
  static_assert(NW % 2 == 0, "swizzle period of 16 rows");
#pragma unroll
  for (int i = 0; i < MYR; ++i)
    voff[i] = (unsigned)(source(8 * (wave + NW * i) + (lane >> 3)) * (i < TOKR ? p.lda : p.ldw) + 16 * cq);
  // scales: wavefront w copies those of stage rows SPW w .. SPW w + SPW - 1
  const unsigned char *scales[SCN];
#pragma unroll
  for (int c = 0; c < SCN; ++c) {
    const int row = SPW * wave + min(64 * c + lane, SPW - 1);
    scales[c] = row < BM ? p.sa + (m0 + source(row)) * p.lsa : p.sw + (n0 + source(row)) * p.lsw;
  }
  auto issue = [&](int kt, int stage) __attribute__((always_inline)) {
    const int k = __builtin_amdgcn_readfirstlane(kt);
    const unsigned to = lds0 + STAGE * stage;
#pragma unroll
    for (int c = 0; c < SCN; ++c)
      if (64 * c + lane < SPW) dma4_to_lds(scales[c] + (k & ~3), to + 128 * ROWS + 4 * (SPW * wave + 64 * c));
#pragma unroll
    for (int i = 0; i < MYR; ++i) dma16_to_lds((i < TOKR ? A : W) + 128LL * k, voff[i], to + 1024 * (wave + NW * i));
  };
  // group g takes the slices kt = g (mod KG); all groups go through the same number of steps
  const int n_mine = (nk - kg + KG - 1) / KG, n_step = (nk + KG - 1) / KG;
  const int npre = n_mine < NST - 1 ? n_mine : NST - 1;
  for (int s = 0; s < npre; ++s) issue(KG * s + kg, s);

  // accumulators start from the bias: lane's features of sub-tile b are 32 (b / 2) + 8 q16 + 4 (b % 2) + 0..3
  f32x4 acc[MS][NS];
#pragma unroll
  for (int b = 0; b < NS; ++b) {
    const int n = n0 + wn * 16 * NS + 32 * (b >> 1) + 8 * q16 + 4 * (b & 1);
    f32x4 bv = {0.0f, 0.0f, 0.0f, 0.0f};
    if (kg == 0 && p.bias && n < N) {
      const bf16x4 b4 = *reinterpret_cast<const bf16x4 *>(p.bias + n);
#pragma unroll
      for (int e = 0; e < 4; ++e) bv[e] = (float)b4[e];
    }
#pragma unroll
    for (int a = 0; a < MS; ++a) acc[a][b] = bv;
  }
  const unsigned op = 128 * l16 + 16 * (q16 ^ gemm_swizzle(l16));
  const int t_row = wm * 16 * MS, w_row = BM + wn * 16 * NS;

  int stage = 0, next = npre % NST;
  for (int s = 0; s < n_step; ++s) {
    // slice s of the group has landed (this wavefront's share); one more may be in flight
    if (NST == 3 && s + 1 < n_mine) __builtin_amdgcn_s_waitcnt(0x0F70 | (MYR + SCN));
    else __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();                        // ... everyone's share; all are done with slice s - 1
    if (s + NST - 1 < n_mine) {
      issue(KG * (s + NST - 1) + kg, next);
      next = next + 1 == NST ? 0 : next + 1;
    }
    if (KG > 1 && s >= n_mine) break;       // the last step, for groups that have no slice left
    const unsigned st = lds0 + STAGE * stage;
    const unsigned ss = st + 128 * ROWS + 4 * l16 + ((KG * s + kg) & 3);   // the slice's byte of each row's scales
    stage = stage + 1 == NST ? 0 : stage + 1;
    i32x8 tf[MS], wf[NS];
    int ts[MS], ws[NS];
#pragma unroll
    for (int a = 0; a < MS; ++a) {
      ts[a] = lds_read_byte(ss + 4 * (t_row + 16 * a));
      tf[a] = lds_read32(st + 128 * (t_row + 16 * a) + op, st + 128 * (t_row + 16 * a) + (op ^ 64));
    }
#pragma unroll
    for (int b = 0; b < NS; ++b) {
      ws[b] = lds_read_byte(ss + 4 * (w_row + 16 * b));
      wf[b] = lds_read32(st + 128 * (w_row + 16 * b) + op, st + 128 * (w_row + 16 * b) + (op ^ 64));
    }
#pragma unroll
    for (int b = 0; b < NS; ++b)
#pragma unroll
      for (int a = 0; a < MS; ++a) acc[a][b] = mfma_q8(wf[b], tf[a], acc[a][b], ws[b], ts[a]);
  }

  if (KG > 1) {   // groups 1 .. leave their sums in LDS, 16 bytes per lane, group 0 adds them to its own
    __syncthreads();
    typedef __attribute__((address_space(3))) f32x4 *lds_ptr_f4;
    const unsigned part = lds_all + 2048 * NW + MAXIMA + 1024 * MS * NS * wave + 16 * lane;
    if (kg) {
#pragma unroll
      for (int a = 0; a < MS; ++a)
#pragma unroll
        for (int b = 0; b < NS; ++b) *(lds_ptr_f4)(size_t)(part + PART * (kg - 1) + 1024 * (NS * a + b)) = acc[a][b];
    }
    __syncthreads();
    if (!OUT8 && kg) return;                // OUT8: the groups meet once more below
    if (kg == 0) {
#pragma unroll
      for (int g = 0; g < KG - 1; ++g)
#pragma unroll
        for (int a = 0; a < MS; ++a)
#pragma unroll
          for (int b = 0; b < NS; ++b) acc[a][b] += *(lds_ptr_f4)(size_t)(part + PART * g + 1024 * (NS * a + b));
    }
  }
  if (ACT == Q8_GELU) {
#pragma unroll
    for (int a = 0; a < MS; ++a)
#pragma unroll
      for (int b = 0; b < NS; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[a][b][e] = gelu_q8(acc[a][b][e]);
  }
  if (KG == 1) __syncthreads();              // the ring is free
  const unsigned xs = lds0 + 2048 * wave;
  const int mw = m0 + wm * 16 * MS, fw = n0 + wn * 16 * NS;

  if constexpr (OUT8) {
    // the largest magnitude of a token's block: over a lane's features, its four lanes, the wavefronts of the block
    constexpr int WPB = 128 / (16 * NS);                   // wavefronts side by side in a block
    typedef __attribute__((address_space(3))) unsigned *lds_ptr_u;
    const unsigned maxima = lds_all + 2048 * NW;
    unsigned big[MS];
#pragma unroll
    for (int a = 0; a < MS; ++a) {
      float x[NS / 2][8];
#pragma unroll
      for (int u = 0; u < NS / 2; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = fw + 32 * u + 8 * q16 < N ? acc[a][2 * u + (e >> 2)][e & 3] : 0.0f;   // padding columns are zero
      big[a] = max_across(block_max(x));
#pragma unroll
      for (int u = 0; u < NS / 2; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[a][2 * u + (e >> 2)][e & 3] = x[u][e];
    }
    if constexpr (WPB > 1) {
      if (kg == 0 && q16 == 0) {
#pragma unroll
        for (int a = 0; a < MS; ++a) *(lds_ptr_u)(size_t)(maxima + 4 * (BM * wn + wm * 16 * MS + 16 * a + l16)) = big[a];
      }
      __syncthreads();
#pragma unroll
      for (int a = 0; a < MS; ++a)
#pragma unroll
        for (int i = 0; i < WPB; ++i)
          big[a] = max(big[a], *(lds_ptr_u)(size_t)(maxima + 4 * (BM * (wn / WPB * WPB + i) + wm * 16 * MS + 16 * a + l16)));
    }
    if (kg) return;
    // 16 tokens x 16 NS bytes at a time: a lane's 8 features of a pair of sub-tiles are 8 bytes
    constexpr int SEG = 16 * NS, CPR = SEG / 16;           // bytes of a row segment, 16-byte chunks of it
#pragma unroll
    for (int a = 0; a < MS; ++a) {
      const int byte = q8_scale_byte(big[a]);
      const float inv = q8_inverse(byte);
#pragma unroll
      for (int u = 0; u < NS / 2; ++u) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = acc[a][2 * u + (e >> 2)][e & 3] * inv;
        *(__attribute__((address_space(3))) u32x2 *)(size_t)(xs + SEG * l16 + 32 * u + 8 * q16) =
            u32x2{pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7])};
      }
      const int m = mw + 16 * a + l16;
      if (wn % WPB == 0 && q16 == 0 && m < M && fw < N) p.s8[m * p.ls8 + (fw >> 7)] = (unsigned char)byte;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int i = 0; i < (16 * CPR + 63) / 64; ++i) {
        const int row = 64 / CPR * i + lane / CPR, mr = mw + 16 * a + row;
        if (row < 16 && mr < M && (fw & ~127) < N)         // a block that has a column is written whole
          *reinterpret_cast<u32x4 *>(p.C8 + mr * p.ld8 + fw + 16 * (lane % CPR)) =
              *(const __attribute__((address_space(3))) u32x4 *)(size_t)(xs + SEG * row + 16 * (lane % CPR));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  } else {
    // ---- 16 tokens x SEG features at a time through 2 KB per wavefront ----
    constexpr int SEG = NS >= 4 ? 64 : 32;
    constexpr int CPR = SEG / 8, RPI = 64 / CPR;           // chunks per row segment, rows per store instruction
    auto xpos = [](int row, int q) { return SEG == 64 ? q ^ gemm_swizzle(row) : q ^ ((row >> 2) & 2); };
#pragma unroll
    for (int h = 0; h < 16 * NS / SEG; ++h) {
      const int n = fw + SEG * h + 8 * (lane % CPR);
#pragma unroll
      for (int a = 0; a < MS; ++a) {
#pragma unroll
        for (int u = 0; u < SEG / 32; ++u) {
          bf16x8 y;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = (bf16_t)acc[a][SEG / 16 * h + 2 * u + (e >> 2)][e & 3];
          lds_write8(xs + 2 * SEG * l16 + 16 * xpos(l16, 4 * u + q16), y);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < 16 / RPI; ++i) {
          const int row = RPI * i + lane / CPR, m = mw + 16 * a + row;
          const bf16x8 r = lds_read8(xs + 2 * SEG * row + 16 * xpos(row, lane % CPR));
          if (m < M && n < N) put16(p.C + m * p.ldc + n, __builtin_bit_cast(u32x4, r), p.past);   // N is a multiple of 8
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
  }
}

}  // namespace pab
