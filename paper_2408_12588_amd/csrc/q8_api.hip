// libpab: the entry points around 8-bit rows and the query / key norm with rotation over several axes (declared in include/pab.h).
// A translation unit of its own because it is built with NaNs honoured: the quantisers look for them.
#include <algorithm>
#include <cmath>

#include "gemm_q8.hpp"
#include "gemm_q8_few.hpp"
#include "gemm_q8_stream.hpp"
#include "pab_internal.hpp"
#include "q8_plan.hpp"
#include "q8_rows.hpp"
#include "qk_norm_axes.hpp"

namespace {

using pab::aligned16;
using pab::fail;

constexpr long long MAX_PITCH = 1LL << 24;   // bytes: 32-bit offsets inside a tile of up to 256 rows

bool float_type(int dtype) { return dtype == PAB_BF16 || dtype == PAB_F32; }
int vector_elems(int dtype) { return dtype == PAB_BF16 ? 8 : 4; }   // elements of 16 bytes
long long blocks_of(long long K) { return (K + 127) / 128; }

int launched() {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(PAB_EDEVICE, "kernel launch failed: %s", hipGetErrorString(e));
  return PAB_OK;
}

// rows of K columns
int check_q8(const char *name, const pab_q8 *y, long long K) {
  if (!y || !y->data || !y->scale) return fail(PAB_EINVAL, "%s: data and scale must not be NULL", name);
  if (!aligned16(y->data) || (reinterpret_cast<uintptr_t>(y->scale) & 3u))
    return fail(PAB_EINVAL, "%s: data must be 16-byte, scale 4-byte aligned", name);
  if (y->ld % 16 || y->ld < 128 * blocks_of(K) || y->ld > MAX_PITCH)
    return fail(PAB_EINVAL, "%s: ld=%lld must be a multiple of 16 in [%lld, %lld]", name, y->ld, 128 * blocks_of(K), MAX_PITCH);
  if (y->ld_scale % 4 || y->ld_scale < (blocks_of(K) + 3) / 4 * 4 || y->ld_scale > MAX_PITCH)
    return fail(PAB_EINVAL, "%s: ld_scale=%lld must be a multiple of 4 in [%lld, %lld]", name, y->ld_scale, (blocks_of(K) + 3) / 4 * 4,
                MAX_PITCH);
  return PAB_OK;
}

int check_rows(long long rows, int K, int dtype) {
  if (!float_type(dtype)) return fail(PAB_EINVAL, "dtype %d is not bf16(0)/f32(1)", dtype);
  if (rows < 1 || K < 8 || K % 8) return fail(PAB_EINVAL, "rows=%lld must be >= 1, K=%d a positive multiple of 8", rows, K);
  if (rows > (1LL << 31) || rows * blocks_of(K) > pab::Q8_BLOCKS)
    return fail(PAB_EINVAL, "%lld rows of %d are too many for one launch", rows, K);
  return PAB_OK;
}

int check_pitch(const char *name, const void *p, long long ld, long long K, int dtype) {
  if (!p || !aligned16(p)) return fail(PAB_EINVAL, "%s must be non-NULL and 16-byte aligned", name);
  if (ld < K || ld % vector_elems(dtype))
    return fail(PAB_EINVAL, "%s: row pitch %lld must be >= %lld and a multiple of 16 bytes", name, ld, K);
  return PAB_OK;
}

// ---- products ----
template <int ACT, bool OUT8>
int launch_product(const pab::GemmPlan &g, const pab::GemmQ8Params &p, hipStream_t st) {
  const dim3 persistent((unsigned)std::min(g.n_units, pab::GEMM_CUS)), tiles((unsigned)((g.n_units + 7) / 8 * 8));
  switch (g.kernel) {
    case 8: hipLaunchKernelGGL((pab::gemm_q8_stream_kernel<8, 4, ACT, OUT8>), persistent, dim3(512), 0, st, p); break;
    case 9:
      if constexpr (!OUT8) hipLaunchKernelGGL((pab::gemm_q8_stream_kernel<9, 3, ACT, false>), persistent, dim3(512), 0, st, p);
      break;
    case 16:
      if constexpr (!OUT8) hipLaunchKernelGGL((pab::gemm_q8_few_kernel<1, ACT>), dim3((unsigned)g.n_units), dim3(512), 0, st, p);
      break;
    case 32:
      if constexpr (!OUT8) hipLaunchKernelGGL((pab::gemm_q8_few_kernel<2, ACT>), dim3((unsigned)g.n_units), dim3(512), 0, st, p);
      break;
    case 48:
      if constexpr (!OUT8) hipLaunchKernelGGL((pab::gemm_q8_few_kernel<4, ACT>), dim3((unsigned)g.n_units), dim3(512), 0, st, p);
      break;
    case 64:
      if constexpr (!OUT8) hipLaunchKernelGGL((pab::gemm_q8_tile_kernel<2, 2, 2, 2, 3, 1, ACT, false>), tiles, dim3(256), 0, st, p);
      break;
    case 65:
      if constexpr (!OUT8) hipLaunchKernelGGL((pab::gemm_q8_tile_kernel<2, 2, 2, 2, 3, 3, ACT, false>), tiles, dim3(768), 0, st, p);
      break;
    case 96:
      if constexpr (OUT8) hipLaunchKernelGGL((pab::gemm_q8_tile_kernel<2, 4, 2, 2, 3, 1, ACT, true>), tiles, dim3(512), 0, st, p);
      break;
    case 97: hipLaunchKernelGGL((pab::gemm_q8_tile_kernel<2, 4, 2, 2, 3, 2, ACT, OUT8>), tiles, dim3(1024), 0, st, p); break;
    case 113: hipLaunchKernelGGL((pab::gemm_q8_tile_kernel<2, 2, 3, 4, 2, 2, ACT, OUT8>), tiles, dim3(512), 0, st, p); break;
    case 128: hipLaunchKernelGGL((pab::gemm_q8_tile_kernel<2, 2, 4, 4, 2, 1, ACT, OUT8>), tiles, dim3(256), 0, st, p); break;
    case 129: hipLaunchKernelGGL((pab::gemm_q8_tile_kernel<2, 2, 4, 4, 2, 2, ACT, OUT8>), tiles, dim3(512), 0, st, p); break;
    case 161: hipLaunchKernelGGL((pab::gemm_q8_tile_kernel<2, 2, 5, 4, 2, 2, ACT, OUT8>), tiles, dim3(512), 0, st, p); break;
    default: return fail(PAB_EINVAL, "no product kernel %d", g.kernel);
  }
  return launched();
}

int plan_product(int M, int N, int K, bool out8, int act, pab::GemmPlan *g) {
  *g = pab::plan_q8(M, N, (int)blocks_of(K), out8, act == PAB_GELU);
  return g->kernel ? PAB_OK : fail(PAB_EINVAL, "M=%d N=%d: matrix too large for one launch", M, N);
}

// arguments checked, g from plan_product
int launch_planned(const pab::GemmPlan &g, int M, int N, int K, const pab_q8 *A, const pab_q8 *W, const void *bias, int act, void *C, long long ldc,
                   const pab_q8 *C8, hipStream_t st) {
  pab::GemmQ8Params p;
  p.A = static_cast<const unsigned char *>(A->data); p.sa = static_cast<const unsigned char *>(A->scale);
  p.W = static_cast<const unsigned char *>(W->data); p.sw = static_cast<const unsigned char *>(W->scale);
  p.lda = A->ld; p.lsa = A->ld_scale; p.ldw = W->ld; p.lsw = W->ld_scale;
  p.bias = static_cast<const pab::bf16_t *>(bias);
  p.C = static_cast<pab::bf16_t *>(C); p.ldc = ldc;
  p.C8 = nullptr; p.s8 = nullptr; p.ld8 = p.ls8 = 0;
  if (C8) {
    p.C8 = static_cast<unsigned char *>(C8->data); p.s8 = static_cast<unsigned char *>(C8->scale);
    p.ld8 = C8->ld; p.ls8 = C8->ld_scale;
  }
  p.M = M; p.N = N; p.nk = (int)blocks_of(K);
  p.n_mt = g.n_mt; p.n_nt = g.n_nt; p.by_feature = g.by_feature; p.n_inner = g.by_feature ? g.n_mt : g.n_nt;
  p.ms_tail = g.ms_tail; p.n_units = g.n_units;
  p.past = C8 ? pab::q8_past_caches(g.kernel, true, M, C8->data, 128 * blocks_of(N), C8->ld)
              : pab::q8_past_caches(g.kernel, false, M, C, 2LL * N, 2 * ldc);
  if (C8) return act ? launch_product<pab::Q8_GELU, true>(g, p, st) : launch_product<pab::Q8_NONE, true>(g, p, st);
  return act ? launch_product<pab::Q8_GELU, false>(g, p, st) : launch_product<pab::Q8_NONE, false>(g, p, st);
}

int product(int M, int N, int K, const pab_q8 *A, const pab_q8 *W, const void *bias, int act, void *C, long long ldc, const pab_q8 *C8,
            hipStream_t st) {
  if (M < 1 || N < 8 || N % 8 || K < 8 || K % 8)
    return fail(PAB_EINVAL, "M=%d must be >= 1, N=%d and K=%d positive multiples of 8", M, N, K);
  if (act != PAB_NONE && act != PAB_GELU) return fail(PAB_EINVAL, "activation %d is not none(0)/gelu(1)", act);
  int rc;
  if ((rc = check_q8("A", A, K)) != PAB_OK || (rc = check_q8("W", W, K)) != PAB_OK) return rc;
  if (bias && !aligned16(bias)) return fail(PAB_EINVAL, "bias must be 16-byte aligned");
  if (!C == !C8) return fail(PAB_EINVAL, "one of C and C8 must be given");
  if (C && (rc = check_pitch("C", C, ldc, N, PAB_BF16)) != PAB_OK) return rc;
  if (C8 && (rc = check_q8("C8", C8, N)) != PAB_OK) return rc;
  pab::GemmPlan g;
  if ((rc = plan_product(M, N, K, C8 != nullptr, act, &g)) != PAB_OK) return rc;
  return launch_planned(g, M, N, K, A, W, bias, act, C, ldc, C8, st);
}

// ---- layernorm + modulate into 8-bit rows ----
int ln_modulate_q8(int n_tok, int C, const void *x, const void *shift, const void *scale, const pab_q8 &h, hipStream_t st) {
  pab::LnQ8Params p;
  p.x = static_cast<const pab::bf16_t *>(x);
  p.shift = static_cast<const pab::bf16_t *>(shift);
  p.scale = static_cast<const pab::bf16_t *>(scale);
  p.data = static_cast<unsigned char *>(h.data); p.scales = static_cast<unsigned char *>(h.scale);
  p.ld = h.ld; p.ld_scale = h.ld_scale;
  p.n_tok = n_tok; p.C = C; p.eps = 1e-6f;
  const dim3 grid((unsigned)((n_tok + 3) / 4)), block(256);
  switch ((C + 511) / 512) {
    case 1: hipLaunchKernelGGL((pab::ln_modulate_q8_kernel<1>), grid, block, 0, st, p); break;
    case 2: hipLaunchKernelGGL((pab::ln_modulate_q8_kernel<2>), grid, block, 0, st, p); break;
    case 3: hipLaunchKernelGGL((pab::ln_modulate_q8_kernel<3>), grid, block, 0, st, p); break;
    default: hipLaunchKernelGGL((pab::ln_modulate_q8_kernel<4>), grid, block, 0, st, p); break;
  }
  return launched();
}

// Workgroups of a long list of rows.  In bf16 a wavefront has as many values for half the bytes and is bound by its instructions: as many as the chip
// holds at once (six per CU, 80 registers), which keep gamma and beta unpacked: 25440 tokens, 16 heads of 72, us at 1024 / 1536 / 2048 /
// 4096 / one row group each: 55.8 / 47.8 / 59.9 / 52.3 / 64.9.  In fp32 nothing is unpacked and more, shorter ones are better: 12720 tokens 51.5 /
// 51.1 / 51.6 / 49.2 / 48.9, at 8192 48.9.
template <typename T> constexpr long long QK_WGS = sizeof(T) == 2 ? 256 * 6 : 256 * 32;

template <typename T, int NORM>
int launch_qk(int D, const pab::QkAxesParams &p, hipStream_t st) {
  auto grid = [&](int lanes) { return dim3((unsigned)std::min((p.n_row + 4LL * (64 / lanes) - 1) / (4 * (64 / lanes)), QK_WGS<T>)); };
  switch (D) {
    case 32: hipLaunchKernelGGL((pab::qk_norm_axes_kernel<T, 4, NORM>), grid(4), dim3(256), 0, st, p); break;
    case 64: hipLaunchKernelGGL((pab::qk_norm_axes_kernel<T, 8, NORM>), grid(8), dim3(256), 0, st, p); break;
    case 72: hipLaunchKernelGGL((pab::qk_norm_axes_kernel<T, 9, NORM>), grid(9), dim3(256), 0, st, p); break;
    case 96: hipLaunchKernelGGL((pab::qk_norm_axes_kernel<T, 12, NORM>), grid(12), dim3(256), 0, st, p); break;
    default: hipLaunchKernelGGL((pab::qk_norm_axes_kernel<T, 16, NORM>), grid(16), dim3(256), 0, st, p); break;
  }
  return launched();
}

template <typename T>
int launch_qk_norm_axes(int norm, int D, const pab::QkAxesParams &p, hipStream_t st) {
  switch (norm) {
    case PAB_NORM_NONE: return launch_qk<T, pab::NORM_NONE>(D, p, st);
    case PAB_NORM_LAYER: return launch_qk<T, pab::NORM_LAYER>(D, p, st);
    default: return launch_qk<T, pab::NORM_RMS>(D, p, st);
  }
}

// places and pairs of the axes
int check_axes(const int places[3], const int axis_dim[3], int head_dim) {
  if (!places || !axis_dim) return fail(PAB_EINVAL, "places and axis_dim must not be NULL");
  long long sum = 0;
  for (int a = 0; a < 3; ++a) {
    if (places[a] < 1) return fail(PAB_EINVAL, "places[%d]=%d must be >= 1", a, places[a]);
    if (axis_dim[a] < 0 || axis_dim[a] % 2) return fail(PAB_EINVAL, "axis_dim[%d]=%d must be even and >= 0", a, axis_dim[a]);
    sum += axis_dim[a];
  }
  if (sum > head_dim) return fail(PAB_EINVAL, "the axes' sections are %lld features of a head of %d", sum, head_dim);
  if ((long long)places[0] * axis_dim[0] + (long long)places[1] * axis_dim[1] + (long long)places[2] * axis_dim[2] > (1LL << 30))
    return fail(PAB_EINVAL, "the axes have too many places");
  return PAB_OK;
}

}  // namespace

namespace pab {

size_t q8_bytes(long long rows, long long K) {
  const long long nb = blocks_of(K);
  if (rows < 1 || K < 1 || rows > (1LL << 40) || nb > (1LL << 17) || rows > (1LL << 56) / (129 * nb + 8)) return 0;
  const size_t data = ((size_t)rows * nb * 128 + 255) / 256 * 256;
  return data + ((size_t)rows * ((nb + 3) / 4 * 4) + 255) / 256 * 256;
}

pab_q8 q8_at(void *buffer, long long rows, long long K) {
  const long long nb = blocks_of(K);
  pab_q8 y;
  y.data = buffer;
  y.scale = static_cast<unsigned char *>(buffer) + ((size_t)rows * nb * 128 + 255) / 256 * 256;
  y.ld = 128 * nb;
  y.ld_scale = (nb + 3) / 4 * 4;
  return y;
}

int quantize(long long rows, int K, int dtype, const void *x, long long ldx, const pab_q8 *y, hipStream_t st) {
  int rc;
  if ((rc = check_rows(rows, K, dtype)) != PAB_OK || (rc = check_pitch("x", x, ldx, K, dtype)) != PAB_OK ||
      (rc = check_q8("y", y, K)) != PAB_OK)
    return rc;
  if (rows * blocks_of(K) >= pab::Q8_BLOCKS) return fail(PAB_EINVAL, "%lld rows of %d are too many for one launch", rows, K);
  QuantizeParams p;
  p.x = x; p.ldx = ldx;
  p.data = static_cast<unsigned char *>(y->data); p.scale = static_cast<unsigned char *>(y->scale);
  p.ld = y->ld; p.ld_scale = y->ld_scale; p.K = K;
  p.nb = divisor((unsigned)blocks_of(K));
  p.n_item = (unsigned)(rows * blocks_of(K));
  const dim3 grid((p.n_item + 15) / 16);
  if (dtype == PAB_BF16) hipLaunchKernelGGL((quantize_kernel<bf16_t>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((quantize_kernel<float>), grid, dim3(256), 0, st, p);
  return launched();
}

}  // namespace pab

extern "C" {

size_t pab_quantized_bytes(long long rows, int K) { return pab::q8_bytes(rows, K); }

int pab_quantized_layout(long long rows, int K, void *buffer, size_t bytes, pab_q8 *out) {
  if (!out) return fail(PAB_EINVAL, "out is NULL");
  const size_t need = pab::q8_bytes(rows, K);
  if (!need) return fail(PAB_EINVAL, "rows=%lld K=%d must be >= 1 and fit in memory", rows, K);
  if (!buffer || (reinterpret_cast<uintptr_t>(buffer) & 255u)) return fail(PAB_EINVAL, "buffer must be non-NULL and 256-byte aligned");
  if (bytes < need) return fail(PAB_ENOMEM, "buffer of %zu bytes, need %zu", bytes, need);
  *out = pab::q8_at(buffer, rows, K);
  return PAB_OK;
}

int pab_quantize(long long rows, int K, int dtype, const void *x, long long ldx, const pab_q8 *y, void *hip_stream) {
  return pab::quantize(rows, K, dtype, x, ldx, y, static_cast<hipStream_t>(hip_stream));
}

int pab_dequantize(long long rows, int K, int dtype, const pab_q8 *y, const void *x, long long ldx, const void *gate, void *out,
                   long long ldo, void *hip_stream) {
  int rc;
  if ((rc = check_rows(rows, K, dtype)) != PAB_OK || (rc = check_q8("y", y, K)) != PAB_OK ||
      (rc = check_pitch("out", out, ldo, K, dtype)) != PAB_OK || (x && (rc = check_pitch("x", x, ldx, K, dtype)) != PAB_OK))
    return rc;
  if (gate && !aligned16(gate)) return fail(PAB_EINVAL, "gate must be 16-byte aligned");
  pab::DequantizeParams p;
  p.data = static_cast<const unsigned char *>(y->data); p.scale = static_cast<const unsigned char *>(y->scale);
  p.x = x; p.gate = gate; p.out = out;
  p.ld = y->ld; p.ld_scale = y->ld_scale; p.ldx = ldx; p.ldo = ldo; p.K = K;
  p.nc = pab::divisor((unsigned)(K / 8));
  if (rows * (K / 8) > 0x7fffffffLL) return fail(PAB_EINVAL, "%lld rows of %d are too many for one launch", rows, K);
  p.n_item = (unsigned)(rows * (K / 8));
  const dim3 grid((unsigned)((p.n_item + 255LL) / 256));
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (dtype == PAB_BF16) hipLaunchKernelGGL((pab::dequantize_kernel<pab::bf16_t>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((pab::dequantize_kernel<float>), grid, dim3(256), 0, st, p);
  return launched();
}

int pab_linear_quantized(int M, int N, int K, const pab_q8 *A, const pab_q8 *W, const void *bias, int act, void *C, long long ldc,
                         const pab_q8 *C8, void *hip_stream) {
  return product(M, N, K, A, W, bias, act, C, ldc, C8, static_cast<hipStream_t>(hip_stream));
}

size_t pab_mlp_scratch_bytes_quantized(long long n_tok, int hidden, int inner) {
  const size_t h = pab::q8_bytes(n_tok, hidden), u = pab::q8_bytes(n_tok, inner);
  return h && u ? h + u : 0;
}

int pab_mlp_compute_quantized(long long n_tok, int hidden, int inner, const void *x, const pab_mlp_weights_quantized *w, void *scratch,
                              size_t scratch_bytes, void *out, void *hip_stream) {
  if (n_tok < 1 || n_tok > (1LL << 25) || hidden < 32 || hidden % 32 || hidden > 2048 || inner < 32 || inner % 32)
    return fail(PAB_EINVAL, "n_tok=%lld, hidden=%d (multiple of 32, <= 2048), inner=%d (multiple of 32)", n_tok, hidden, inner);
  if (!x || !w || !scratch || !out) return fail(PAB_EINVAL, "x, weights, scratch and out must be non-NULL");
  if (!w->shift || !w->scale) return fail(PAB_EINVAL, "MLP needs shift and scale");
  if (!aligned16(x) || !aligned16(out) || !aligned16(w->shift) || !aligned16(w->scale) || (reinterpret_cast<uintptr_t>(scratch) & 255u))
    return fail(PAB_EINVAL, "x, out, shift and scale must be 16-byte, scratch 256-byte aligned");
  const size_t need = pab_mlp_scratch_bytes_quantized(n_tok, hidden, inner);
  if (!need || scratch_bytes < need) return fail(PAB_ENOMEM, "scratch of %zu bytes, need %zu", scratch_bytes, need);
  int rc;   // everything is checked before the first launch
  if ((rc = check_q8("w1", &w->w1, hidden)) != PAB_OK || (rc = check_q8("w2", &w->w2, inner)) != PAB_OK) return rc;
  if (!aligned16(w->b1) || !aligned16(w->b2)) return fail(PAB_EINVAL, "b1 and b2 must be 16-byte aligned");
  pab::GemmPlan up, down;
  if ((rc = plan_product((int)n_tok, inner, hidden, true, PAB_GELU, &up)) != PAB_OK ||
      (rc = plan_product((int)n_tok, hidden, inner, false, PAB_NONE, &down)) != PAB_OK)
    return rc;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const pab_q8 h = pab::q8_at(scratch, n_tok, hidden);
  const pab_q8 u = pab::q8_at(static_cast<unsigned char *>(scratch) + pab::q8_bytes(n_tok, hidden), n_tok, inner);
  if ((rc = ln_modulate_q8((int)n_tok, hidden, x, w->shift, w->scale, h, st)) != PAB_OK) return rc;
  if ((rc = launch_planned(up, (int)n_tok, inner, hidden, &h, &w->w1, w->b1, PAB_GELU, nullptr, 0, &u, st)) != PAB_OK) return rc;
  return launch_planned(down, (int)n_tok, hidden, inner, &u, &w->w2, w->b2, PAB_NONE, out, hidden, nullptr, st);
}

long long pab_rope_factors_count(const int places[3], const int axis_dim[3]) {
  const int rc = check_axes(places, axis_dim, 1 << 30);
  if (rc != PAB_OK) return rc;
  long long n = 0;
  for (int a = 0; a < 3; ++a) n += (long long)places[a] * (axis_dim[a] / 2);
  return n;
}

int pab_rope_factors(const int places[3], const int axis_dim[3], const double origin[3], const double step[3], double theta, void *factors,
                     void *hip_stream) {
  const long long n = pab_rope_factors_count(places, axis_dim);
  if (n < 0) return (int)n;
  if (!(theta > 0.0) || !std::isfinite(theta)) return fail(PAB_EINVAL, "theta=%g must be positive", theta);
  pab::RopeFactorsParams p;
  for (int a = 0; a < 3; ++a) {
    p.n[a] = places[a]; p.half[a] = axis_dim[a] / 2;
    p.origin[a] = origin ? origin[a] : 0.0; p.step[a] = step ? step[a] : 1.0;
    if (!std::isfinite(p.origin[a]) || !std::isfinite(p.step[a])) return fail(PAB_EINVAL, "origin and step must be finite");
  }
  if (n == 0) return PAB_OK;
  if (!factors || !aligned16(factors)) return fail(PAB_EINVAL, "factors must be non-NULL and 16-byte aligned");
  p.out = static_cast<pab::f32x2 *>(factors);
  p.log_theta = std::log(theta);
  p.n_pair = (unsigned)n;
  hipLaunchKernelGGL(pab::rope_factors_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
  return launched();
}

int pab_qk_norm_rope(const pab_qk_norm *d, void *hip_stream) {
  if (!d) return fail(PAB_EINVAL, "the description is NULL");
  if (!float_type(d->dtype)) return fail(PAB_EINVAL, "dtype %d is not bf16(0)/f32(1)", d->dtype);
  const int D = d->head_dim;
  if (D != 32 && D != 64 && D != 72 && D != 96 && D != 128) return fail(PAB_EINVAL, "head_dim %d unsupported (32, 64, 72, 96 or 128)", D);
  if (d->norm != PAB_NORM_NONE && d->norm != PAB_NORM_LAYER && d->norm != PAB_NORM_RMS)
    return fail(PAB_EINVAL, "norm %d is not none(0)/layer(1)/rms(2)", d->norm);
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return fail(PAB_EINVAL, "eps=%g must be >= 0", (double)d->eps);
  int rc = check_axes(d->places, d->axis_dim, D);
  if (rc != PAB_OK) return rc;
  if (d->n_batch < 1 || d->heads_q < 1 || d->heads_k < 0) return fail(PAB_EINVAL, "n_batch=%d heads_q=%d must be >= 1, heads_k=%d >= 0", d->n_batch, d->heads_q, d->heads_k);
  const int heads = std::max(d->heads_q, d->heads_k);
  long long n = (long long)d->n_batch;
  for (int a = 0; a < 3; ++a) {
    n *= d->places[a];
    if (n > 0x7fffffffLL) return fail(PAB_EINVAL, "too many tokens");
  }
  if (n * heads > (1LL << 30)) return fail(PAB_EINVAL, "%lld tokens of %d heads are too many for one launch", n, heads);
  if ((rc = check_pitch("q", d->q, d->ld_q, (long long)d->heads_q * D, d->dtype)) != PAB_OK ||
      (rc = check_pitch("q_out", d->q_out, d->ld_q_out, (long long)d->heads_q * D, d->dtype)) != PAB_OK)
    return rc;
  if (d->heads_k && ((rc = check_pitch("k", d->k, d->ld_k, (long long)d->heads_k * D, d->dtype)) != PAB_OK ||
                     (rc = check_pitch("k_out", d->k_out, d->ld_k_out, (long long)d->heads_k * D, d->dtype)) != PAB_OK))
    return rc;
  if (!aligned16(d->gamma_q) || !aligned16(d->beta_q) || !aligned16(d->gamma_k) || !aligned16(d->beta_k) || !aligned16(d->factors))
    return fail(PAB_EINVAL, "gamma, beta and factors must be 16-byte aligned");
  pab::QkAxesParams p;
  p.q = d->q; p.q_out = d->q_out; p.ld_q = d->ld_q; p.ld_q_out = d->ld_q_out;
  p.k = d->k; p.k_out = d->k_out; p.ld_k = d->ld_k; p.ld_k_out = d->ld_k_out;
  p.gq = d->gamma_q; p.bq = d->beta_q; p.gk = d->gamma_k; p.bk = d->beta_k;
  p.factors = static_cast<const pab::f32x2 *>(d->factors);
  p.heads_q = d->heads_q; p.heads_k = d->heads_k; p.eps = d->eps;
  p.n_row = (unsigned)(n * heads);
  p.heads = pab::divisor((unsigned)heads);
  p.YX = pab::divisor((unsigned)((long long)d->places[1] * d->places[2]));
  p.X = pab::divisor((unsigned)d->places[2]);
  p.tokens = pab::divisor((unsigned)(n / d->n_batch));
  p.end_t = d->axis_dim[0] / 2; p.end_y = p.end_t + d->axis_dim[1] / 2; p.end_x = p.end_y + d->axis_dim[2] / 2;
  p.first_y = d->places[0] * (d->axis_dim[0] / 2); p.first_x = p.first_y + d->places[1] * (d->axis_dim[1] / 2);
  p.whole = d->axis_dim[0] % 8 == 0 && d->axis_dim[1] % 8 == 0 && d->axis_dim[2] % 8 == 0;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return d->dtype == PAB_BF16 ? launch_qk_norm_axes<pab::bf16_t>(d->norm, D, p, st) : launch_qk_norm_axes<float>(d->norm, D, p, st);
}

}  // extern "C"
