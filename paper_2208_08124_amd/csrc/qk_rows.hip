// Host side of the norm, rotation and cache-append entry points declared in include/fmha_varlen.h:
// argument checks (host memory only) and launches on the caller's stream.  Nothing here
// allocates, copies to the host or waits.
#include <hip/hip_runtime.h>

#include <cmath>

#include "host_checks.h"
#include "qk_rows_kernels.h"

namespace {

using fmha_host::fail;

using fmha_host::check_ptr;
using fmha_host::check_stride;
using fmha_host::misaligned;

// What all of the entry points have: sizes, dtype, norm, rotation.
int check_heads(int32_t q_heads, int32_t k_heads, int32_t head_dim, int32_t dtype, float eps, const float* gamma_q,
                const float* gamma_k, const fmha_rope_t* rope, fmha::QkRows* a) {
  if (int rc = fmha_host::check_dtype(dtype)) return rc;
  if (q_heads < 0 || k_heads < 0 || q_heads > 65536 || k_heads > 65536)
    return fail(FMHA_ERR_INVALID_ARG, "%d query heads, %d key heads: invalid numbers", q_heads, k_heads);
  if (head_dim <= 0 || (head_dim & 15)) return fail(FMHA_ERR_INVALID_ARG, "head_dim=%d must be a positive multiple of 16", head_dim);
  if (head_dim > 256) return fail(FMHA_ERR_UNSUPPORTED, "head_dim=%d, at most 256 is supported", head_dim);
  if (!(eps >= 0.f) || eps - eps != 0.f) return fail(FMHA_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (misaligned(gamma_q, 16) || misaligned(gamma_k, 16)) return fail(FMHA_ERR_INVALID_ARG, "gamma is not 16-byte aligned");
  const int r = rope->rotary_dim;
  if (r < 0 || (r & 15) || r > head_dim) return fail(FMHA_ERR_INVALID_ARG, "rotary_dim=%d must be a multiple of 16 from 0 to head_dim=%d", r, head_dim);
  if (r) {
    if (rope->layout != FMHA_ROPE_HALF && rope->layout != FMHA_ROPE_INTERLEAVED)
      return fail(FMHA_ERR_INVALID_ARG, "rope layout=%d is neither FMHA_ROPE_HALF nor FMHA_ROPE_INTERLEAVED", rope->layout);
    int rc = check_ptr("inv_freq", rope->inv_freq, 8);
    if (rc) return rc;
    if (rope->magnitude - rope->magnitude != 0.f) return fail(FMHA_ERR_INVALID_ARG, "rope magnitude is not finite");
  }
  *a = fmha::QkRows{};
  a->nq = q_heads;
  a->nk = k_heads;
  a->dim = head_dim;
  a->lph = head_dim / 16;
  a->lp2 = 1;
  while (a->lp2 < a->lph) a->lp2 *= 2;
  a->eps = eps;
  a->gamma_q = gamma_q;
  a->gamma_k = gamma_k;
  a->rot = r;
  a->inv_freq = rope->inv_freq;
  a->magnitude = rope->magnitude;
  return FMHA_OK;
}

// Heads that a wavefront takes of a row at a time: a power of two up to 64 / lp2, the largest that leaves no more than a fifth
// of the places empty over `heads` (neighbouring heads share lines and a position; 18 000 rows of 12 + 1 heads of 64 take 22 us
// forward sixteen heads at a time, 33 one at a time).
int heads_at_a_time(int heads, int slots) {
  int g = slots;
  while (g > 1 && (heads + g - 1) / g * g * 4 > heads * 5) g /= 2;
  return g;
}

// How the work is cut: see QkRows.  A wavefront forms the angles of its rows once for all heads that it takes, but
// while there are fewer than `enough` wavefronts, the heads of a row are dealt to several.  Returns their number.
int64_t cut(fmha::QkRows* a, int64_t enough) {
  const int slots = 64 / a->lp2, heads = a->nq + a->nk + a->nv;
  a->gs = heads_at_a_time(heads, slots);
  const int tpw = slots / a->gs, times = (heads + a->gs - 1) / a->gs;
  const int64_t groups = ((int64_t)a->rows + tpw - 1) / tpw;
  int64_t iters = groups * times / enough;
  iters = iters < 1 ? 1 : iters > times ? times : iters;
  a->iters = (int)iters;
  a->parts = (times + a->iters - 1) / a->iters;
  return groups * a->parts;
}

constexpr int kWaves = fmha::kQkThreads / 64, kFwdWaves = 256 * 4 * 8, kBwdGroups = 256 * 3;  // (what the chip holds at a time)

int64_t fwd_grid(fmha::QkRows* a) { return (cut(a, kFwdWaves) + kWaves - 1) / kWaves; }

// Workgroups of the backward, which go over the items in strides: as many as run at a time.  32 265 rows, 32 + 8 heads of 128:
// 206 us, 233 with 1024 workgroups, the last 256 of which run by themselves.
int bwd_grid(fmha::QkRows* a) {
  const int64_t g = (cut(a, kBwdGroups * kWaves) + kWaves - 1) / kWaves;
  return (int)(g > kBwdGroups ? kBwdGroups : g < 1 ? 1 : g);
}

template <bool CACHE>
int launch_rows(const fmha::QkRows& a, int64_t grid, int dtype, int layout, hipStream_t st) {
  if (grid >= (int64_t)1 << 24)  // (a launch holds less than 2^32 threads)
    return fail(FMHA_ERR_INVALID_ARG, "rows=%d of %d heads: more workgroups than a launch holds", a.rows, a.nq + a.nk + a.nv);
  const bool inter = layout == FMHA_ROPE_INTERLEAVED && a.rot;
  if (dtype == FMHA_F16) {
    if (inter)
      fmha::qk_rows_kernel<_Float16, true, CACHE><<<(unsigned)grid, fmha::kQkThreads, 0, st>>>(a);
    else
      fmha::qk_rows_kernel<_Float16, false, CACHE><<<(unsigned)grid, fmha::kQkThreads, 0, st>>>(a);
  } else {
    if (inter)
      fmha::qk_rows_kernel<__bf16, true, CACHE><<<(unsigned)grid, fmha::kQkThreads, 0, st>>>(a);
    else
      fmha::qk_rows_kernel<__bf16, false, CACHE><<<(unsigned)grid, fmha::kQkThreads, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "norm and rotation launch failed: %s", hipGetErrorString(e));
  return FMHA_OK;
}

int check_qk(const fmha_qk_params_t* p, fmha::QkRows* a) {
  if (!p) return fail(FMHA_ERR_INVALID_ARG, "params is null");
  if (p->rows < 0) return fail(FMHA_ERR_INVALID_ARG, "rows=%d is negative", p->rows);
  int rc = check_heads(p->q_heads, p->k_heads, p->head_dim, p->dtype, p->eps, p->gamma_q, p->gamma_k, &p->rope, a);
  if (rc) return rc;
  if (p->rope.rotary_dim && !p->positions && !p->cu_seqlens)
    return fail(FMHA_ERR_INVALID_ARG, "positions and cu_seqlens are both null: a rotation needs one of them");
  if (p->cu_seqlens && p->batch < 1) return fail(FMHA_ERR_INVALID_ARG, "batch=%d, cu_seqlens needs at least one sequence", p->batch);
  if (misaligned(p->positions, 4) || misaligned(p->cu_seqlens, 4) || misaligned(p->n_rows, 4))
    return fail(FMHA_ERR_INVALID_ARG, "positions / cu_seqlens / n_rows must be 4-byte aligned");
  a->rows = p->rows;
  a->positions = p->positions;
  a->cu = p->cu_seqlens;
  a->batch = p->batch;
  a->n_rows = p->n_rows;
  const int64_t dense_q = (int64_t)p->q_heads * p->head_dim, dense_k = (int64_t)p->k_heads * p->head_dim;
  if ((rc = check_stride("q", p->q_stride, dense_q, &a->q_stride)) || (rc = check_stride("k", p->k_stride, dense_k, &a->k_stride)) ||
      (rc = check_stride("q_out", p->q_out_stride, dense_q, &a->qo_stride)) ||
      (rc = check_stride("k_out", p->k_out_stride, dense_k, &a->ko_stride)))
    return rc;
  return FMHA_OK;
}

}  // namespace

extern "C" {

int fmha_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, int32_t original_context,
                          double fast, double slow, double* inv_freq, float* magnitude) {
  if (rotary_dim <= 0 || (rotary_dim & 1)) return fail(FMHA_ERR_INVALID_ARG, "rotary_dim=%d must be positive and even", rotary_dim);
  if (!(base > 1.) || std::isinf(base)) return fail(FMHA_ERR_INVALID_ARG, "base=%g must be finite and above 1", base);
  if (scaling < FMHA_ROPE_PLAIN || scaling > FMHA_ROPE_PARTS) return fail(FMHA_ERR_INVALID_ARG, "scaling=%d is not one of FMHA_ROPE_*", scaling);
  if (scaling != FMHA_ROPE_PLAIN && (!(factor >= 1.) || std::isinf(factor)))
    return fail(FMHA_ERR_INVALID_ARG, "factor=%g must be finite and at least 1", factor);
  if (scaling == FMHA_ROPE_BASE && rotary_dim <= 2) return fail(FMHA_ERR_INVALID_ARG, "FMHA_ROPE_BASE needs rotary_dim > 2");
  if (scaling == FMHA_ROPE_PARTS && (original_context <= 0 || !(fast > slow) || !(slow > 0.) || std::isinf(fast)))
    return fail(FMHA_ERR_INVALID_ARG, "FMHA_ROPE_PARTS needs original_context=%d > 0 and fast=%g > slow=%g > 0", original_context, fast, slow);
  if (!inv_freq) return fail(FMHA_ERR_INVALID_ARG, "inv_freq is null");
  fmha_host::g_err[0] = 0;
  const double r = rotary_dim;
  if (scaling == FMHA_ROPE_BASE) base *= std::pow(factor, r / (r - 2.));
  double low = 0., high = 0.;
  if (scaling == FMHA_ROPE_PARTS) {
    const double two_pi = 6.283185307179586477;
    low = std::floor(r * std::log(original_context / (two_pi * fast)) / (2. * std::log(base)));
    high = std::ceil(r * std::log(original_context / (two_pi * slow)) / (2. * std::log(base)));
    low = low < 0. ? 0. : low > r - 1. ? r - 1. : low;
    high = high < 0. ? 0. : high > r - 1. ? r - 1. : high;
    if (high <= low) high = low + 0.001;  // a step
  }
  for (int i = 0; i < rotary_dim / 2; i++) {
    const double f = std::pow(base, -2. * i / r);
    double share = 0.;  // of the pair's frequency that is divided
    if (scaling == FMHA_ROPE_LINEAR) share = 1.;
    if (scaling == FMHA_ROPE_PARTS) {
      share = (i - low) / (high - low);
      share = share < 0. ? 0. : share > 1. ? 1. : share;
    }
    inv_freq[i] = share > 0. ? f * (1. - share) + f / factor * share : f;
  }
  if (magnitude) *magnitude = scaling == FMHA_ROPE_PARTS ? (float)(0.1 * std::log(factor) + 1.) : 1.f;
  return FMHA_OK;
}

int fmha_qk_norm_rope_fwd(const fmha_qk_params_t* p, const void* q, const void* k, void* q_out, void* k_out, void* stream) {
  fmha::QkRows a;
  int rc = check_qk(p, &a);
  if (rc) return rc;
  fmha_host::g_err[0] = 0;
  if (a.rows == 0 || a.nq + a.nk == 0) return FMHA_OK;
  if (a.nq && ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("q_out", q_out, 16)))) return rc;
  if (a.nk && ((rc = check_ptr("k", k, 16)) || (rc = check_ptr("k_out", k_out, 16)))) return rc;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.qo = static_cast<uint16_t*>(q_out);
  a.ko = static_cast<uint16_t*>(k_out);
  const int64_t grid = fwd_grid(&a);
  return launch_rows<false>(a, grid, p->dtype, p->rope.layout, static_cast<hipStream_t>(stream));
}

size_t fmha_qk_norm_rope_bwd_workspace_size(int32_t rows, int32_t q_heads, int32_t k_heads, int32_t head_dim) {
  if (rows < 0 || q_heads < 0 || k_heads < 0 || q_heads > 65536 || k_heads > 65536 || head_dim <= 0 || (head_dim & 15) || head_dim > 256)
    return 0;
  fmha::QkRows a = {};
  a.rows = rows;
  a.nq = q_heads;
  a.nk = k_heads;
  a.lp2 = 1;
  while (a.lp2 < head_dim / 16) a.lp2 *= 2;
  return (size_t)bwd_grid(&a) * 2 * (size_t)head_dim * sizeof(float);
}

int fmha_qk_norm_rope_bwd(const fmha_qk_params_t* p, const void* dq_out, const void* dk_out, const void* q, const void* k,
                          void* dq, void* dk, float* dgamma_q, float* dgamma_k, void* workspace, size_t workspace_bytes,
                          void* stream) {
  fmha::QkRows a;
  int rc = check_qk(p, &a);
  if (rc) return rc;
  if ((rc = check_stride("dq", p->dq_stride, (int64_t)a.nq * a.dim, &a.dq_stride)) ||
      (rc = check_stride("dk", p->dk_stride, (int64_t)a.nk * a.dim, &a.dk_stride)))
    return rc;
  if (!a.nq) a.gamma_q = nullptr;
  if (!a.nk) a.gamma_k = nullptr;
  const bool rows = a.rows > 0;
  if (rows && a.nq && ((rc = check_ptr("dq_out", dq_out, 16)) || (rc = check_ptr("dq", dq, 16)))) return rc;
  if (rows && a.nk && ((rc = check_ptr("dk_out", dk_out, 16)) || (rc = check_ptr("dk", dk, 16)))) return rc;
  if (a.gamma_q && ((rows && (rc = check_ptr("q", q, 16))) || (rc = check_ptr("dgamma_q", dgamma_q, 4)))) return rc;
  if (a.gamma_k && ((rows && (rc = check_ptr("k", k, 16))) || (rc = check_ptr("dgamma_k", dgamma_k, 4)))) return rc;
  const bool sums = a.gamma_q || a.gamma_k;
  const int grid = bwd_grid(&a);
  if (sums) {
    const size_t need = (size_t)grid * 2 * (size_t)a.dim * sizeof(float);
    if (!workspace || misaligned(workspace, 16)) return fail(FMHA_ERR_WORKSPACE, "workspace is null or not 16-byte aligned (%zu bytes needed)", need);
    if (workspace_bytes < need) return fail(FMHA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  }
  fmha_host::g_err[0] = 0;
  if (!sums && (!rows || a.nq + a.nk == 0)) return FMHA_OK;
  // (with no rows the kernels still run where there is a gamma: its gradient is written, zeros)
  a.dyq = static_cast<const uint16_t*>(dq_out);
  a.dyk = static_cast<const uint16_t*>(dk_out);
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.dq = static_cast<uint16_t*>(dq);
  a.dk = static_cast<uint16_t*>(dk);
  a.partial = static_cast<float*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool inter = p->rope.layout == FMHA_ROPE_INTERLEAVED && a.rot;
  if (p->dtype == FMHA_F16) {
    if (inter)
      fmha::qk_rows_bwd_kernel<_Float16, true><<<grid, fmha::kQkThreads, 0, st>>>(a);
    else
      fmha::qk_rows_bwd_kernel<_Float16, false><<<grid, fmha::kQkThreads, 0, st>>>(a);
  } else {
    if (inter)
      fmha::qk_rows_bwd_kernel<__bf16, true><<<grid, fmha::kQkThreads, 0, st>>>(a);
    else
      fmha::qk_rows_bwd_kernel<__bf16, false><<<grid, fmha::kQkThreads, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "norm and rotation backward launch failed: %s", hipGetErrorString(e));
  if (!sums) return FMHA_OK;
  fmha::qk_gamma_kernel<<<(unsigned)((2 * a.dim + 63) / 64), fmha::kQkGammaThreads, 0, st>>>(a.partial, grid, a.dim,
                                                                                          a.gamma_q ? dgamma_q : nullptr,
                                                                                          a.gamma_k ? dgamma_k : nullptr);
  e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "gamma-sum launch failed: %s", hipGetErrorString(e));
  return FMHA_OK;
}

int fmha_cache_append(const fmha_cache_t* c, const fmha_append_params_t* p, const void* q, const void* k, const void* v,
                      void* q_out, void* k_cache, void* v_cache, void* stream) {
  if (!c || !p) return fail(FMHA_ERR_INVALID_ARG, "cache or params is null");
  fmha::QkRows a;
  int rc = check_heads(p->q_heads, c->kv_heads, c->head_dim, c->dtype, p->eps, p->gamma_q, p->gamma_k, &p->rope, &a);
  if (rc) return rc;
  int64_t page_stride;
  if ((rc = fmha_host::check_cache(c, &page_stride))) return rc;
  if (p->rows < 0) return fail(FMHA_ERR_INVALID_ARG, "rows=%d is negative", p->rows);
  if (!p->cu_seqlens && p->rows != c->batch)
    return fail(FMHA_ERR_INVALID_ARG, "rows=%d differs from batch=%d, and there are no cu_seqlens", p->rows, c->batch);
  const int64_t dense_q = (int64_t)p->q_heads * c->head_dim, dense_k = (int64_t)c->kv_heads * c->head_dim;
  int64_t v_stride;
  if ((rc = check_stride("q", p->q_stride, dense_q, &a.q_stride)) || (rc = check_stride("k", p->k_stride, dense_k, &a.k_stride)) ||
      (rc = check_stride("v", p->v_stride, dense_k, &v_stride)) || (rc = check_stride("q_out", p->q_out_stride, dense_q, &a.qo_stride)))
    return rc;
  fmha_host::g_err[0] = 0;
  if (p->rows == 0 || c->batch == 0) return FMHA_OK;
  if ((rc = check_ptr("k", k, 16)) || (rc = check_ptr("v", v, 16)) || (rc = fmha_host::check_cache_pointers(c, k_cache, v_cache))) return rc;
  if (p->q_heads && ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("q_out", q_out, 16)))) return rc;
  if (misaligned(p->cu_seqlens, 4)) return fail(FMHA_ERR_INVALID_ARG, "cu_seqlens must be 4-byte aligned");
  a.rows = p->rows;
  a.nv = c->kv_heads;
  a.v_stride = v_stride;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.qo = static_cast<uint16_t*>(q_out);
  a.kc = static_cast<uint16_t*>(k_cache);
  a.vc = static_cast<uint16_t*>(v_cache);
  a.cu = p->cu_seqlens;
  a.batch = c->batch;
  a.seqlens = c->seqlens;
  a.table = c->block_table;
  a.page_stride = page_stride;
  a.page_shift = fmha_host::page_shift(c);
  a.num_pages = c->num_pages;
  a.max_pages = c->max_pages;
  const int64_t grid = fwd_grid(&a);
  return launch_rows<true>(a, grid, c->dtype, p->rope.layout, static_cast<hipStream_t>(stream));
}

}  // extern "C"
