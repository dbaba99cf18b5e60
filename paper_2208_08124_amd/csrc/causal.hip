// Host side of the causal attention declared in include/fmha_varlen.h: argument checks (host memory only),
// workspace, and the launches on the caller's stream.  Nothing here allocates, copies to the host or waits.
#include <hip/hip_runtime.h>

#include "causal_bwd_kernels.h"
#include "causal_fwd_kernel.h"
#include "host_checks.h"

namespace {

using fmha_host::check_ptr;
using fmha_host::check_stride;
using fmha_host::fail;
using fmha_host::misaligned;

constexpr size_t kAlign = 256;
size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

// Tiles of 128 rows at most, for any lengths.
int64_t tile_capacity(int64_t batch, int64_t total) { return total / fmha::kTileRows + batch; }

struct Workspace {
  size_t list, lse2, dsum, bytes_fwd, bytes_bwd;  // offsets (the number of tiles stands at 0), sizes
};

Workspace carve(int64_t batch, int64_t total, int64_t heads) {
  Workspace w;
  w.list = kAlign;
  w.bytes_fwd = round_up(w.list + sizeof(fmha::TileItem) * (size_t)tile_capacity(batch, total));
  const size_t stat = round_up(sizeof(float) * ((size_t)total * (size_t)heads + 1));
  w.lse2 = w.bytes_fwd;
  w.dsum = w.lse2 + stat;
  w.bytes_bwd = w.dsum + stat;
  return w;
}

int check_common(const fmha_causal_params_t* p, bool bwd, fmha::CausalArgs* a) {
  if (!p) return fail(FMHA_ERR_INVALID_ARG, "params is null");
  if (p->head_dim != 64 && p->head_dim != 128) return fail(FMHA_ERR_UNSUPPORTED, "head_dim=%d, only 64 and 128 are supported", p->head_dim);
  if (int rc = fmha_host::check_dtype(p->dtype)) return rc;
  if (p->batch < 0) return fail(FMHA_ERR_INVALID_ARG, "batch=%d is negative", p->batch);
  if (p->total_tokens < 0) return fail(FMHA_ERR_INVALID_ARG, "total_tokens=%d is negative", p->total_tokens);
  if (p->heads <= 0 || p->heads > 65536 || p->kv_heads <= 0 || p->heads % p->kv_heads)
    return fail(FMHA_ERR_INVALID_ARG, "heads=%d must be a positive multiple of kv_heads=%d (and at most 65536)", p->heads, p->kv_heads);
  if (tile_capacity(p->batch, p->total_tokens) * p->heads > (int64_t)1 << 30)
    return fail(FMHA_ERR_INVALID_ARG, "total_tokens=%d, batch=%d, heads=%d: more than 2^30 tiles", p->total_tokens, p->batch, p->heads);
  if (p->flags & ~FMHA_FLAG_REUSE_SCHEDULE) return fail(FMHA_ERR_INVALID_ARG, "flags=%u: only FMHA_FLAG_REUSE_SCHEDULE is known here", p->flags);
  if (p->scale - p->scale != 0.f) return fail(FMHA_ERR_INVALID_ARG, "scale is not finite");
  if (!p->cu_seqlens) return fail(FMHA_ERR_INVALID_ARG, "cu_seqlens is null");
  if (misaligned(p->cu_seqlens, 4)) return fail(FMHA_ERR_INVALID_ARG, "cu_seqlens must be 4-byte aligned");
  if (const int32_t* cu = p->cu_seqlens_host) {
    if (cu[0] != 0) return fail(FMHA_ERR_INVALID_ARG, "cu_seqlens_host[0]=%d, expected 0", cu[0]);
    for (int i = 0; i < p->batch; i++) {
      if (cu[i + 1] < cu[i]) return fail(FMHA_ERR_INVALID_ARG, "cu_seqlens_host decreases at %d (%d -> %d)", i, cu[i], cu[i + 1]);
      if (p->max_seqlen > 0 && cu[i + 1] - cu[i] > p->max_seqlen)
        return fail(FMHA_ERR_INVALID_ARG, "sequence %d has %d tokens, more than max_seqlen=%d", i, cu[i + 1] - cu[i], p->max_seqlen);
    }
    if (cu[p->batch] > p->total_tokens)
      return fail(FMHA_ERR_INVALID_ARG, "cu_seqlens_host[batch]=%d exceeds total_tokens=%d", cu[p->batch], p->total_tokens);
  }
  const Workspace w = carve(p->batch, p->total_tokens, p->heads);
  const size_t need = bwd ? w.bytes_bwd : w.bytes_fwd;
  if (!p->workspace) return fail(FMHA_ERR_WORKSPACE, "workspace is null (%zu bytes needed)", need);
  if (misaligned(p->workspace, kAlign)) return fail(FMHA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (p->workspace_bytes < need) return fail(FMHA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", p->workspace_bytes, need);
  *a = fmha::CausalArgs{};
  const int64_t dense_q = (int64_t)p->heads * p->head_dim, dense_k = (int64_t)p->kv_heads * p->head_dim;
  int rc;
  if ((rc = check_stride("q", p->q_stride, dense_q, &a->q_stride)) || (rc = check_stride("k", p->k_stride, dense_k, &a->k_stride)) ||
      (rc = check_stride("v", p->v_stride, dense_k, &a->v_stride)) || (rc = check_stride("o", p->o_stride, dense_q, &a->o_stride)))
    return rc;
  if (bwd && ((rc = check_stride("do", p->do_stride, dense_q, &a->do_stride)) || (rc = check_stride("dq", p->dq_stride, dense_q, &a->dq_stride)) ||
              (rc = check_stride("dk", p->dk_stride, dense_k, &a->dk_stride)) || (rc = check_stride("dv", p->dv_stride, dense_k, &a->dv_stride))))
    return rc;
  char* base = static_cast<char*>(p->workspace);
  a->cu = p->cu_seqlens;
  a->batch = p->batch;
  a->total = p->total_tokens;
  a->heads = p->heads;
  a->kv_heads = p->kv_heads;
  a->group = p->heads / p->kv_heads;
  a->scale = p->scale;
  if (p->batch > fmha::kCausalSelf) {
    a->count = reinterpret_cast<int32_t*>(base);
    a->list = reinterpret_cast<fmha::TileItem*>(base + w.list);
  }
  if (bwd) {
    a->lse2 = reinterpret_cast<float*>(base + w.lse2);
    a->dsum = reinterpret_cast<float*>(base + w.dsum);
  }
  return FMHA_OK;
}

// Workgroups for the tiles of `heads` heads: one each, by the sizes that the host knows (the kernels go on in strides, so
// that a wrong max_seqlen costs time only).
unsigned grid_of(const fmha_causal_params_t* p, int heads) {
  int64_t tiles = tile_capacity(p->batch, p->total_tokens);
  if (p->max_seqlen > 0) {
    const int64_t by_length = ((int64_t)p->max_seqlen + fmha::kTileRows - 1) / fmha::kTileRows * p->batch;
    if (by_length < tiles) tiles = by_length;
  }
  int64_t g = tiles * heads;
  return (unsigned)(g < 1 ? 1 : g);
}

int launch_list(const fmha_causal_params_t* p, const fmha::CausalArgs& a, hipStream_t st) {
  if (!a.list || (p->flags & FMHA_FLAG_REUSE_SCHEDULE)) return FMHA_OK;
  fmha::causal_list_kernel<<<1, fmha::kCausalListThreads, 0, st>>>(a, const_cast<int32_t*>(a.count), const_cast<fmha::TileItem*>(a.list),
                                                                   (int)tile_capacity(p->batch, p->total_tokens));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "tile list launch failed: %s", hipGetErrorString(e));
  return FMHA_OK;
}

template <typename T, int D>
int launch_fwd(const fmha_causal_params_t* p, const fmha::CausalArgs& a, hipStream_t st) {
  fmha::causal_fwd_kernel<T, D><<<grid_of(p, a.heads), fmha::kThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "causal forward launch failed: %s", hipGetErrorString(e));
  return FMHA_OK;
}

template <typename T, int D>
int launch_bwd(const fmha_causal_params_t* p, const fmha::CausalArgs& a, hipStream_t st) {
  fmha::causal_dq_kernel<T, D><<<grid_of(p, a.heads), fmha::kThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "causal dQ launch failed: %s", hipGetErrorString(e));
  fmha::causal_dkv_kernel<T, D><<<grid_of(p, a.kv_heads), fmha::kThreads, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "causal dK/dV launch failed: %s", hipGetErrorString(e));
  return FMHA_OK;
}

const uint16_t* in(const void* p) { return static_cast<const uint16_t*>(p); }
uint16_t* out(void* p) { return static_cast<uint16_t*>(p); }

}  // namespace

extern "C" {

size_t fmha_causal_workspace_size(int32_t batch, int32_t total_tokens, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                  int32_t need_bwd) {
  if (batch < 0 || total_tokens < 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || (head_dim != 64 && head_dim != 128)) return 0;
  const Workspace w = carve(batch, total_tokens, heads);
  return need_bwd ? w.bytes_bwd : w.bytes_fwd;
}

int fmha_causal_fwd(const fmha_causal_params_t* p, const void* q, const void* k, const void* v, void* o, float* lse, void* stream) {
  fmha::CausalArgs a;
  int rc = check_common(p, false, &a);
  if (rc) return rc;
  fmha_host::g_err[0] = 0;
  if (p->batch == 0 || p->total_tokens == 0) return FMHA_OK;
  if ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("k", k, 16)) || (rc = check_ptr("v", v, 16)) || (rc = check_ptr("o", o, 16)) ||
      (rc = check_ptr("lse", lse, 4)))
    return rc;
  a.q = in(q);
  a.k = in(k);
  a.v = in(v);
  a.o = out(o);
  a.lse = lse;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if ((rc = launch_list(p, a, st))) return rc;
  if (p->dtype == FMHA_F16) return p->head_dim == 64 ? launch_fwd<_Float16, 64>(p, a, st) : launch_fwd<_Float16, 128>(p, a, st);
  return p->head_dim == 64 ? launch_fwd<__bf16, 64>(p, a, st) : launch_fwd<__bf16, 128>(p, a, st);
}

int fmha_causal_bwd(const fmha_causal_params_t* p, const void* q, const void* k, const void* v, const void* o, const void* d_o,
                    const float* lse, void* dq, void* dk, void* dv, void* stream) {
  fmha::CausalArgs a;
  int rc = check_common(p, true, &a);
  if (rc) return rc;
  fmha_host::g_err[0] = 0;
  if (p->batch == 0 || p->total_tokens == 0) return FMHA_OK;
  if ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("k", k, 16)) || (rc = check_ptr("v", v, 16)) || (rc = check_ptr("o", o, 16)) ||
      (rc = check_ptr("d_o", d_o, 16)) || (rc = check_ptr("lse", lse, 4)) || (rc = check_ptr("dq", dq, 16)) || (rc = check_ptr("dk", dk, 16)) ||
      (rc = check_ptr("dv", dv, 16)))
    return rc;
  a.q = in(q);
  a.k = in(k);
  a.v = in(v);
  a.o_in = in(o);
  a.d_o = in(d_o);
  a.lse = const_cast<float*>(lse);
  a.dq = out(dq);
  a.dk = out(dk);
  a.dv = out(dv);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if ((rc = launch_list(p, a, st))) return rc;
  if (p->dtype == FMHA_F16) return p->head_dim == 64 ? launch_bwd<_Float16, 64>(p, a, st) : launch_bwd<_Float16, 128>(p, a, st);
  return p->head_dim == 64 ? launch_bwd<__bf16, 64>(p, a, st) : launch_bwd<__bf16, 128>(p, a, st);
}

}  // extern "C"
