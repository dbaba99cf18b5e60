// Host side of fmha_cache_attention (include/fmha_varlen.h): argument checks (host memory only), the split of
// the cache over workgroups, and the launches on the caller's stream.
#include <hip/hip_runtime.h>

#include "cache_attention_kernels.h"
#include "host_checks.h"

namespace {

using fmha_host::check_ptr;
using fmha_host::check_stride;
using fmha_host::fail;
using fmha_host::misaligned;

struct Split {
  int32_t chunk, splits;
};

// Keys of a workgroup, and how many workgroups that makes of a sequence of `keys` keys.
Split split_of(int32_t batch, int32_t heads, int32_t kv_heads, int64_t keys) {
  const int64_t tiles = (heads / kv_heads + 15) / 16, items = batch * kv_heads * tiles;
  int64_t parts = (2048 + items - 1) / (items > 0 ? items : 1);
  const int64_t most = (keys + 255) / 256;
  if (parts > most) parts = most;
  if (parts < 1) parts = 1;
  int64_t chunk = (keys + parts - 1) / parts;
  chunk = (chunk + fmha::kCacheStep - 1) / fmha::kCacheStep * fmha::kCacheStep;
  if (chunk < fmha::kCacheStep) chunk = fmha::kCacheStep;
  parts = (keys + chunk - 1) / chunk;
  return Split{(int32_t)chunk, (int32_t)(parts < 1 ? 1 : parts)};
}

size_t bytes_of(const Split& s, int32_t batch, int32_t heads, int32_t head_dim) {
  return s.splits > 1 ? (size_t)s.splits * (size_t)batch * (size_t)heads * (size_t)(head_dim + 1) * sizeof(float) : 0;
}

template <typename T, int D>
int launch(const fmha::CacheArgs& a, hipStream_t st) {
  const int64_t grid = (int64_t)a.splits * a.batch * a.kv_heads * a.tiles;
  if (grid > 0x7fffffff) return fail(FMHA_ERR_INVALID_ARG, "%lld workgroups: too many", (long long)grid);
  fmha::cache_attention_kernel<T, D><<<(unsigned)grid, fmha::kCacheThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "cache attention launch failed: %s", hipGetErrorString(e));
  if (a.splits == 1) return FMHA_OK;
  const int64_t rows = (int64_t)a.batch * a.heads, per = fmha::kCacheThreads / 64;
  fmha::cache_join_kernel<T, D><<<(unsigned)((rows + per - 1) / per), fmha::kCacheThreads, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return fail(FMHA_ERR_HIP, "cache attention join launch failed: %s", hipGetErrorString(e));
  return FMHA_OK;
}

}  // namespace

extern "C" {

size_t fmha_cache_attention_workspace_size(int32_t batch, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t max_seqlen) {
  if (batch <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || (head_dim != 64 && head_dim != 128) || max_seqlen < 0) return 0;
  return bytes_of(split_of(batch, heads, kv_heads, max_seqlen), batch, heads, head_dim);
}

int fmha_cache_attention(const fmha_cache_t* c, int32_t heads, int32_t max_seqlen, float scale, const void* q, int64_t q_stride,
                         const void* k_cache, const void* v_cache, void* o, int64_t o_stride, float* lse, void* workspace,
                         size_t workspace_bytes, void* stream) {
  if (!c) return fail(FMHA_ERR_INVALID_ARG, "cache is null");
  fmha::CacheArgs a = {};
  int rc = fmha_host::check_cache(c, &a.page_stride);
  if (rc) return rc;
  if (c->head_dim != 64 && c->head_dim != 128) return fail(FMHA_ERR_UNSUPPORTED, "head_dim=%d, only 64 and 128 are supported", c->head_dim);
  if (heads <= 0 || heads > 65536 || heads % c->kv_heads)
    return fail(FMHA_ERR_INVALID_ARG, "heads=%d must be a positive multiple of kv_heads=%d", heads, c->kv_heads);
  if (scale - scale != 0.f) return fail(FMHA_ERR_INVALID_ARG, "scale is not finite");
  const int64_t dense = (int64_t)heads * c->head_dim;
  if ((rc = check_stride("q", q_stride, dense, &a.q_stride)) || (rc = check_stride("o", o_stride, dense, &a.o_stride))) return rc;
  fmha_host::g_err[0] = 0;
  if (c->batch == 0) return FMHA_OK;
  if ((rc = check_ptr("q", q, 16)) || (rc = check_ptr("o", o, 16)) || (rc = check_ptr("lse", lse, 4)) ||
      (rc = fmha_host::check_cache_pointers(c, k_cache, v_cache)))
    return rc;
  int64_t keys = max_seqlen > 0 ? max_seqlen : (int64_t)c->max_pages * c->page_size;
  if (keys > 0x7fffffff) keys = 0x7fffffff;
  const Split s = split_of(c->batch, heads, c->kv_heads, keys);
  const size_t need = bytes_of(s, c->batch, heads, c->head_dim);
  if (need) {
    if (!workspace) return fail(FMHA_ERR_WORKSPACE, "workspace is null (%zu bytes needed)", need);
    if (misaligned(workspace, 256)) return fail(FMHA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(FMHA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  }
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k_cache);
  a.v = static_cast<const uint16_t*>(v_cache);
  a.o = static_cast<uint16_t*>(o);
  a.lse = lse;
  a.table = c->block_table;
  a.seqlens = c->seqlens;
  a.batch = c->batch;
  a.heads = heads;
  a.kv_heads = c->kv_heads;
  a.group = heads / c->kv_heads;
  a.tiles = (a.group + 15) / 16;
  a.page_shift = fmha_host::page_shift(c);
  a.num_pages = c->num_pages;
  a.max_pages = c->max_pages;
  a.chunk = s.chunk;
  a.splits = s.splits;
  a.scale = scale;
  a.part_o = static_cast<float*>(workspace);
  a.part_lse = a.part_o + (size_t)s.splits * (size_t)c->batch * (size_t)heads * (size_t)c->head_dim;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (c->dtype == FMHA_F16) return c->head_dim == 64 ? launch<_Float16, 64>(a, st) : launch<_Float16, 128>(a, st);
  return c->head_dim == 64 ? launch<__bf16, 64>(a, st) : launch<__bf16, 128>(a, st);
}

}  // extern "C"
