// Argument checks that the host sides of the decoder's entry points share (host memory only).
#pragma once
#include <stdint.h>

#include "../../include/fmha_varlen.h"
#include "host_error.h"

namespace fmha_host {

inline bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

inline int check_ptr(const char* name, const void* ptr, size_t align) {
  if (!ptr) return fail(FMHA_ERR_INVALID_ARG, "%s is null", name);
  if (misaligned(ptr, align)) return fail(FMHA_ERR_INVALID_ARG, "%s is not %zu-byte aligned", name, align);
  return FMHA_OK;
}

inline int check_dtype(int32_t dtype) {
  if (dtype != FMHA_F16 && dtype != FMHA_BF16) return fail(FMHA_ERR_UNSUPPORTED, "dtype=%d is neither FMHA_F16 nor FMHA_BF16", dtype);
  return FMHA_OK;
}

// Elements between the rows (tokens) of a tensor; 0 stands for `dense`.
inline int check_stride(const char* name, int64_t s, int64_t dense, int64_t* out) {
  if (s == 0) s = dense;
  if (s < dense || (s & 7) || s > ((int64_t)1 << 24))
    return fail(FMHA_ERR_INVALID_ARG, "%s_stride=%lld must be 0 or a multiple of 8 from heads*head_dim=%lld to 2^24", name,
                (long long)s, (long long)dense);
  *out = s;
  return FMHA_OK;
}

// The cache's sizes (not its pointers, which a call with nothing to do does not look at); *page_stride <- elements between pages.
inline int check_cache(const fmha_cache_t* c, int64_t* page_stride) {
  int rc = check_dtype(c->dtype);
  if (rc) return rc;
  if (c->kv_heads < 1 || c->kv_heads > 65536) return fail(FMHA_ERR_INVALID_ARG, "kv_heads=%d must be positive (and at most 65536)", c->kv_heads);
  if (c->batch < 0) return fail(FMHA_ERR_INVALID_ARG, "batch=%d is negative", c->batch);
  if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
    return fail(FMHA_ERR_INVALID_ARG, "page_size=%d must be a power of two, at most 65536", c->page_size);
  if (c->num_pages < 0 || c->max_pages < 0) return fail(FMHA_ERR_INVALID_ARG, "num_pages=%d, max_pages=%d: negative", c->num_pages, c->max_pages);
  if ((int64_t)c->max_pages * c->page_size > (int64_t)1 << 30)
    return fail(FMHA_ERR_INVALID_ARG, "max_pages=%d pages of %d tokens: more than 2^30 tokens", c->max_pages, c->page_size);
  const int64_t dense = (int64_t)c->kv_heads * c->page_size * c->head_dim;
  if (c->page_stride && (c->page_stride < dense || (c->page_stride & 7)))
    return fail(FMHA_ERR_INVALID_ARG, "page_stride=%lld must be 0 or a multiple of 8 that is >= kv_heads*page_size*head_dim=%lld",
                (long long)c->page_stride, (long long)dense);
  *page_stride = c->page_stride ? c->page_stride : dense;
  return FMHA_OK;
}

inline int check_cache_pointers(const fmha_cache_t* c, const void* k_cache, const void* v_cache) {
  int rc;
  if ((rc = check_ptr("k_cache", k_cache, 16)) || (rc = check_ptr("v_cache", v_cache, 16)) ||
      (rc = check_ptr("block_table", c->block_table, 4)) || (rc = check_ptr("seqlens", c->seqlens, 4)))
    return rc;
  return FMHA_OK;
}

inline int page_shift(const fmha_cache_t* c) {
  int s = 0;
  while ((1 << s) < c->page_size) s++;
  return s;
}

}  // namespace fmha_host
