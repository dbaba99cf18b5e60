/* The host-side validation of the decoder's entry points (no GPU work: every call below is refused before anything
 * is launched, or has nothing to do) in a library whose host code was built with -fsanitize=address,undefined.  What is
 * read on the host (cu_seqlens_host) and written there (inv_freq) has exactly the promised size. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "fmha_varlen.h"

#define EXPECT(call, code)                                                                       \
  do {                                                                                           \
    const int rc_ = (call);                                                                      \
    if (rc_ != (code)) {                                                                         \
      fprintf(stderr, "%s:%d: %s returned %d (%s), expected %d\n", __FILE__, __LINE__, #call, rc_, \
              fmha_last_error(), (code));                                                        \
      return 1;                                                                                  \
    }                                                                                            \
  } while (0)

int main(void) {
  void* dev = aligned_alloc(256, 1 << 16);
  /* frequencies: every scaling, the smallest sizes, extreme arguments */
  for (int32_t r = 2; r <= 256; r += 2) {
    double* f = malloc(sizeof(double) * (size_t)(r / 2));
    float m;
    EXPECT(fmha_rope_frequencies(r, 10000., FMHA_ROPE_PLAIN, 0., 0, 0., 0., f, NULL), FMHA_OK);
    EXPECT(fmha_rope_frequencies(r, 1e9, FMHA_ROPE_LINEAR, 1e6, 0, 0., 0., f, &m), FMHA_OK);
    EXPECT(fmha_rope_frequencies(r, 1.0000001, FMHA_ROPE_PARTS, 1., 1, 1e9, 1e-9, f, &m), FMHA_OK);
    EXPECT(fmha_rope_frequencies(r, 10000., FMHA_ROPE_PARTS, 64., 0x7fffffff, 32., 1., f, &m), FMHA_OK);
    for (int32_t i = 0; i < r / 2; i++)
      if (!isfinite(f[i])) return 1;
    EXPECT(fmha_rope_frequencies(r, 10000., FMHA_ROPE_BASE, 8., 0, 0., 0., f, &m), r > 2 ? FMHA_OK : FMHA_ERR_INVALID_ARG);
    EXPECT(fmha_rope_frequencies(r, NAN, FMHA_ROPE_PLAIN, 1., 0, 0., 0., f, &m), FMHA_ERR_INVALID_ARG);
    EXPECT(fmha_rope_frequencies(r + 1, 10000., FMHA_ROPE_PLAIN, 1., 0, 0., 0., f, &m), FMHA_ERR_INVALID_ARG);
    free(f);
  }
  /* norm and rotation */
  fmha_qk_params_t q;
  memset(&q, 0, sizeof(q));
  q.rows = 3, q.q_heads = 2, q.k_heads = 1, q.head_dim = 64, q.dtype = FMHA_BF16, q.cu_seqlens = dev, q.batch = 1;
  q.rope.rotary_dim = 64, q.rope.inv_freq = dev, q.rope.magnitude = 1.f, q.gamma_q = dev;
  EXPECT(fmha_qk_norm_rope_fwd(NULL, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  EXPECT(fmha_qk_norm_rope_fwd(&q, NULL, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  EXPECT(fmha_qk_norm_rope_bwd(&q, dev, dev, dev, dev, dev, dev, dev, dev, dev, 4, NULL), FMHA_ERR_WORKSPACE);
  EXPECT(fmha_qk_norm_rope_bwd(&q, dev, dev, NULL, dev, dev, dev, dev, dev, dev, 1 << 16, NULL), FMHA_ERR_INVALID_ARG);
  for (int32_t rows = 0; rows < 2; rows++) /* the largest sizes that are taken: no overflow on the way to the workspace check */
    for (int32_t h = 0; h <= 65536; h += 65536) {
      fmha_qk_params_t x = q;
      x.rows = rows ? 0x7fffffff : 0, x.q_heads = h, x.k_heads = h, x.head_dim = 16, x.rope.rotary_dim = 16;
      x.q_stride = x.k_stride = x.q_out_stride = x.k_out_stride = x.dq_stride = x.dk_stride = h ? 1 << 20 : 8;
      fmha_qk_norm_rope_bwd_workspace_size(x.rows, h, h, 16);
      EXPECT(fmha_qk_norm_rope_bwd(&x, dev, dev, dev, dev, dev, dev, dev, dev, NULL, 0, NULL), h ? FMHA_ERR_WORKSPACE : FMHA_OK);
    }
  /* the cache */
  fmha_cache_t c;
  memset(&c, 0, sizeof(c));
  c.batch = 2, c.kv_heads = 1, c.head_dim = 64, c.dtype = FMHA_F16, c.page_size = 16, c.num_pages = 2, c.max_pages = 2;
  c.block_table = dev, c.seqlens = dev;
  fmha_append_params_t a;
  memset(&a, 0, sizeof(a));
  a.rows = 3;
  EXPECT(fmha_cache_append(&c, &a, dev, dev, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  a.rows = 2, a.q_heads = 1;
  EXPECT(fmha_cache_append(&c, &a, NULL, dev, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  EXPECT(fmha_cache_append(NULL, &a, dev, dev, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  EXPECT(fmha_cache_attention(NULL, 1, 16, 1.f, dev, 0, dev, dev, dev, 0, dev, dev, 1 << 16, NULL), FMHA_ERR_INVALID_ARG);
  EXPECT(fmha_cache_attention(&c, 1, 1 << 20, 1.f, dev, 0, dev, dev, dev, 0, dev, dev, 64, NULL), FMHA_ERR_WORKSPACE);
  c.max_pages = 0x7fffffff;
  EXPECT(fmha_cache_attention(&c, 1, 16, 1.f, dev, 0, dev, dev, dev, 0, dev, dev, 1 << 16, NULL), FMHA_ERR_INVALID_ARG);
  c.max_pages = 1 << 26;
  EXPECT(fmha_cache_attention(&c, 16, 0, 1.f, dev, 0, dev, dev, dev, 0, dev, NULL, 0, NULL), FMHA_ERR_WORKSPACE);
  c.batch = 0x7fffffff, c.kv_heads = 65536;
  fmha_cache_attention_workspace_size(0x7fffffff, 65536, 65536, 128, 0x7fffffff);
  EXPECT(fmha_cache_append(&c, &a, dev, dev, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  /* causal attention */
  int32_t* cu = malloc(sizeof(int32_t) * 4);
  cu[0] = 0, cu[1] = 5, cu[2] = 5, cu[3] = 12;
  fmha_causal_params_t p;
  memset(&p, 0, sizeof(p));
  p.batch = 3, p.total_tokens = 20, p.heads = 4, p.kv_heads = 2, p.head_dim = 128, p.scale = 0.1f, p.cu_seqlens = dev, p.cu_seqlens_host = cu;
  p.workspace = dev, p.workspace_bytes = 16;
  EXPECT(fmha_causal_fwd(&p, dev, dev, dev, dev, dev, NULL), FMHA_ERR_WORKSPACE);
  p.max_seqlen = 6;
  EXPECT(fmha_causal_fwd(&p, dev, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  p.max_seqlen = 0, cu[2] = 3;
  EXPECT(fmha_causal_bwd(&p, dev, dev, dev, dev, dev, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  cu[2] = 5, p.total_tokens = 11;
  EXPECT(fmha_causal_bwd(&p, dev, dev, dev, dev, dev, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  p.total_tokens = 20, p.workspace_bytes = 1 << 16;
  EXPECT(fmha_causal_fwd(&p, dev, NULL, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  p.cu_seqlens_host = NULL, p.batch = p.total_tokens = 0x7fffffff, p.heads = p.kv_heads = 65536;
  EXPECT(fmha_causal_fwd(&p, dev, dev, dev, dev, dev, NULL), FMHA_ERR_INVALID_ARG);
  for (int32_t b = 0; b <= 1000000; b = b * 10 + 1)
    for (int32_t t = 0; t <= 100000000; t = t * 10 + 7)
      for (int32_t need = 0; need < 2; need++)
        if (!fmha_causal_workspace_size(b, t, 64, 8, 128, need)) return 1;
  fmha_causal_workspace_size(0x7fffffff, 0x7fffffff, 65536, 65536, 128, 1);
  free(cu);
  free(dev);
  puts("decoder entry points under sanitizers: ok");
  return 0;
}
