// Attention of new rows over a paged cache of their own type: the kernels of paged_attn.h.
#include "paged_attn.h"

using namespace spec;

extern "C" int spec_paged_attention_workspace_bytes(const spec_paged_cache *cache, const spec_paged_batch *batch, int32_t n_q_heads,
                                                    size_t *bytes) {
  const char *who = "spec_paged_attention_workspace_bytes";
  AttendArgs a{};
  Shape s;
  if (!bytes) return fail_noctx(SPEC_ERR_INVALID_ARG, "%s: bytes is null", who);
  int rc = paged_args(who, cache, batch, &a.p);
  if (!rc) rc = attend_check(who, cache, batch, n_q_heads, 0, a, s);  // without a window: the largest need
  if (rc) return rc;
  *bytes = attend_bytes(cache, s);
  return SPEC_OK;
}

extern "C" int spec_paged_attention(void *hip_stream, const spec_paged_cache *cache, const spec_paged_batch *batch, int32_t n_q_heads,
                                    const void *d_q, int64_t q_stride, float scale, int32_t window, void *d_workspace,
                                    size_t workspace_bytes, void *d_out, int64_t out_stride) {
  const char *who = "spec_paged_attention";
  AttendArgs a{};
  Shape s;
  bool nothing;
  int rc = paged_args(who, cache, batch, &a.p);
  if (!rc)
    rc = attend_prepare(who, cache, batch, n_q_heads, d_q, q_stride, scale, window, d_workspace, workspace_bytes, d_out,
                        out_stride, a, s, nothing);
  if (rc || nothing) return rc;
  if (s.qt == 16) {
    const hipError_t e = allow_chunk_lds<bf16_t, f16_t>();
    if (e != hipSuccess) return fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
  }
  SPEC_DISPATCH_DTYPE(cache->dtype, T, { attend_dispatch<T, T>(cache->head_dim, a, s, (hipStream_t)hip_stream); });
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPEC_OK : fail_noctx(SPEC_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}
