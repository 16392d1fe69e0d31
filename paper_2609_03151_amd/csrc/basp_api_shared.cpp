// basp_api_shared.cpp -- the extern "C" surface of attention of one new token for
// sequences that share prefixes.  As in basp_api.cpp every argument check runs on the
// host before the first HIP call, and nothing here allocates, frees or synchronises.
#include "basp_api_checks.hpp"
#include "basp_shared.hpp"

extern "C" {

size_t basp_attn_decode_shared_workspace_bytes(int b, int n_q, int n_k, int d, int max_len,
                                               int n_groups) {
  if (b < 1 || n_groups < 0 || check_decode(b, n_q, n_k, d, max_len) != BASP_OK) return 0;
  return basp::shared_cut(b, n_q, n_k, d, max_len, n_groups).bytes;
}

int basp_attn_decode_shared(const void *q, const void *k_pages, const void *v_pages,
                            const unsigned char *k_scales, const unsigned char *v_scales,
                            const int *block_table, const int *lens, const int *groups,
                            const int *prefix_lens, const float *slopes, void *o, float *lse,
                            void *workspace, size_t workspace_bytes, int b, int n_q, int n_k,
                            int d, int page, int n_pages, int max_pages, int max_len,
                            int n_groups, long long q_row, float scale, float cap,
                            basp_dtype cache_dtype, void *stream) {
  int rc = check_cache(b, n_k, d, page, n_pages, max_pages, cache_dtype);
  if (!rc) rc = check_decode(b, n_q, n_k, d, max_len);
  if (rc) return rc;
  if (q_row < (long long)n_q * d || n_groups < 0) return BASP_ERR_SHAPE;
  if (!(scale > 0.f) || !isfinite(scale) || !(cap >= 0.f) || !(cap <= 1024.f))
    return BASP_ERR_UNSUPPORTED;
  if (cap > 0.f && !isfinite(2.f * scale * 1.4426950408889634f / cap)) return BASP_ERR_UNSUPPORTED;
  if (n_groups >= 1 << 22) return BASP_ERR_UNSUPPORTED;
  if (b == 0) return BASP_OK;  // empty: no pointer is inspected
  if (!q || !o || !lens || (n_groups > 0 && (!groups || !prefix_lens))) return BASP_ERR_NULL;
  rc = check_pages(k_pages, v_pages, k_scales, v_scales, block_table, cache_dtype);
  if (rc) return rc;
  if (!aligned(q, 16) || !aligned(o, 16) || !aligned(lse, 4) || !aligned(lens, 4) ||
      !aligned(groups, 4) || !aligned(prefix_lens, 4) || !aligned(slopes, 4) || q_row % 8 != 0)
    return BASP_ERR_ALIGN;
  if (workspace_bytes < basp::shared_cut(b, n_q, n_k, d, max_len, n_groups).bytes)
    return BASP_ERR_WORKSPACE;
  if (!workspace) return BASP_ERR_NULL;
  if (!aligned(workspace, 16)) return BASP_ERR_ALIGN;
  basp::SharedArgs a{};
  a.d = decode_args(q, k_pages, v_pages, k_scales, v_scales, block_table, lens, o, lse, b, n_q, n_k,
                    d, page, n_pages, max_pages, max_len, q_row, scale, cache_dtype);
  a.d.workspace = workspace;
  a.groups = groups;
  a.prefix_lens = prefix_lens;
  a.slopes = slopes;
  a.n_groups = n_groups;
  a.cap = cap;
  (void)hipGetLastError();
  return hip_status(basp::launch_attn_decode_shared(a, (hipStream_t)stream));
}

}  // extern "C"
