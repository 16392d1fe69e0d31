// basp_api_span.cpp -- the extern "C" surface of attention over spans.  As in
// basp_api.cpp every argument check runs on the host before the first HIP call,
// and nothing here allocates, frees or synchronises.
#include <initializer_list>

#include "basp_api_checks.hpp"
#include "basp_span.hpp"

namespace {

int check_shape(int b, int S, int n_q, int n_k, int d) {
  if (b < 0 || S < 0 || n_q < 1 || n_k < 1 || d < 1 || n_q % n_k != 0) return BASP_ERR_SHAPE;
  if (!head_dim(d)) return BASP_ERR_UNSUPPORTED;
  if ((uint64_t)b * (uint64_t)S == 0) return BASP_OK;
  // the kernels' counts of rows padded to 64 (a launch's threads, 16 a row, are a
  // 32-bit number), and sequences as a grid's second dimension
  const unsigned __int128 rows =
      (unsigned __int128)(unsigned)b * (((uint64_t)S + 63) / 64 * 64) * (unsigned)n_q;
  if (rows >= ((unsigned __int128)1 << 27) || b > 65535) return BASP_ERR_UNSUPPORTED;
  if (((uint64_t)S + 256) * (uint64_t)n_q * (uint64_t)d * 2 >= (1ull << 31))
    return BASP_ERR_UNSUPPORTED;
  return BASP_OK;
}

int check_rule(int S, int n_q, int n_k, int d, long long q_row, long long k_row, long long v_row,
               float scale, float cap) {
  if (q_row < (long long)n_q * d || k_row < (long long)n_k * d || v_row < (long long)n_k * d)
    return BASP_ERR_SHAPE;
  if (!(scale >= 0x1p-40f) || !(scale <= 0x1p40f) || !(cap >= 0.f) || !(cap <= 1024.f))
    return BASP_ERR_UNSUPPORTED;
  if (cap > 0.f && !isfinite(2.f * scale * basp::kSpanLog2e / cap)) return BASP_ERR_UNSUPPORTED;
  for (long long row : {q_row, k_row, v_row})  // 32-bit offsets inside a sequence
    if ((unsigned __int128)row * ((uint64_t)S + 256) * 2 >= (1ull << 31))
      return BASP_ERR_UNSUPPORTED;
  return BASP_OK;
}

int check_pointers(const void *q, const void *k, const void *v, const int *spans,
                   const float *slopes, const void *o, const float *lse, long long q_row,
                   long long k_row, long long v_row) {
  if (!q || !k || !v || !o || !lse) return BASP_ERR_NULL;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) ||
      !aligned(lse, 4) || !aligned(spans, 8) || !aligned(slopes, 4) || q_row % 8 != 0 ||
      k_row % 8 != 0 || v_row % 8 != 0)
    return BASP_ERR_ALIGN;
  return BASP_OK;
}

basp::SpanArgs span_args(const void *q, const void *k, const void *v, const int *spans,
                         const float *slopes, int b, int S, int n_q, int n_k, int d,
                         long long q_row, long long k_row, long long v_row, float scale,
                         float cap) {
  basp::SpanArgs a{};
  a.q = {static_cast<const uint16_t *>(q), (uint32_t)q_row};
  a.k = {static_cast<const uint16_t *>(k), (uint32_t)k_row};
  a.v = {static_cast<const uint16_t *>(v), (uint32_t)v_row};
  a.spans = spans;
  a.slopes = slopes;
  a.b = b, a.S = S, a.Hl = n_q, a.Hkl = n_k, a.d = d;
  a.scale = scale;
  a.cap = cap;
  return a;
}

}  // namespace

extern "C" {

int basp_attn_span_fwd(const void *q, const void *k, const void *v, const int *spans,
                       const float *slopes, void *o, float *lse, int b, int S, int n_q, int n_k,
                       int d, long long q_row, long long k_row, long long v_row, float scale,
                       float cap, void *stream) {
  int rc = check_shape(b, S, n_q, n_k, d);
  if (!rc) rc = check_rule(S, n_q, n_k, d, q_row, k_row, v_row, scale, cap);
  if (rc) return rc;
  if ((uint64_t)b * (uint64_t)S == 0) return BASP_OK;  // empty: no pointer is inspected
  rc = check_pointers(q, k, v, spans, slopes, o, lse, q_row, k_row, v_row);
  if (rc) return rc;
  (void)hipGetLastError();
  return hip_status(basp::launch_span_fwd(
      span_args(q, k, v, spans, slopes, b, S, n_q, n_k, d, q_row, k_row, v_row, scale, cap),
      static_cast<uint16_t *>(o), lse, (hipStream_t)stream));
}

size_t basp_attn_span_bwd_workspace_bytes(int b, int S, int n_q, int n_k, int d) {
  if (b < 1 || S < 1 || check_shape(b, S, n_q, n_k, d) != BASP_OK) return 0;
  return basp::span_bwd_workspace_bytes(span_args(nullptr, nullptr, nullptr, nullptr, nullptr, b, S,
                                                  n_q, n_k, d, 0, 0, 0, 1.f, 0.f));
}

int basp_attn_span_bwd(const void *q, const void *k, const void *v, const int *spans,
                       const float *slopes, const void *o, const float *lse, const void *d_o,
                       void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes,
                       int b, int S, int n_q, int n_k, int d, long long q_row, long long k_row,
                       long long v_row, float scale, float cap, basp_dtype grad_dtype,
                       void *stream) {
  int rc = check_shape(b, S, n_q, n_k, d);
  if (!rc) rc = check_rule(S, n_q, n_k, d, q_row, k_row, v_row, scale, cap);
  if (rc) return rc;
  if (grad_dtype != BASP_BF16 && grad_dtype != BASP_F32) return BASP_ERR_UNSUPPORTED;
  if ((uint64_t)b * (uint64_t)S == 0) return BASP_OK;  // empty: no pointer is inspected
  if (!d_o || !dq || !dk || !dv) return BASP_ERR_NULL;
  rc = check_pointers(q, k, v, spans, slopes, o, lse, q_row, k_row, v_row);
  if (rc) return rc;
  if (!aligned(d_o, 16) || !aligned(dq, 16) || !aligned(dk, 16) || !aligned(dv, 16))
    return BASP_ERR_ALIGN;
  const basp::SpanArgs a = span_args(q, k, v, spans, slopes, b, S, n_q, n_k, d, q_row, k_row,
                                     v_row, scale, cap);
  if (!basp::span_bwd_fits(a)) return BASP_ERR_UNSUPPORTED;
  if (workspace_bytes < basp::span_bwd_workspace_bytes(a)) return BASP_ERR_WORKSPACE;
  if (!workspace) return BASP_ERR_NULL;
  if (!aligned(workspace, 16)) return BASP_ERR_ALIGN;
  (void)hipGetLastError();
  return hip_status(basp::launch_span_bwd(a, static_cast<const uint16_t *>(o), lse,
                                          static_cast<const uint16_t *>(d_o), dq, dk, dv,
                                          grad_dtype == BASP_BF16, workspace,
                                          (hipStream_t)stream));
}

}  // extern "C"
