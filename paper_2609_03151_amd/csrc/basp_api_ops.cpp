// basp_api_ops.cpp -- the extern "C" surface of the operators around
// attention: norm and rotation of Q and K, the paged key-value cache, and
// attention of one token over it.  As in basp_api.cpp every argument check
// runs on the host before the first HIP call, and nothing here allocates,
// frees or synchronises.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/basp.h"
#include "basp_api_checks.hpp"

namespace {

// b*S*n rows, 0 where there are 2^bits or more.
uint64_t rows_of(int b, int S, int n, int bits) {
  const unsigned __int128 r = (unsigned __int128)(unsigned)b * (unsigned)S * (unsigned)n;
  return r < ((unsigned __int128)1 << bits) ? (uint64_t)r : 0;
}

// Shape rules of norm and rotation, forward and backward; pointers are looked
// at by the callers.  A launch's threads are a 32-bit count, 16 of them four heads
// of a token in the forward.
int check_norm(int b, int S, int n_q, int n_k, int d, int rot, int table_rows, long long q_row,
               long long k_row, float eps, int pos0, bool positions, int dtype, int grad_dtype) {
  if (b < 0 || S < 0 || n_q < 1 || n_k < 1 || d < 1) return BASP_ERR_SHAPE;
  if (rot < 0 || rot > d || rot % 8 != 0 || table_rows < 0 || pos0 < 0) return BASP_ERR_SHAPE;
  if (!head_dim(d)) return BASP_ERR_UNSUPPORTED;
  for (int t : {dtype, grad_dtype})
    if (t != BASP_BF16 && t != BASP_F32) return BASP_ERR_UNSUPPORTED;
  if (!(eps >= 0.f) || !isfinite(eps)) return BASP_ERR_UNSUPPORTED;
  if ((uint64_t)b * (uint64_t)S != 0 &&
      (rows_of(b, S, n_q, 29) == 0 || rows_of(b, S, n_k, 29) == 0 ||
       rows_of(b, S, (n_q - 1) / 4 + (n_k - 1) / 4 + 2, 27) == 0))
    return BASP_ERR_UNSUPPORTED;
  if (q_row < (long long)n_q * d || k_row < (long long)n_k * d) return BASP_ERR_SHAPE;
  if (rot > 0 && !positions && (long long)pos0 + S > table_rows) return BASP_ERR_SHAPE;
  return BASP_OK;
}

// The arguments both directions share.
int check_norm_pointers(const float *qw, const float *kw, const float *cos, const float *sin,
                        const int *positions, int rot, long long q_row, long long k_row) {
  if (!qw != !kw || !cos != !sin || (rot > 0) != (cos != nullptr)) return BASP_ERR_NULL;
  if (!aligned(qw, 16) || !aligned(kw, 16) || !aligned(cos, 16) || !aligned(sin, 16) ||
      !aligned(positions, 4) || q_row % 4 != 0 || k_row % 4 != 0)
    return BASP_ERR_ALIGN;
  return BASP_OK;
}

basp::NormArgs norm_args(const void *q, const void *k, const float *qw, const float *kw,
                         const float *cos, const float *sin, const int *positions, int b, int S,
                         int n_q, int n_k, int rot, int table_rows, long long q_row,
                         long long k_row, float eps, int pos0) {
  basp::NormArgs a{};
  const int n[2] = {n_q, n_k};
  for (int i = 0; i < 2; ++i) {
    basp::NormSide &s = a.side[i];
    s.x = i ? k : q;
    s.w = i ? kw : qw;
    s.x_row = i ? k_row : q_row;
    s.n = (uint32_t)n[i];
    s.by_n = basp::FastDiv::make(s.n);
    s.rows = (uint32_t)((uint64_t)b * S * n[i]);
  }
  a.cos = cos;
  a.sin = sin;
  a.positions = positions;
  a.S = (uint32_t)S;
  a.by_S = basp::FastDiv::make(a.S);
  a.rot = rot;
  a.table_rows = table_rows;
  a.pos0 = rot > 0 ? pos0 : 0;  // else bounded by no table: pos0 + t may pass 2^31
  a.eps = eps;
  return a;
}

}  // namespace

extern "C" {

int basp_qk_norm_rope(const void *q, const void *k, void *qo, void *ko, const float *qw,
                      const float *kw, const float *cos, const float *sin, const int *positions,
                      int b, int S, int n_q, int n_k, int d, int rot, int table_rows,
                      long long q_row, long long k_row, long long qo_row, long long ko_row,
                      float eps, int pos0, int interleaved, basp_dtype dtype, void *stream) {
  int rc = check_norm(b, S, n_q, n_k, d, rot, table_rows, q_row, k_row, eps, pos0,
                      positions != nullptr, dtype, dtype);
  if (rc) return rc;
  if (qo_row < (long long)n_q * d || ko_row < (long long)n_k * d) return BASP_ERR_SHAPE;
  if ((uint64_t)b * (uint64_t)S == 0) return BASP_OK;  // empty: no pointer is inspected
  if (!q || !k || !qo || !ko) return BASP_ERR_NULL;
  rc = check_norm_pointers(qw, kw, cos, sin, positions, rot, q_row, k_row);
  if (rc) return rc;
  const uintptr_t unit = dtype == BASP_BF16 ? 8 : 16;
  if (!aligned(q, unit) || !aligned(k, unit) || !aligned(qo, unit) || !aligned(ko, unit) ||
      qo_row % 4 != 0 || ko_row % 4 != 0)
    return BASP_ERR_ALIGN;
  basp::NormArgs a = norm_args(q, k, qw, kw, cos, sin, positions, b, S, n_q, n_k, rot, table_rows,
                               q_row, k_row, eps, pos0);
  a.side[0].y = qo;
  a.side[1].y = ko;
  a.side[0].y_row = qo_row;
  a.side[1].y_row = ko_row;
  (void)hipGetLastError();
  return hip_status(basp::launch_norm_rope(a, d, interleaved != 0, dtype == BASP_F32,
                                           (hipStream_t)stream));
}

size_t basp_qk_norm_rope_bwd_workspace_bytes(int b, int S, int n_q, int n_k, int d) {
  if (b < 1 || S < 1 || n_q < 1 || n_k < 1 || !head_dim(d)) return 0;
  const uint64_t rq = rows_of(b, S, n_q, 29), rk = rows_of(b, S, n_k, 29);
  if (rq == 0 || rk == 0) return 0;
  return ((size_t)basp::norm_bwd_blocks((uint32_t)rq, d) +
          basp::norm_bwd_blocks((uint32_t)rk, d)) * d * sizeof(float);
}

int basp_qk_norm_rope_bwd(const void *q, const void *k, const void *dqo, const void *dko, void *dq,
                          void *dk, const float *qw, const float *kw, float *dqw, float *dkw,
                          const float *cos, const float *sin, const int *positions,
                          void *workspace, size_t workspace_bytes, int b, int S, int n_q, int n_k,
                          int d, int rot, int table_rows, long long q_row, long long k_row,
                          float eps, int pos0, int interleaved, basp_dtype dtype,
                          basp_dtype grad_dtype, void *stream) {
  int rc = check_norm(b, S, n_q, n_k, d, rot, table_rows, q_row, k_row, eps, pos0,
                      positions != nullptr, dtype, grad_dtype);
  if (rc) return rc;
  if ((uint64_t)b * (uint64_t)S == 0) return BASP_OK;  // empty: no pointer is inspected
  if (!dqo || !dko || !dq || !dk) return BASP_ERR_NULL;
  rc = check_norm_pointers(qw, kw, cos, sin, positions, rot, q_row, k_row);
  if (rc) return rc;
  const uintptr_t unit = dtype == BASP_BF16 ? 8 : 16, gunit = grad_dtype == BASP_BF16 ? 8 : 16;
  if (!aligned(dqo, gunit) || !aligned(dko, gunit) || !aligned(dq, gunit) || !aligned(dk, gunit))
    return BASP_ERR_ALIGN;
  if (qw) {
    if (!q || !k || !dqw || !dkw) return BASP_ERR_NULL;
    if (!aligned(q, unit) || !aligned(k, unit) || !aligned(dqw, 4) || !aligned(dkw, 4))
      return BASP_ERR_ALIGN;
    if (workspace_bytes < basp_qk_norm_rope_bwd_workspace_bytes(b, S, n_q, n_k, d))
      return BASP_ERR_WORKSPACE;
    if (!workspace) return BASP_ERR_NULL;
    if (!aligned(workspace, 16)) return BASP_ERR_ALIGN;
  }
  basp::NormArgs a = norm_args(q, k, qw, kw, cos, sin, positions, b, S, n_q, n_k, rot, table_rows,
                               q_row, k_row, eps, pos0);
  a.side[0].dy = dqo, a.side[0].y = dq, a.side[0].dw = dqw;
  a.side[1].dy = dko, a.side[1].y = dk, a.side[1].dw = dkw;
  (void)hipGetLastError();
  return hip_status(basp::launch_norm_rope_bwd(a, static_cast<float *>(workspace), d,
                                               interleaved != 0, dtype == BASP_F32,
                                               grad_dtype == BASP_F32, (hipStream_t)stream));
}

}  // extern "C"

namespace {

int run_cache(bool write, const void *k, const void *v, const void *k_pages, const void *v_pages,
              const unsigned char *k_scales, const unsigned char *v_scales, const int *table,
              const int *start, const int *count, int b, int T, int n_k, int d, int page,
              int n_pages, int max_pages, long long k_row, long long v_row, int cache_dtype,
              void *stream) {
  if (T < 0) return BASP_ERR_SHAPE;
  int rc = check_cache(b, n_k, d, page, n_pages, max_pages, cache_dtype);
  if (rc) return rc;
  if (k_row < (long long)n_k * d || v_row < (long long)n_k * d) return BASP_ERR_SHAPE;
  if ((uint64_t)b * (uint64_t)T == 0) return BASP_OK;  // empty: no pointer is inspected
  // A launch's threads are a 32-bit count, 16 of them a (token, head).
  const uint64_t rows = rows_of(b, T, n_k, 27);
  if (rows == 0) return BASP_ERR_UNSUPPORTED;
  if (!k || !v || (write && !start)) return BASP_ERR_NULL;
  rc = check_pages(k_pages, v_pages, k_scales, v_scales, table, cache_dtype);
  if (rc) return rc;
  if (!aligned(k, 16) || !aligned(v, 16) || k_row % 8 != 0 || v_row % 8 != 0 ||
      !aligned(start, 4) || !aligned(count, 4))
    return BASP_ERR_ALIGN;
  basp::CacheArgs a{};
  a.s = cache_shape(b, n_k, d, page, n_pages, max_pages, cache_dtype);
  a.pages[0] = const_cast<void *>(k_pages), a.pages[1] = const_cast<void *>(v_pages);
  a.scales[0] = const_cast<unsigned char *>(k_scales);
  a.scales[1] = const_cast<unsigned char *>(v_scales);
  a.table = table;
  a.start = start;
  a.count = count;
  a.x[0] = const_cast<void *>(k), a.x[1] = const_cast<void *>(v);
  a.x_row[0] = k_row, a.x_row[1] = v_row;
  a.T = T;
  a.rows = (uint32_t)rows;
  a.by_n = basp::FastDiv::make((uint32_t)n_k);
  a.by_T = basp::FastDiv::make((uint32_t)T);
  (void)hipGetLastError();
  return hip_status(write ? basp::launch_kv_write(a, (hipStream_t)stream)
                          : basp::launch_kv_read(a, (hipStream_t)stream));
}

}  // namespace

extern "C" {

int basp_kv_write(const void *k, const void *v, void *k_pages, void *v_pages,
                  unsigned char *k_scales, unsigned char *v_scales, const int *block_table,
                  const int *start, const int *count, int b, int T, int n_k, int d, int page,
                  int n_pages, int max_pages, long long k_row, long long v_row,
                  basp_dtype cache_dtype, void *stream) {
  return run_cache(true, k, v, k_pages, v_pages, k_scales, v_scales, block_table, start, count, b,
                   T, n_k, d, page, n_pages, max_pages, k_row, v_row, cache_dtype, stream);
}

int basp_kv_read(const void *k_pages, const void *v_pages, const unsigned char *k_scales,
                 const unsigned char *v_scales, const int *block_table, const int *start,
                 const int *count, void *k, void *v, int b, int T, int n_k, int d, int page,
                 int n_pages, int max_pages, basp_dtype cache_dtype, void *stream) {
  const long long row = (long long)n_k * d;
  return run_cache(false, k, v, k_pages, v_pages, k_scales, v_scales, block_table, start, count, b,
                   T, n_k, d, page, n_pages, max_pages, row, row, cache_dtype, stream);
}

size_t basp_attn_decode_workspace_bytes(int b, int n_q, int n_k, int d, int max_len) {
  if (b < 1 || check_decode(b, n_q, n_k, d, max_len) != BASP_OK) return 0;
  return basp::decode_cut(b, n_q, n_k, d, max_len).bytes;
}

int basp_attn_decode(const void *q, const void *k_pages, const void *v_pages,
                     const unsigned char *k_scales, const unsigned char *v_scales,
                     const int *block_table, const int *lens, void *o, float *lse, void *workspace,
                     size_t workspace_bytes, int b, int n_q, int n_k, int d, int page, int n_pages,
                     int max_pages, int max_len, long long q_row, float scale,
                     basp_dtype cache_dtype, void *stream) {
  int rc = check_cache(b, n_k, d, page, n_pages, max_pages, cache_dtype);
  if (!rc) rc = check_decode(b, n_q, n_k, d, max_len);
  if (rc) return rc;
  if (q_row < (long long)n_q * d) return BASP_ERR_SHAPE;
  if (!(scale > 0.f) || !isfinite(scale)) return BASP_ERR_UNSUPPORTED;
  if (b == 0) return BASP_OK;  // empty: no pointer is inspected
  if (!q || !o || !lens) return BASP_ERR_NULL;
  rc = check_pages(k_pages, v_pages, k_scales, v_scales, block_table, cache_dtype);
  if (rc) return rc;
  if (!aligned(q, 16) || !aligned(o, 16) || !aligned(lse, 4) || !aligned(lens, 4) || q_row % 8 != 0)
    return BASP_ERR_ALIGN;
  const size_t need = basp::decode_cut(b, n_q, n_k, d, max_len).bytes;
  if (workspace_bytes < need) return BASP_ERR_WORKSPACE;
  if (need > 0 && !workspace) return BASP_ERR_NULL;
  if (!aligned(workspace, 16)) return BASP_ERR_ALIGN;
  basp::DecodeArgs a = decode_args(q, k_pages, v_pages, k_scales, v_scales, block_table, lens, o, lse,
                                   b, n_q, n_k, d, page, n_pages, max_pages, max_len, q_row, scale,
                                   cache_dtype);
  a.workspace = need > 0 ? workspace : nullptr;
  (void)hipGetLastError();
  return hip_status(basp::launch_attn_decode(a, (hipStream_t)stream));
}

}  // extern "C"
