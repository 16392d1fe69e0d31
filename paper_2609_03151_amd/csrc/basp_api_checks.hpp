// basp_api_checks.hpp -- argument checks that several files of the C ABI layer share.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/basp.h"
#include "basp_ops.hpp"

namespace {

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int hip_status(hipError_t e) { return e == hipSuccess ? BASP_OK : BASP_ERR_HIP; }

inline bool head_dim(int d) { return d == 64 || d == 80 || d == 96 || d == 128; }

// Shape rules of the cache's three calls.
inline int check_cache(int b, int n_k, int d, int page, int n_pages, int max_pages, int cache_dtype) {
  if (b < 0 || n_k < 1 || d < 1 || page < 1 || n_pages < 1 || max_pages < 1) return BASP_ERR_SHAPE;
  if (!head_dim(d)) return BASP_ERR_UNSUPPORTED;
  if (page != 16 && page != 32 && page != 64 && page != 128 && page != 256)
    return BASP_ERR_UNSUPPORTED;
  if (cache_dtype != BASP_BF16 && cache_dtype != BASP_E4M3) return BASP_ERR_UNSUPPORTED;
  if ((uint64_t)n_pages * (uint64_t)n_k >= (1ull << 31)) return BASP_ERR_UNSUPPORTED;
  return BASP_OK;
}

inline int check_pages(const void *k_pages, const void *v_pages, const unsigned char *k_scales,
                const unsigned char *v_scales, const int *table, int cache_dtype) {
  if (!k_pages || !v_pages || !table) return BASP_ERR_NULL;
  const bool e4m3 = cache_dtype == BASP_E4M3;
  if (e4m3 != (k_scales != nullptr) || e4m3 != (v_scales != nullptr)) return BASP_ERR_NULL;
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(k_scales, 4) ||
      !aligned(v_scales, 4) || !aligned(table, 4))
    return BASP_ERR_ALIGN;
  return BASP_OK;
}

inline basp::CacheShape cache_shape(int b, int n_k, int d, int page, int n_pages, int max_pages,
                             int cache_dtype) {
  basp::CacheShape s{b, n_k, d, 0, n_pages, max_pages, cache_dtype == BASP_E4M3};
  while ((1 << s.page_log2) < page) ++s.page_log2;
  return s;
}

// Shape rules of basp_attn_decode.  The kernel counts units of 128 keys or more
// per (sequence, head), what it deals out by adding the workgroups less one, and keys
// up to a unit past a length, in 32 bits.
inline int check_decode(int b, int n_q, int n_k, int d, int max_len) {
  if (b < 0 || n_q < 1 || n_k < 1 || d < 1 || max_len < 1 || n_q % n_k != 0) return BASP_ERR_SHAPE;
  if (!head_dim(d) || (uint64_t)b * (uint64_t)n_q >= (1ull << 22) || max_len > (1 << 30))
    return BASP_ERR_UNSUPPORTED;
  if ((uint64_t)b * (uint64_t)n_q * (((uint64_t)max_len + 127) / 128) >= (1ull << 30))
    return BASP_ERR_UNSUPPORTED;
  return BASP_OK;
}

inline basp::DecodeArgs decode_args(const void *q, const void *k_pages, const void *v_pages,
                             const unsigned char *k_scales, const unsigned char *v_scales,
                             const int *block_table, const int *lens, void *o, float *lse, int b,
                             int n_q, int n_k, int d, int page, int n_pages, int max_pages,
                             int max_len, long long q_row, float scale, int cache_dtype) {
  basp::DecodeArgs a{};
  a.s = cache_shape(b, n_k, d, page, n_pages, max_pages, cache_dtype);
  a.q = q;
  a.q_row = q_row;
  a.k_pages = k_pages, a.v_pages = v_pages;
  a.k_scales = k_scales, a.v_scales = v_scales;
  a.table = block_table;
  a.lens = lens;
  a.o = o;
  a.lse = lse;
  a.n_q = n_q;
  a.max_len = max_len;
  a.scale = scale;
  return a;
}

}  // namespace
