// basp_ops.hpp -- host-side launch interfaces of the operators around
// attention: norm and rotation of Q and K, the paged key-value cache, and
// attention of one token over it.  Shapes arrive here already validated.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "basp_internal.hpp"

namespace basp {

// ------------------------------------------------- norm and rotation of Q, K
// One of the two tensors: b*S tokens of n heads.
struct NormSide {
  const void *x;     // [tokens, n, d], tokens x_row elements apart
  const void *dy;    // backward: gradient of y, contiguous
  void *y;           // forward: output; backward: gradient of x, contiguous
  const float *w;    // [d] or NULL
  float *dw;         // backward, with w: [d]
  uint32_t rows;     // tokens * n
  FastDiv by_n;      // division by n
  uint32_t n;
  uint32_t units, chunks;  // forward: (token, chunk of heads), chunks per token
  FastDiv by_chunks;
  long long x_row, y_row;
};

struct NormArgs {
  NormSide side[2];  // Q, K
  const float *cos, *sin;
  const int *positions;
  FastDiv by_S;
  uint32_t S;
  int rot, table_rows, pos0;
  float eps;
};

hipError_t launch_norm_rope(NormArgs a, int d, bool interleaved, bool f32, hipStream_t stream);

// Workgroups of the backward for a tensor of `rows` rows of d elements; each
// writes one partial sum of dw.
int norm_bwd_blocks(uint32_t rows, int d);
// `f32`, `grad_f32`: types of x and of the gradients.  partials:
// (norm_bwd_blocks of Q + of K) * d floats.
hipError_t launch_norm_rope_bwd(const NormArgs &a, float *partials, int d, bool interleaved,
                                bool f32, bool grad_f32, hipStream_t stream);

// ----------------------------------------------------------- key-value cache
struct CacheShape {
  int b, n_k, d;
  int page_log2, n_pages, max_pages;
  bool e4m3;
};

struct CacheArgs {
  CacheShape s;
  void *pages[2];           // K, V
  unsigned char *scales[2]; // NULL unless e4m3
  const int *table;
  const int *start, *count; // either may be NULL (0, T)
  void *x[2];               // K, V rows: read by the write, written by the read
  long long x_row[2];       // elements between tokens
  int T;
  uint32_t rows;            // b * T * n_k
  FastDiv by_n, by_T;
};

hipError_t launch_kv_write(const CacheArgs &a, hipStream_t stream);
hipError_t launch_kv_read(const CacheArgs &a, hipStream_t stream);

// ------------------------------------------------ attention of one new token
struct DecodeArgs {
  CacheShape s;
  const void *q;
  long long q_row;
  const void *k_pages, *v_pages;
  const unsigned char *k_scales, *v_scales;
  const int *table, *lens;
  void *o;
  float *lse;
  int n_q, max_len;
  float scale;
  void *workspace;  // NULL where no head is shared by two workgroups
};

// How a call is cut.  A workgroup serves up to 16 query heads of a kv head at
// once, 32 where a kv head has more than 16.
constexpr int kDecodeUnit = 128;  // keys of a unit

// For each head, as dealt out, or workgroup that may leave partial results: where
// they lie.
struct DecodeOpen {
  int row0, heads, count, first;
};

struct DecodeCut {
  int rows;        // query heads of a workgroup: 16 or 32
  int row_groups;  // workgroups' worth of query heads per kv head
  int groups;      // workgroups
  int opens;       // DecodeOpen descriptors: the smaller of heads and workgroups
  size_t bytes;    // workspace; 0 where no head is shared by two workgroups
};

// Workgroups: three per CU at most (two of 32 rows).  One per CU alone has enough
// bytes in flight to fill the memory; three let more of them start on a short call
// (8 ragged sequences of up to 8K tokens, 8 heads on 2: 14.9 us against 16.1 with
// two), four leave a long sequence in more parts to join (one of 128K in 8 bits:
// 16.5 us with three, 19.5 with four).
inline DecodeCut decode_cut(int b, int n_q, int n_k, int d, int max_len) {
  DecodeCut c;
  const int rep = n_q / n_k;
  c.rows = rep > 16 ? 32 : 16;
  c.row_groups = (rep + c.rows - 1) / c.rows;
  const long long most = 256 * (c.rows == 16 ? 3 : 2);
  const long long heads = (long long)b * n_k * c.row_groups;
  const long long units = heads * (((long long)max_len + kDecodeUnit - 1) / kDecodeUnit);
  c.groups = (int)(units < most ? units : most);
  c.opens = (int)(heads < c.groups ? heads : c.groups);
  // per workgroup its first and its last head's rows: (m, l) and O
  c.bytes = max_len <= kDecodeUnit
                ? 0
                : c.opens * sizeof(DecodeOpen) +
                      (size_t)c.groups * 2 * c.rows * (2 + d) * sizeof(float);
  return c;
}

hipError_t launch_attn_decode(const DecodeArgs &a, hipStream_t stream);

}  // namespace basp
