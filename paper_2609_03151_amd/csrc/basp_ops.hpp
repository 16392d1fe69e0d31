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

size_t decode_workspace_bytes(int b, int n_q, int n_k, int d, int max_len);

hipError_t launch_attn_decode(const DecodeArgs &a, hipStream_t stream);

}  // namespace basp
