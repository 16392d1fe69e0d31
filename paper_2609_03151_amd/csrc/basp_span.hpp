// basp_span.hpp -- attention whose scores are capped, biased by distance and
// masked by spans: host-side launch interfaces, and the score rule that the
// kernels share.  Shapes arrive here already validated.
//
//   s_ij = scale q_i.k_j
//   u_ij = cap tanh(s_ij / cap) - slope_h |i - j|     (u = s without a cap)
//   P_ij = exp(u_ij) / sum over lo_i <= j < hi_i, 0 elsewhere
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "basp_internal.hpp"

namespace basp {

constexpr float kSpanLog2e = 1.4426950408889634f;
constexpr float kSpanLn2 = 0.69314718055994531f;

// Up to this cap the exponents' reference needs no running maximum: a capped
// score is at most cap and at least -cap, so with the largest bias of the row
// as its reference P lies in 2^(+-92.4), and sums of P over 2^24 keys in fp32's range.
// Their products with V need not: rows whose sum is far from 1 are done again against
// their maximum where it matters (basp_span_fwd.hip).
constexpr float kSpanFixedCap = 64.f;

// A tensor [b, S, n, d] whose tokens lie row_elems elements apart.
struct SpanRows {
  const uint16_t *p;
  uint32_t row_elems;
};

struct SpanArgs {
  SpanRows q, k, v;
  const int *spans;     // [b, S, 2], or NULL: causal
  const float *slopes;  // [Hl], or NULL
  int b, S, Hl, Hkl, d;
  float scale, cap;     // cap 0: none
};

// The backward's: planes of -LSE and -D, the rows' hulls, which units of the key
// pass saw anything, and their partial sums of dK and dV.
size_t span_bwd_workspace_bytes(const SpanArgs &s);
bool span_bwd_fits(const SpanArgs &s);  // its workgroups in one launch, a unit's steps in LDS
hipError_t launch_span_bwd(const SpanArgs &s, const uint16_t *o, const float *lse,
                           const uint16_t *d_o, void *dq, void *dk, void *dv, bool grad_bf16,
                           void *workspace, hipStream_t stream);

hipError_t launch_span_fwd(const SpanArgs &a, uint16_t *o, float *lse, hipStream_t stream);

}  // namespace basp
