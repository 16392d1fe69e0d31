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

// ------------------------------------------------ how the backward is cut
constexpr int kSpanThreads = 512;   // of a workgroup of either pass
constexpr int kSpanStep = 64;       // rows of a step of the key pass
constexpr int kSpanHullBytes = 16;  // of the hull of 32 rows' spans
constexpr int kSpanPlanes = 4;      // numbers kept of a row and head, and of a row, with slopes

// Steps of a chunk at most: a sixteenth of the longest sequence (a row of d elements takes
// 2 d of its 2^31 bytes), rounded up to whole key tiles.  A unit lists them in LDS.
constexpr int span_max_steps(int d) { return (1 << 20) / d + 2; }

inline AttnShape span_shape(const SpanArgs &s, size_t workspace_bytes) {
  AttnShape x{s.b, s.S, s.Hl, s.Hkl, s.d, s.scale};
  x.workspace_bytes = workspace_bytes;
  return x;
}

// How the key pass is cut, and where things lie in the workspace.
struct SpanCut {
  int chunk_rows, nchunks, nsplits, ktiles, Sp;
  size_t rows, hulls, touched, parts, bytes;  // byte offsets, aux at 0
};

inline SpanCut span_cut(const SpanArgs &s) {
  auto align256 = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const BwdChunks ck = bwd_chunks(span_shape(s, (size_t)-1));
  SpanCut c;
  c.chunk_rows = ck.rows;
  c.nchunks = (s.S + c.chunk_rows - 1) / c.chunk_rows;
  c.nsplits = ck.splits;
  c.ktiles = (s.S + kKvKeys - 1) / kKvKeys;
  c.Sp = bwd_plane_rows(s.S);
  c.rows = align256((size_t)s.b * s.Hl * c.Sp * kSpanPlanes * sizeof(float));
  c.hulls = align256(c.rows + (size_t)s.b * c.Sp * kSpanPlanes * sizeof(int));
  c.touched = align256(c.hulls + (size_t)s.b * c.Sp / 32 * kSpanHullBytes);
  const size_t slots = (size_t)c.nchunks * c.nsplits;
  c.parts = align256(c.touched + slots * s.b * s.Hkl * c.ktiles * sizeof(int));
  c.bytes = c.parts;
  if (slots > 1) c.bytes += 2 * slots * s.b * s.S * s.Hkl * s.d * sizeof(float);
  return c;
}

// Row groups of the dQ pass: the causal backward's rule, but with spans 128 rows a
// workgroup up to 96K query rows: documents make workgroups of very different
// lengths, and twice as many of half the length even out better; one document wants the
// larger ones.  The host does not see which it is, and the sides do not cross at one
// size.  us with 128 and 256 rows (8 heads on 2 of 128, 7 on 1 at 79K; two draws of documents):
//   rows   one document  of S / 8             of 1200              of 300
//   42K    247, 239      165 164, 190 190     200 201, 208 222     123 125, 118 136
//   64K    487, 468      235 232, 323 314     268 267, 372 369     126 126, 195 200
//   79K    446, 421      289 293, 358 361     376 375, 383 387     199 200, 282 282
//   96K    985, 985      263 264, 432 417     226 243, 331 343     150 172, 170 209
//   128K   1686, 1652    391 388, 683 669     278 287, 406 428     196 185, 214 223
//   192K   3708, 3753    748 928, 1378 1477   459 560, 618 807     264 311, 308 356
inline int span_row_groups(const SpanArgs &s) {
  const int R = dq_row_groups(span_shape(s, (size_t)-1));
  return R == 8 && s.spans && (long long)s.b * s.Hl * s.S <= 98304 ? 4 : R;
}
inline long long span_dq_blocks(const SpanArgs &s) {
  const int rows = 32 * span_row_groups(s);
  return (long long)((s.S + rows - 1) / rows) * s.b * s.Hl;
}

// Workgroups of the key pass: (key tile, row chunk) pairs with rows at or after the
// keys first, then, with spans, those of rows before the keys.
inline long long span_key_blocks(const SpanArgs &s, const SpanCut &ck) {
  const long long pairs = kv_units(ck.nchunks, ck.chunk_rows / kKvKeys) +
                          (s.spans ? (long long)ck.nchunks * ck.ktiles : 0);
  return pairs * ck.nsplits * s.b * s.Hkl;
}

// Planes of -LSE (with slopes two) and -D, the rows' spans and hulls, which units of the key pass saw
// anything, and their partial sums of dK and dV.
inline size_t span_bwd_workspace_bytes(const SpanArgs &s) { return span_cut(s).bytes; }

// Its workgroups in one launch, and a unit's steps in LDS.
inline bool span_bwd_fits(const SpanArgs &s) {
  const SpanCut ck = span_cut(s);
  return (span_dq_blocks(s) + span_key_blocks(s, ck)) * kSpanThreads <= 0xFFFFFFFFll &&
         ck.chunk_rows <= span_max_steps(s.d) * kSpanStep;
}

hipError_t launch_span_bwd(const SpanArgs &s, const uint16_t *o, const float *lse,
                           const uint16_t *d_o, void *dq, void *dk, void *dv, bool grad_bf16,
                           void *workspace, hipStream_t stream);

hipError_t launch_span_fwd(const SpanArgs &a, uint16_t *o, float *lse, hipStream_t stream);

}  // namespace basp
