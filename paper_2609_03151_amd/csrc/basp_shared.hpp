// basp_shared.hpp -- host-side launch interface of attention of one new token for
// sequences that share prefixes.  Shapes arrive here already validated.
#pragma once

#include "basp_ops.hpp"

namespace basp {

struct SharedArgs {
  DecodeArgs d;             // as basp_attn_decode
  const int *groups;        // [n_groups + 1]
  const int *prefix_lens;   // [n_groups]
  const float *slopes;      // [n_q] or NULL
  int n_groups;
  float cap;                // 0: none
};

// Rows (a query head of a sequence that shares) that a workgroup of the prefix pass
// takes, and the keys of its tiles.
constexpr int kSharedRows = 64, kSharedTile = 64;

// How a call is cut, and where things lie in the workspace (byte offsets).
struct SharedCut {
  int chunks;      // of kSharedRows rows: at most, in all groups
  int splits;      // of a prefix's keys
  int prefix_blocks;
  DecodeCut own;   // of the sequences' own keys
  int vheads;      // kv head x group of own.rows query heads, of a sequence
  size_t ints, records, open, own_ml, own_o, row_ml, row_o, part_ml, part_o, bytes;
};

inline SharedCut shared_cut(int b, int n_q, int n_k, int d, int max_len, int n_groups) {
  SharedCut c;
  const long long rep = n_q / n_k;
  // a group's rows in whole chunks; no group that shares has fewer than two sequences
  const long long sharing = n_groups < b / 2 ? n_groups : b / 2;
  c.chunks = (int)(sharing == 0 ? 0 : sharing + b * rep / kSharedRows);
  // Enough workgroups for two per CU, of two tiles or more.
  const long long per_split = (long long)c.chunks * n_k;
  long long splits = per_split == 0 ? 0 : (512 + per_split - 1) / per_split;
  const long long most = ((long long)max_len + 2 * kSharedTile - 1) / (2 * kSharedTile);
  if (splits > most) splits = most;
  if (splits > 8) splits = splits / 8 * 8;
  c.splits = (int)splits;
  c.prefix_blocks = (int)(per_split * splits);
  c.own = decode_cut(b, n_q, n_k, d, max_len);
  c.vheads = n_k * c.own.row_groups;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t row = (size_t)d * sizeof(float), ml = 2 * sizeof(float);
  // total chunks; then start, row, members, units so far [b + 1]; of a group rows and chunks
  c.ints = 0;
  c.records = up((4 * (size_t)b + 2 + 2 * (size_t)n_groups) * sizeof(int));
  c.open = up(c.records + (size_t)c.chunks * 4 * sizeof(int));
  c.own_ml = up(c.open + (size_t)b * c.vheads * sizeof(DecodeOpen));
  c.own_o = up(c.own_ml + (size_t)c.own.groups * 2 * c.own.rows * ml);
  c.row_ml = up(c.own_o + (size_t)c.own.groups * 2 * c.own.rows * row);
  c.row_o = up(c.row_ml + (sharing ? (size_t)b * n_q * ml : 0));
  c.part_ml = up(c.row_o + (sharing ? (size_t)b * n_q * row : 0));
  c.part_o = up(c.part_ml + (size_t)c.prefix_blocks * kSharedRows * ml);
  c.bytes = c.part_o + (size_t)c.prefix_blocks * kSharedRows * row;
  return c;
}

hipError_t launch_attn_decode_shared(const SharedArgs &a, hipStream_t stream);

}  // namespace basp
