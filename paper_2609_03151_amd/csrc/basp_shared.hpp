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

// Keys of a tile of the prefix pass.
constexpr int kSharedTile = 64;

// Up to so many sequences and groups every workgroup plans by itself, in LDS; past them a
// kernel of its own does it first.
constexpr int kLocalSeqs = 512, kLocalGroups = 128;

// How a call is cut, and where things lie in the workspace (byte offsets).
struct SharedCut {
  bool local;      // no plan kernel
  int rows;        // (a query head of a sequence that shares) of a prefix workgroup: 64 or 128
  int chunks;      // of so many rows: at most, in all groups
  int splits;      // of a prefix's keys
  int prefix_blocks;
  DecodeCut own;   // of the sequences' own keys
  int vheads;      // kv head x group of own.rows query heads, of a sequence
  size_t ints, records, open, own_ml, own_o, row_ml, row_o, part_ml, part_o, bytes;
};

inline SharedCut shared_cut(int b, int n_q, int n_k, int d, int max_len, int n_groups) {
  SharedCut c;
  c.local = b <= kLocalSeqs && n_groups <= kLocalGroups;
  const long long rep = n_q / n_k;
  // a group's rows in whole chunks; no group that shares has fewer than two sequences
  const long long sharing = n_groups < b / 2 ? n_groups : b / 2;
  // A tile's way through LDS is paid once for 64 or 128 rows; a workgroup leaves O of all of
  // them.  us with 64 and with 128, prompts of 16K, 8 heads on 2 of 128: 64 rows of a kv
  // head 20.6, 20.7; 128 rows 21.7, 25.9; 192 rows 25.2, 24.9; 256 rows 26.4, 25.9; 512 rows 37.2,
  // 33.1; four prompts of 8K and 256 rows each 35.6, 28.8, in 8 bits and 64 rows 23.3, 24.7.
  c.rows = b * rep > 192 * sharing ? 128 : 64;
  c.chunks = (int)((b * rep + sharing * (c.rows - 1)) / c.rows);
  if (sharing == 0) c.chunks = 0;
  const long long per_split = (long long)c.chunks * n_k;
  // A workgroup of either kind per CU, which has room for two: more for the prefix leave
  // more partial results, fewer leave CUs without one.  us with 128, 192, 256, 384: the 128
  // rows above 23.8, 22.7, 21.7, 29.6; 256 rows 30.2, 27.4, 25.9, 35.0; 512 rows on one prompt
  // of 32K 45.3, 37.3, 33.4, 42.0; four prompts of 8K and 64 rows each 33.5, 33.5, 25.5, 27.5.
  // The cut goes by what the host knows, not by the prefixes' lengths, and is the same for
  // all: one long prefix among many short ones is cut into few parts.
  long long splits = per_split == 0 ? 0 : (256 + per_split - 1) / per_split;
  const long long most = ((long long)max_len + 2 * kSharedTile - 1) / (2 * kSharedTile);
  if (splits > most) splits = most;
  if (splits > 8) splits = splits / 8 * 8;
  c.splits = (int)splits;
  c.prefix_blocks = (int)(per_split * splits);
  c.own = decode_cut(b, n_q, n_k, d, max_len);
  if (c.own.groups > (sharing ? 256 : 512)) c.own.groups = sharing ? 256 : 512;
  c.vheads = n_k * c.own.row_groups;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t row = (size_t)d * sizeof(float), ml = 2 * sizeof(float);
  // total chunks; then start, row, member, units [b + 1]; of a group members, first, chunk
  c.ints = 0;
  c.records = up((4 * (size_t)b + 2 + 3 * (size_t)n_groups) * sizeof(int));
  c.open = up(c.records + (size_t)c.chunks * 4 * sizeof(int));
  c.own_ml = up(c.open + (size_t)b * c.vheads * sizeof(DecodeOpen));
  c.own_o = up(c.own_ml + (size_t)c.own.groups * 2 * c.own.rows * ml);
  c.row_ml = up(c.own_o + (size_t)c.own.groups * 2 * c.own.rows * row);
  c.row_o = up(c.row_ml + (sharing ? (size_t)b * n_q * ml : 0));
  c.part_ml = up(c.row_o + (sharing ? (size_t)b * n_q * row : 0));
  c.part_o = up(c.part_ml + (size_t)c.prefix_blocks * c.rows * ml);
  c.bytes = c.part_o + (size_t)c.prefix_blocks * c.rows * row;
  return c;
}

hipError_t launch_attn_decode_shared(const SharedArgs &a, hipStream_t stream);

}  // namespace basp
