// basp_shared.hip -- attention of one new token per sequence over a paged
// key-value cache, for sequences in groups that share a prefix; scores capped and
// biased by distance (basp_span.hpp) where the model has them.
//
// A group's sequences list the same pages for its prefix's tokens, so those keys are
// read once for all of them: the rows of the product are then (sequence, query head)
// pairs, many enough for the matrix cores' 32-row tiles.  Bound by HBM for the keys and
// values, each read once, up to some 200 rows a kv head, by the matrix cores (and
// with a cap the vector units) past that.  On MI355X, 32 sequences on one prompt of 16K
// tokens, 8 heads on 2 of 128: 21.7 us, 8 of them dependent loads, 11 tiles, 5 the join
// (its bytes alone take 5.5); read sequence by sequence the prompt would be 0.5 GB.
//
//   shared_plan   which sequences share, and where their rows go (past 512 sequences or 128
//                 groups; else each workgroup of the next kernel finds out by itself)
//   shared_main   prefix workgroups: 64 or 128 rows of a group and kv head times a
//                 split of the prefix's keys, as the causal forward's (S^T = K Q^T, O^T =
//                 V^T P^T on v_mfma_f32_32x32x16_bf16, K and V through LDS, widened to bf16
//                 on the way from 8 bits).
//                 Own workgroups: every sequence's other keys, dealt out evenly over
//                 the workgroups as basp_decode.hip does.
//   shared_join   a row's partial results of both kinds, by their maxima and sums
#include <math.h>

#include "basp_decode_device.hpp"
#include "basp_shared.hpp"

namespace basp {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kUnit = kWaves * kBlockKeys;  // own keys: a block per wave
static_assert(kUnit == kDecodeUnit, "the host's cut");
constexpr float kRescaleSlack = 8.f;   // log2 headroom before the reference max moves
constexpr int kPlanThreads = 1024;

// The plan, in the workspace.
struct Plan {
  int *total;    // chunks there are
  int *start;    // [b] a sequence's first own key: its group's prefix length, or 0
  int *row;      // [b] its first prefix row, in chunks of SharedCut.rows; -1: it shares nothing
  int *member;   // [b] sequences that share, group by group
  int *units;    // [b + 1] units of the sequences before, times their heads
  int *group_n, *group_first, *group_chunk;  // [n_groups] members, places in `member`, chunks
  // Of a chunk of rows: its group's first place in `member` and the members' number, the
  // prefix's length, the chunk's first row in the group.
  int4 *chunk;
};
__device__ __forceinline__ Plan plan_at(const SharedArgs &a, const SharedCut &c) {
  char *ws = static_cast<char *>(a.d.workspace);
  Plan p;
  const int b = a.d.s.b;
  p.total = reinterpret_cast<int *>(ws + c.ints);
  p.start = p.total + 1;
  p.row = p.start + b;
  p.member = p.row + b;
  p.units = p.member + b;
  p.group_n = p.units + b + 1;
  p.group_first = p.group_n + a.n_groups;
  p.group_chunk = p.group_first + a.n_groups;
  p.chunk = reinterpret_cast<int4 *>(ws + c.records);
  return p;
}

// Units of a sequence's own keys, from the tile of 16 that `start` is in.
__device__ __forceinline__ int units_of(int len, int start, int max_len) {
  return len <= start || len > max_len ? 0 : (len - (start & ~15) - 1) / kUnit + 1;
}

__device__ __forceinline__ int clamp(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// Sums of x and y over the threads before this one, and over all WAVES waves.
template <int WAVES>
__device__ __forceinline__ void before(int x, int y, int (*sums)[WAVES], int &tx, int &ty, int &ax,
                                       int &ay) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int ix = wave_scan(x), iy = wave_scan(y);
  __syncthreads();  // sums of the turn before are read
  if (lane == 63) sums[0][wave] = ix, sums[1][wave] = iy;
  __syncthreads();
  tx = ix - x, ty = iy - y, ax = ay = 0;
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) tx += sums[0][w], ty += sums[1][w];
    ax += sums[0][w], ay += sums[1][w];
  }
}

// The group that sequence s is in and whose prefix it is at least as long as, or -1. `bound`:
// groups' first sequences, then b; one group whatever their order.
template <class Bound, class Prefix>
__device__ __forceinline__ int group_of(int s, int len, int n_groups, int max_len, Bound bound,
                                        Prefix prefix) {
  if (n_groups == 0 || len <= 0 || len > max_len) return -1;
  int lo = 0, hi = n_groups;  // the last group that starts at s or before
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (bound(mid) <= s) lo = mid;
    else hi = mid;
  }
  if (s < bound(lo) || s >= bound(lo + 1)) return -1;
  const int p = prefix(lo);
  return p > 0 && len >= p ? lo : -1;
}

__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(const SharedArgs a,
                                                                   const SharedCut c) {
  const Plan p = plan_at(a, c);
  const int b = a.d.s.b, rep = a.d.n_q / a.d.s.n_k, n_groups = a.n_groups;
  const int tid = threadIdx.x;
  __shared__ int sums[2][kPlanThreads / 64];
  for (int g = tid; g < n_groups; g += kPlanThreads)
    __hip_atomic_store(p.group_n + g, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  for (int s = tid; s < b; s += kPlanThreads) {
    const int g = group_of(
        s, a.d.lens[s], n_groups, a.d.max_len, [&](int i) { return a.groups[i]; },
        [&](int i) { return a.prefix_lens[i]; });
    p.row[s] = g;  // until the last pass
    if (g >= 0) atomicAdd(p.group_n + g, 1);
  }
  __syncthreads();
  auto members_of = [&](int g) {  // at least two share, or nobody does
    const int n =
        __hip_atomic_load(p.group_n + g, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return n < 2 ? 0 : n;
  };
  int members = 0, chunks = 0, x, y, ax, ay;
  for (int g0 = 0; g0 < n_groups; g0 += kPlanThreads) {
    const int g = g0 + tid, n = g < n_groups ? members_of(g) : 0;
    const int mine = (n * rep + c.rows - 1) / c.rows;
    before<kPlanThreads / 64>(n, mine, sums, x, y, ax, ay);
    x += members, y += chunks;
    members += ax, chunks += ay;
    if (g >= n_groups) continue;
    p.group_first[g] = x;
    p.group_chunk[g] = y;
    for (int i = 0; i < mine; ++i) p.chunk[y + i] = int4{x, n, a.prefix_lens[g], i * c.rows};
  }
  if (tid == 0) *p.total = chunks;
  __syncthreads();
  members = 0;
  int units = 0;
  for (int s0 = 0; s0 < b; s0 += kPlanThreads) {
    const int s = s0 + tid, g = s < b ? p.row[s] : -1, n = g >= 0 ? members_of(g) : 0;
    const bool in = n > 0;
    const int start = in ? a.prefix_lens[g] : 0;
    before<kPlanThreads / 64>(
        in, s < b ? units_of(a.d.lens[s], start, a.d.max_len) * c.vheads : 0, sums, x, y, ax, ay);
    x += members, y += units;
    members += ax, units += ay;
    if (s >= b) continue;
    p.start[s] = start;
    p.units[s] = y;
    if (in) p.member[x] = s;
    const int rank = in ? clamp(x - p.group_first[g], 0, n - 1) : 0;
    p.row[s] = in ? p.group_chunk[g] * c.rows + rank * rep : -1;
  }
  if (tid == 0) p.units[b] = units;
}

// What a main workgroup goes by: the plan in the workspace, or its own in LDS.
struct View {
  const int *start, *member, *units;
  int4 rec;  // of its chunk
  int lead;
  bool chunk;  // there is one
};
struct Local {
  int start[kLocalSeqs], member[kLocalSeqs], units[kLocalSeqs + 1];
  int bound[kLocalGroups + 1], prefix[kLocalGroups], n[kLocalGroups];
  int first[kLocalGroups], chunk0[kLocalGroups];
  int sums[2][kWaves], rec[4];
};

// The plan of one workgroup (a launch of its own costs 4.5 us and its round trips
// through memory).  `chunk` < 0: an own workgroup, number g of G, which also leaves its
// share of the sequences' prefix rows for the join.
__device__ __forceinline__ View plan_here(const SharedArgs &a, const SharedCut &c, Local &p,
                                          int chunk, int g, int G) {
  const int b = a.d.s.b, rep = a.d.n_q / a.d.s.n_k, n_groups = a.n_groups;
  const int tid = threadIdx.x;
  constexpr int kTurns = kLocalSeqs / kThreads;
  int len[kTurns];
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int s = tid + k * kThreads;
    len[k] = s < b ? a.d.lens[s] : 0;
  }
  if (tid < n_groups) {
    p.bound[tid] = a.groups[tid];
    p.prefix[tid] = a.prefix_lens[tid];
    p.n[tid] = 0;
  }
  if (n_groups > 0 && tid == n_groups) p.bound[tid] = a.groups[tid];
  if (tid == 0) p.rec[1] = 0;
  __syncthreads();
  int of[kTurns];  // a sequence's group, if it is as long as its prefix
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    of[k] = group_of(
        tid + k * kThreads, len[k], n_groups, a.d.max_len, [&](int i) { return p.bound[i]; },
        [&](int i) { return p.prefix[i]; });
    if (of[k] >= 0) atomicAdd(&p.n[of[k]], 1);
  }
  __syncthreads();
  int all_first, all_chunks;
  {
    const int n = tid < n_groups && p.n[tid] >= 2 ? p.n[tid] : 0;
    const int mine = (n * rep + c.rows - 1) / c.rows;
    int first, chunk0;
    before<kWaves>(n, mine, p.sums, first, chunk0, all_first, all_chunks);
    if (tid < n_groups) p.first[tid] = first, p.chunk0[tid] = chunk0;
    if (mine > 0 && chunk >= chunk0 && chunk < chunk0 + mine) {
      p.rec[0] = first, p.rec[1] = n, p.rec[2] = p.prefix[tid];
      p.rec[3] = (chunk - chunk0) * c.rows;
    }
  }
  int members = 0, units = 0;
  for (int k = 0; k * kThreads < b; ++k) {
    const int s = tid + k * kThreads;
    const int gr = s < b ? of[k] : -1, n = gr >= 0 ? p.n[gr] : 0;
    const bool in = n >= 2;
    const int start = in ? p.prefix[gr] : 0;
    int at, u, am, au;
    before<kWaves>(in, s < b ? units_of(len[k], start, a.d.max_len) * c.vheads : 0, p.sums, at, u, am,
                   au);
    at += members, u += units;
    members += am, units += au;
    if (s < b) {
      p.start[s] = start;
      p.units[s] = u;
      if (in) p.member[at] = s;
      if (chunk < 0 && s % G == g) {
        const int rank = in ? clamp(at - p.first[gr], 0, n - 1) : 0;
        plan_at(a, c).row[s] = in ? p.chunk0[gr] * c.rows + rank * rep : -1;
      }
    }
  }
  if (tid == 0) p.units[b] = units;
  __syncthreads();
  View v{p.start, p.member, p.units, int4{p.rec[0], p.rec[1], p.rec[2], p.rec[3]}, 0, false};
  v.chunk = chunk >= 0 && v.rec.y > 0;
  v.lead = v.chunk ? p.member[v.rec.x] : 0;
  return v;
}

// The plan kernel's, for one workgroup.
__device__ __forceinline__ View plan_there(const SharedArgs &a, const SharedCut &c, int chunk) {
  const Plan p = plan_at(a, c);
  View v{p.start, p.member, p.units, int4{0, 0, 0, 0}, 0, false};
  if (chunk >= 0 && chunk < *p.total) {
    v.rec = p.chunk[chunk];
    v.lead = p.member[v.rec.x];
    v.chunk = true;
  }
  return v;
}

// ------------------------------------------------------------- prefix pass
// 64 rows: two row groups of 32 times two key parts of a tile; 128: four row groups.
template <int D, int RG>
struct PrefixCfg {
  static constexpr int R = RG, P = kWaves / R;  // row groups, key parts
  static constexpr int KM = kSharedTile / 32 / P;  // 32-key blocks per wave and tile
  static constexpr int DC = HeadDim<D>::DC;
  static constexpr int LW = HeadDim<D>::LW;
  static constexpr int TILE_BYTES = kSharedTile * LW * 2;
  static constexpr int LDS_BYTES = 2 * 2 * TILE_BYTES;  // two stages of K and V
  static constexpr int NS = D / 16;
  static constexpr int NE = DC / 32;
  static constexpr int PART_BYTES = NE * 4 * 1024 + 512;
  static_assert((P - 1) * R * PART_BYTES <= LDS_BYTES, "the merge area fits the stages");
};

// What a thread carries from the pages to LDS: 16 bytes of one row in each of N blocks
// of 16 keys (a tile has four; a block lies in one page, so its address is a scalar).
// Where a row is short, two or all of the blocks are carried at once, by other waves.
template <int D, bool E4M3>
struct Carry {
  static constexpr int kRowBytes = D * (E4M3 ? 1 : 2), kPerRow = kRowBytes / 16;
  static constexpr int kAtOnce = kPerRow <= 4 ? 4 : kPerRow <= 8 ? 2 : 1;
  static constexpr int kPerBlock = kThreads / kAtOnce;  // threads
  static constexpr int N = kSharedTile / 16 / kAtOnce;
  u32x4 k[N], v[N];
  uint32_t ks[N], vs[N];  // scale bytes
  int id[N];              // page numbers of the next tile (wave-uniform)
  bool bad[N];            // this tile's block lies on no valid page (wave-uniform)
};

template <int D, bool E4M3, int RG>
__device__ void prefix_unit(const SharedArgs &a, const SharedCut &c, unsigned char *smem,
                            Local &local) {
  using C = PrefixCfg<D, RG>;
  using T = LdsTile<C::LW>;
  using W = Carry<D, E4M3>;
  constexpr int kVRegion = 2 * C::TILE_BYTES;
  const CacheShape &cs = a.d.s;
  const int rep = a.d.n_q / cs.n_k;
  // Splits fastest, in eights where there are as many: workgroups go round the eight
  // XCDs, so a split's chunks of rows read its keys through one L2.
  const int x = blockIdx.x;
  const int split = scalar(x % c.splits), rest = scalar(x / c.splits);
  const int chunk = scalar(rest / cs.n_k), kvh = scalar(rest % cs.n_k);
  const View plan =
      c.local ? plan_here(a, c, local, chunk, 0, 1) : plan_there(a, c, chunk);  // uniform
  if (!plan.chunk) return;  // workgroup-uniform
  const int4 rec = plan.rec;
  const int lead = scalar(plan.lead);
  const int first = scalar(rec.x), members = scalar(rec.y), prefix = scalar(rec.z),
            row0 = scalar(rec.w);
  const int rows = members * rep - row0;  // of this chunk (and those after it)
  const int *table = a.d.table + (size_t)lead * cs.max_pages;
  const int tiles = (prefix + kSharedTile - 1) / kSharedTile;
  const int t0 = (int)((long long)split * tiles / c.splits);
  const int t1 = (int)((long long)(split + 1) * tiles / c.splits);

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = scalar(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const int rg = w % C::R, part = w / C::R;
  const int i = 32 * rg + l32;  // the lane's row
  const bool live = i < rows;
  const int seq = live ? plan.member[first + (row0 + i) / rep] : 0;
  const int head = kvh * rep + (live ? (row0 + i) % rep : 0);
  bf16x8 qf[C::NS];
  {
    const uint16_t *qp = static_cast<const uint16_t *>(a.d.q) + (long long)seq * a.d.q_row +
                         (size_t)head * D;
#pragma unroll
    for (int s = 0; s < C::NS; ++s) {
      u32x4 v = {0, 0, 0, 0};
      if (live) v = *reinterpret_cast<const u32x4 *>(qp + 16 * s + 8 * hh);
      qf[s] = as_bf16x8(v);
    }
  }
  const int at = live ? a.d.lens[seq] - 1 : 0;
  const float sl = a.slopes && live ? a.slopes[head] * kLog2e : 0.f;
  const float c2 = a.d.scale * kLog2e;
  const bool capped = a.cap > 0.f;
  const float c1 = capped ? 2.f * c2 / a.cap : 0.f, cap2 = a.cap * kLog2e;
  float m_ref = -INFINITY, l_run = 0.f;

  f32x16 oacc[C::NE];
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[n][r] = 0.f;

  W x_;
  const int block = scalar(tid / W::kPerBlock);  // of those at once
  const int mine = tid % W::kPerBlock, row = mine / W::kPerRow, cc = mine % W::kPerRow;
  const bool carries = mine < 16 * W::kPerRow;
  auto first_key = [&](int t, int j) { return t * kSharedTile + 16 * (W::kAtOnce * j + block); };
  auto load_pages = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < W::N; ++j) {
      const int pi = first_key(t, j) >> cs.page_log2;
      x_.id[j] = t < t1 && first_key(t, j) < prefix && pi < cs.max_pages ? scalar_load(table, pi) : -1;
    }
  };
  auto load_rows = [&](int t) __attribute__((always_inline)) {  // of the pages at hand
#pragma unroll
    for (int j = 0; j < W::N; ++j) {
      const int key = first_key(t, j), id = scalar(x_.id[j]);
      const bool there = id >= 0 && id < cs.n_pages;
      const size_t at = there ? (((size_t)id * cs.n_k + kvh) << cs.page_log2) +
                                    (key & ((1 << cs.page_log2) - 1))
                              : 0;
      // keys past the end: the last row again, or (a whole block) any; put() clears V
      const int last = there ? prefix - key - 1 : 0;
      const uint32_t r = (uint32_t)(row < last ? row : last);
      const uint32_t off = r * W::kRowBytes + cc * 16;
      const gptr kb = scalar_base(static_cast<const char *>(a.d.k_pages) + at * W::kRowBytes);
      const gptr vb = scalar_base(static_cast<const char *>(a.d.v_pages) + at * W::kRowBytes);
      if (carries) {
        x_.k[j] = load_at<u32x4>(kb, off);
        x_.v[j] = load_at<u32x4>(vb, off);
        if constexpr (E4M3) {
          x_.ks[j] = load_at<uint8_t>(scalar_base(a.d.k_scales + at), r);
          x_.vs[j] = load_at<uint8_t>(scalar_base(a.d.v_scales + at), r);
        }
      }
      x_.bad[j] = !there && key < prefix;
    }
  };
  auto widen8 = [&](uint32_t lo, uint32_t hi, uint32_t byte) __attribute__((always_inline)) {
    const float scale = __builtin_bit_cast(float, byte << 23);
    return u32x4{
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
  };
  const int to0 = T::off(row + 16 * block, E4M3 ? 2 * cc : cc);
  const int to1 = E4M3 ? T::off(row + 16 * block, 2 * cc + 1) : 0;
  auto put = [&](int t, int stage) __attribute__((always_inline)) {  // into LDS
    if (!carries) return;
    unsigned char *Ks = smem + stage * C::TILE_BYTES;
    if ((t + 1) * kSharedTile > prefix) {  // workgroup-uniform: the last tile
      // V of keys past the end must not meet their weight of 0 as infinities or NaN
#pragma unroll
      for (int j = 0; j < W::N; ++j)
        if (first_key(t, j) + row >= prefix) {
          x_.v[j] = u32x4{0, 0, 0, 0};
          if constexpr (E4M3) x_.vs[j] = 127;
        }
    }
#pragma unroll
    for (int j = 0; j < W::N; ++j) {
      const int at = j * 16 * W::kAtOnce * T::ROW_BYTES;
      u32x4 k0 = x_.k[j], v0 = x_.v[j];
      if constexpr (E4M3) {
        *reinterpret_cast<u32x4 *>(Ks + to1 + at) = widen8(k0.z, k0.w, x_.ks[j]);
        *reinterpret_cast<u32x4 *>(Ks + kVRegion + to1 + at) = widen8(v0.z, v0.w, x_.vs[j]);
        k0 = widen8(k0.x, k0.y, x_.ks[j]);
        v0 = widen8(v0.x, v0.y, x_.vs[j]);
      }
      if (x_.bad[j]) k0 = u32x4{0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu};  // NaN
      *reinterpret_cast<u32x4 *>(Ks + to0 + at) = k0;
      *reinterpret_cast<u32x4 *>(Ks + kVRegion + to0 + at) = v0;
    }
  };

  const int part_off = part * 32 * C::KM * T::ROW_BYTES;
  int k_off[C::NS], v_off[C::NE][2];
#pragma unroll
  for (int s = 0; s < C::NS; ++s) k_off[s] = T::off(l32, 2 * s + hh) + part_off;
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int y = 0; y < 2; ++y)
      v_off[n][y] = kVRegion + part_off +
                    tr_piece_off<C::LW>(4 * hh + 8 * y, 32 * n + 16 * ((lane >> 4) & 1), lane);
  auto tile = [&](int t, int stage) __attribute__((always_inline)) {
    const unsigned char *Ks = smem + stage * C::TILE_BYTES;
#pragma unroll
    for (int m = 0; m < C::KM; ++m) {
      const int mo = m * 32 * T::ROW_BYTES;
      f32x16 sc;
#pragma unroll
      for (int s = 0; s < C::NS; ++s)
        sc = mfma32x32x16(*reinterpret_cast<const bf16x8 *>(Ks + k_off[s] + mo), qf[s],
                          s == 0 ? f32x16{} : sc);
      // sc[r] = (q . k) of key jl + 8(r/4) + r%4 for this lane's row
      const int jl = t * kSharedTile + 32 * (C::KM * part + m) + 4 * hh;
      const float away = (float)(at - jl);
      if (capped) {  // workgroup-uniform, as the next
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = fmaf(cap_r(sc[r], c1), -2.f * cap2, cap2);
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] *= c2;
      }
      if (a.slopes) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          sc[r] = fmaf(-sl, away - (float)(8 * (r >> 2) + (r & 3)), sc[r]);
      }
      if (jl - 4 * hh + 32 > prefix) {  // wave-uniform: the last tile
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (jl + 8 * (r >> 2) + (r & 3) >= prefix) sc[r] = -INFINITY;
      }
      // Against a running maximum with a cap too: that bounds the scores, but with a reference
      // that stands still P lies in 2^(+-92) at a cap of 64, too wide for its products with V,
      // and a weight alone in its row is rounded (64 sequences on one prompt of 32K, 8 heads on
      // 1, a cap of 50: 37.2 us standing still, 35.8).
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
      mx = pair_max(mx);
      const bool grow = mx > m_ref + kRescaleSlack;
      if (__builtin_amdgcn_ballot_w64(grow)) {  // wave-uniform, rare after the first tiles
        asm volatile("" ::: "memory");
        const float alpha = grow ? fast_exp2(m_ref - mx) : 1.f;
        m_ref = grow ? mx : m_ref;
        l_run *= alpha;
#pragma unroll
        for (int n = 0; n < C::NE; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[n][r] *= alpha;
      }
      const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
      float psum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[r] = fast_exp2(sc[r] - m_use);
        psum += sc[r];
      }
      l_run += psum;
      bf16x8 pf[2];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const int b8 = 8 * s2;
        pf[s2] = as_bf16x8(
            u32x4{pack_bf16x2(sc[b8 + 0], sc[b8 + 1]), pack_bf16x2(sc[b8 + 2], sc[b8 + 3]),
                  pack_bf16x2(sc[b8 + 4], sc[b8 + 5]), pack_bf16x2(sc[b8 + 6], sc[b8 + 7])});
      }
#pragma unroll
      for (int n = 0; n < C::NE; ++n)
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          const int ro = mo + s2 * 16 * T::ROW_BYTES;
          oacc[n] =
              mfma32x32x16(tr_operand(Ks, v_off[n][0] + ro, v_off[n][1] + ro), pf[s2], oacc[n]);
        }
    }
  };
  // One tile of rows and the next one's page numbers in flight over a tile's
  // products; two stages, so that one barrier a tile is enough.
  __syncthreads();  // the plan in LDS has been read
  load_pages(t0);
  if (t0 < t1) load_rows(t0);
  load_pages(t0 + 1);
  auto turn = [&](int t, int stage) __attribute__((always_inline)) {
    put(t, stage);
    if (t + 1 < t1) {
      load_rows(t + 1);
      load_pages(t + 2);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier_no_fence();
    tile(t, stage);
  };
  for (int t = t0; t < t1; t += 2) {
    turn(t, 0);
    if (t + 1 < t1) turn(t + 1, 1);
  }

  // The parts of a row group brought together, and out.
  float l_tot = pair_sum(l_run), m = m_ref, w0 = 1.f, w1 = 0.f;
  unsigned char *area = smem + rg * C::PART_BYTES;
  if constexpr (C::P == 2) {
    constexpr int kScalars = C::NE * 4 * 1024;
    __syncthreads();
    if (part == 1) {
#pragma unroll
      for (int n = 0; n < C::NE; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4 *>(area + (n * 4 + g) * 1024 + 16 * lane) =
              f32x4{oacc[n][4 * g], oacc[n][4 * g + 1], oacc[n][4 * g + 2], oacc[n][4 * g + 3]};
      *reinterpret_cast<float *>(area + kScalars + 4 * lane) = m_ref;
      *reinterpret_cast<float *>(area + kScalars + 256 + 4 * lane) = l_tot;
    }
    __syncthreads();
    if (part == 1) return;
    const float m1 = *reinterpret_cast<const float *>(area + kScalars + 4 * lane);
    const float l1 = *reinterpret_cast<const float *>(area + kScalars + 256 + 4 * lane);
    m = fmaxf(m_ref, m1);
    const float ref = m == -INFINITY ? 0.f : m;
    w0 = fast_exp2(m_ref - ref), w1 = fast_exp2(m1 - ref);
    l_tot = l_tot * w0 + l1 * w1;
  }
  if (!live) return;
  char *ws = static_cast<char *>(a.d.workspace);
  const size_t slot = ((size_t)(chunk * cs.n_k + kvh) * c.splits + split) * c.rows + i;
  float *po = reinterpret_cast<float *>(ws + c.part_o) + slot * D;
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (32 * n + 8 * g >= D) continue;  // padding columns
      f32x4 y = {oacc[n][4 * g], oacc[n][4 * g + 1], oacc[n][4 * g + 2], oacc[n][4 * g + 3]};
      if constexpr (C::P == 2) {
        const f32x4 z = *reinterpret_cast<const f32x4 *>(area + (n * 4 + g) * 1024 + 16 * lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = y[e] * w0 + z[e] * w1;
      }
      *reinterpret_cast<f32x4 *>(po + 32 * n + 8 * g + 4 * hh) = y;
    }
  if (hh == 0) reinterpret_cast<f32x2 *>(ws + c.part_ml)[slot] = f32x2{m, l_tot};
}

// ------------------------------------------------------------ the own keys
// Workgroup g of `own.groups`: its run of units, as in basp_decode.hip.  A head that is whole
// in one run is final where its sequence shares nothing, else it goes to its rows'
// places; one that several runs share leaves partial results in the slot of either's
// first (0) or last (1) head.  open[sequence * vheads + vhead] says which: `count` 0: final,
// or nothing; -1: in the rows' places; else the partial results, the first in slot
// first % 2 of workgroup first / 2, the others in slot 0 of the next ones.
template <int D, bool E4M3, int RG>
__device__ void own_unit(const SharedArgs &a, const SharedCut &c, int g, unsigned char *smem,
                         int *found, Local &local) {
  using B = Block<D, E4M3>;
  constexpr int kRows = 16 * RG;
  const DecodeArgs &d = a.d;
  const View plan =
      c.local ? plan_here(a, c, local, -1, g, c.own.groups) : plan_there(a, c, -1);  // uniform
  const int rep = scalar(d.n_q / d.s.n_k), row_groups = c.own.row_groups, R = c.vheads;
  const int b = d.s.b, G = c.own.groups;
  const int wave = scalar(threadIdx.x / 64);
  const int lane = threadIdx.x % 64, m = lane % 16, cq = lane / 16;
  float(*so)[kRows][D + 4] = reinterpret_cast<float(*)[kRows][D + 4]>(smem);
  float(*sm)[kRows] = reinterpret_cast<float(*)[kRows]>(so + kWaves);
  float(*sl)[kRows] = sm + kWaves;
  char *ws = static_cast<char *>(d.workspace);
  DecodeOpen *opens = reinterpret_cast<DecodeOpen *>(ws + c.open);
  f32x2 *own_ml = reinterpret_cast<f32x2 *>(ws + c.own_ml);
  float *own_o = reinterpret_cast<float *>(ws + c.own_o);
  f32x2 *row_ml = reinterpret_cast<f32x2 *>(ws + c.row_ml);
  float *row_o = reinterpret_cast<float *>(ws + c.row_o);

  // Sequences without own keys, or with more than the call allows, are shared out.
  for (int s = g; s < b; s += G) {
    const int len = scalar_load(d.lens, s), start = plan.start[s];
    if (units_of(len, start, d.max_len) > 0) continue;
    for (int i = threadIdx.x; i < R; i += kThreads) opens[(size_t)s * R + i].count = 0;
    if (len == start && start > 0) continue;  // all of it is the prefix
    uint16_t *o = static_cast<uint16_t *>(d.o) + (size_t)s * d.n_q * D;
    for (int i = threadIdx.x; i < d.n_q * D; i += kThreads) o[i] = len <= 0 ? 0 : 0x7FFF;
    if (d.lse)
      for (int i = threadIdx.x; i < d.n_q; i += kThreads)
        d.lse[(size_t)s * d.n_q + i] = len <= 0 ? -INFINITY : __builtin_nanf("");
  }

  const int total = plan.units[b];
  const int quota = scalar((total + G - 1) / G);
  const long long first = (long long)g * quota;
  if (first >= total) return;
  const int begin = (int)first, end = total - begin < quota ? total : begin + quota;
  if (b <= 8 * kThreads) {
    for (int s = threadIdx.x; s < b; s += kThreads)
      if (begin >= plan.units[s] && begin < plan.units[s + 1]) *found = s;
  } else if (threadIdx.x == 0) {
    int lo = 0, hi = b;  // units[lo] <= begin < units[hi]
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (plan.units[mid] <= begin) lo = mid;
      else hi = mid;
    }
    *found = lo;
  }
  __syncthreads();
  int seq = scalar(*found);
  int len = 0, start = 0, n = 0;
  auto enter = [&]() {
    len = scalar(d.lens[seq]);
    start = scalar(plan.start[seq]);
    n = units_of(len, start, d.max_len);
  };
  enter();
  if (n == 0) return;  // not reached while lens stays as it is
  const int at0 = begin - scalar(plan.units[seq]);
  int head = scalar(at0 / n), u = scalar(at0 % n);

  Pages pg;
  pg.k = static_cast<const char *>(d.k_pages);
  pg.v = static_cast<const char *>(d.v_pages);
  pg.ks = d.k_scales;
  pg.vs = d.v_scales;
  pg.page_log2 = d.s.page_log2;
  pg.n_pages = d.s.n_pages;
  pg.max_pages = d.s.max_pages;
  pg.n_k = d.s.n_k;
  const float scale2 = d.scale * kLog2e;
  KeyRule rule;
  rule.capped = a.cap > 0.f;
  rule.c1 = rule.capped ? 2.f * scale2 / a.cap : 0.f;
  rule.cap2 = a.cap * kLog2e;

  for (int pos = begin; pos < end;) {
    const int take = n - u < end - pos ? n - u : end - pos;  // units of this head
    const int base = start & ~15;
    const int lo = base + u * kUnit;
    const int hi = lo + take * kUnit < len ? lo + take * kUnit : len;
    const int kvh = scalar(head / row_groups), grp = scalar(head % row_groups);
    const int h0 = kvh * rep + grp * kRows;  // first query head
    const int heads = rep - grp * kRows < kRows ? rep - grp * kRows : kRows;
    pg.table = d.table + (size_t)seq * d.s.max_pages;
    pg.kvh = kvh;
    rule.at = len - 1;
    rule.lo = start;

    int t = lo + wave * kBlockKeys;
    Block<D, E4M3> x;
    int ids[kTiles];
    load_ids(pg, t, hi, ids);
    State<B> st[RG];
    float slope[RG];
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      const int h = 16 * rg + m;
      const uint16_t *qp = static_cast<const uint16_t *>(d.q) + (long long)seq * d.q_row +
                           (size_t)(h0 + h) * D;
#pragma unroll
      for (int s = 0; s < B::kSteps; ++s) {
        const int e = E4M3 ? 64 * (s / 2) + 16 * cq + 8 * (s % 2) : 32 * s + 8 * cq;
        u32x4 w = {0, 0, 0, 0};
        if (h < heads && e < D) w = *reinterpret_cast<const u32x4 *>(qp + e);
        st[rg].q[s] = as_bf16x8(w);
      }
      slope[rg] = a.slopes && h < heads ? a.slopes[h0 + h] * kLog2e : 0.f;
      st[rg].m = -INFINITY;
      st[rg].l = 0.f;
#pragma unroll
      for (int i = 0; i < B::kCols; ++i) st[rg].o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    while (t < hi) {
      load_block<D, E4M3>(x, pg, t, hi, ids);
      load_ids(pg, t + kUnit, hi, ids);
      take_block<D, E4M3, RG, true>(x, st, scale2, hi - t, rule, slope, t);
      t += kUnit;
    }

    // The four waves.
    __syncthreads();  // the last head's
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      const float l = column_sum(st[rg].l);
      if (cq == 0) sm[wave][16 * rg + m] = st[rg].m, sl[wave][16 * rg + m] = l;
    }
    __syncthreads();
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      const int h = 16 * rg + m;
      float M = sm[0][h];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm[w][h]);
      const float f = fast_exp2(st[rg].m - (M == -INFINITY ? 0.f : M));
      const f32x4 *acc = st[rg].o;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (B::kCols * (4 * cq + r) < D) {
#pragma unroll
          for (int i = 0; i < B::kCols; i += 4)
            *reinterpret_cast<f32x4 *>(&so[wave][h][B::kCols * (4 * cq + r) + i]) =
                f32x4{acc[i][r] * f, acc[i + 1][r] * f, acc[i + 2][r] * f, acc[i + 3][r] * f};
        }
    }
    __syncthreads();
    const size_t row0 = (size_t)seq * d.n_q + h0;
    const bool whole = take == n, shares = start > 0;
    const int slot = pos != begin;
    if (u == 0 && threadIdx.x == 0)
      opens[(size_t)seq * R + head] =
          DecodeOpen{0, heads, !whole ? (pos + n - 1) / quota - g + 1 : shares ? -1 : 0,
                     2 * g + slot};
    for (int i = threadIdx.x; i < heads * (D / 4); i += kThreads) {
      const int h = i / (D / 4), e = i % (D / 4) * 4;
      float mx = sm[0][h], L = 0.f;
#pragma unroll
      for (int w = 1; w < kWaves; ++w) mx = fmaxf(mx, sm[w][h]);
      const float ref = mx == -INFINITY ? 0.f : mx;
      f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        L += fast_exp2(sm[w][h] - ref) * sl[w][h];
        O += *reinterpret_cast<const f32x4 *>(&so[w][h][e]);
      }
      if (whole && !shares) {
        O *= 1.f / L;
        *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(d.o) + (row0 + h) * D + e) =
            u32x2{pack_bf16x2(O.x, O.y), pack_bf16x2(O.z, O.w)};
        if (e == 0 && d.lse) d.lse[row0 + h] = (mx + fast_log2(L)) * kLn2;
      } else {
        const size_t at = whole ? row0 + h : ((size_t)g * 2 + slot) * kRows + h;
        *reinterpret_cast<f32x4 *>((whole ? row_o : own_o) + at * D + e) = O;
        if (e == 0) (whole ? row_ml : own_ml)[at] = f32x2{mx, L};
      }
    }
    pos += take;
    if (pos < end) {  // the next head, of the next sequence that has own keys
      u = 0;
      if (++head == R) {
        head = 0;
        n = 0;
        while (n == 0 && ++seq < b) enter();
        if (n == 0) break;  // not reached while lens stays as it is
      }
    }
  }
}

template <int D, bool E4M3, int PR, int RG>
__global__ __launch_bounds__(kThreads, 2) void shared_main_kernel(const SharedArgs a,
                                                                  const SharedCut c) {
  constexpr int kOwn = kWaves * 16 * RG * ((D + 4) + 2) * 4;
  // The plan behind what the own keys take, among what the prefix's tiles take later.
  constexpr int kPrefix = PrefixCfg<D, PR>::LDS_BYTES, kPlanned = kOwn + (int)sizeof(Local);
  constexpr int kLds = kPlanned > kPrefix ? kPlanned : kPrefix;
  __shared__ __attribute__((aligned(16))) unsigned char smem[kLds];
  __shared__ int found;
  Local &local = *reinterpret_cast<Local *>(smem + kOwn);
  if ((int)blockIdx.x < c.prefix_blocks)  // workgroup-uniform
    prefix_unit<D, E4M3, PR>(a, c, smem, local);
  else
    own_unit<D, E4M3, RG>(a, c, (int)blockIdx.x - c.prefix_blocks, smem, &found, local);
}

// ------------------------------------------------------------------ the join
// A workgroup per row that has partial results: these in turn over the four waves,
// two elements of d a lane, each wave with a running maximum.
template <int D>
__global__ __launch_bounds__(kThreads) void shared_join_kernel(const SharedArgs a,
                                                               const SharedCut c) {
  const DecodeArgs &d = a.d;
  const Plan plan = plan_at(a, c);
  const int row = blockIdx.x, seq = scalar(row / d.n_q), h = scalar(row % d.n_q);
  const int rep = scalar(d.n_q / d.s.n_k), kvh = scalar(h / rep), hr = scalar(h % rep);
  char *ws = static_cast<char *>(d.workspace);
  const DecodeOpen open = reinterpret_cast<const DecodeOpen *>(
      ws + c.open)[(size_t)seq * c.vheads + kvh * c.own.row_groups + hr / c.own.rows];
  const int prow = plan.row[seq];
  const int own = open.count < 0 ? 1 : open.count, shared = prow >= 0 ? c.splits : 0;
  const int n = own + shared;
  if (n == 0) return;
  const int at_p = prow + hr;
  const size_t base =
      ((size_t)(at_p / c.rows * d.s.n_k + kvh) * c.splits) * c.rows + at_p % c.rows;
  const f32x2 *part_ml = reinterpret_cast<const f32x2 *>(ws + c.part_ml);
  const float *part_o = reinterpret_cast<const float *>(ws + c.part_o);
  auto find = [&](int i, const f32x2 *&ml, const float *&o) {
    if (i < shared) {
      const size_t x = base + (size_t)i * c.rows;
      ml = part_ml + x, o = part_o + x * D;
    } else if (open.count < 0) {
      ml = reinterpret_cast<const f32x2 *>(ws + c.row_ml) + row;
      o = reinterpret_cast<const float *>(ws + c.row_o) + (size_t)row * D;
    } else {
      const int j = i - shared;
      const size_t x = (size_t)(j ? (open.first | 1) - 1 + 2 * j : open.first) * c.own.rows +
                       hr % c.own.rows;
      ml = reinterpret_cast<const f32x2 *>(ws + c.own_ml) + x;
      o = reinterpret_cast<const float *>(ws + c.own_o) + x * D;
    }
  };
  const int wave = scalar(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int col = 2 * lane < D ? 2 * lane : 0;
  float M = -INFINITY, l = 0.f;
  f32x2 O = {0.f, 0.f};
  constexpr int kAtOnce = 8;
  for (int i0 = wave; i0 < n; i0 += kAtOnce * kWaves) {
    f32x2 x[kAtOnce], o[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = i0 + u * kWaves < n ? i0 + u * kWaves : i0;  // again the first: dropped below
      const f32x2 *ml;
      const float *po;
      find(i, ml, po);
      x[u] = *ml;
      o[u] = *reinterpret_cast<const f32x2 *>(po + col);
    }
    float mx = M;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) mx = fmaxf(mx, x[u].x);
    const float ref = mx == -INFINITY ? 0.f : mx, f = fast_exp2(M - ref);
    M = mx;
    l *= f;
    O *= f;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      if (i0 + u * kWaves < n) {
        const float w = fast_exp2(x[u].x - ref);
        l += w * x[u].y;
        O += w * o[u];
      }
  }
  __shared__ float so[kWaves][D + 2], sm[kWaves], sl[kWaves];
  if (2 * lane < D) so[wave][2 * lane] = O.x, so[wave][2 * lane + 1] = O.y;
  if (lane == 0) sm[wave] = M, sl[wave] = l;
  __syncthreads();
  if (wave != 0) return;
  M = sm[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm[w]);
  const float ref = M == -INFINITY ? 0.f : M;
  l = 0.f;
  O = f32x2{0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float f = fast_exp2(sm[w] - ref);
    l += f * sl[w];
    O += f * f32x2{so[w][col], so[w][col + 1]};
  }
  const float inv = 1.f / l;
  if (2 * lane < D)
    static_cast<uint32_t *>(d.o)[((size_t)row * D + 2 * lane) / 2] =
        pack_bf16x2(O.x * inv, O.y * inv);
  if (lane == 0 && d.lse) d.lse[row] = (M + fast_log2(l)) * kLn2;
}

template <int D, bool E4M3>
void main_typed(const SharedArgs &a, const SharedCut &c, hipStream_t stream) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(c.prefix_blocks + c.own.groups), dim3(kThreads), 0, stream, a,
                       c);
  };
  if (c.own.rows == 16)
    c.rows == 64 ? go(shared_main_kernel<D, E4M3, 2, 1>) : go(shared_main_kernel<D, E4M3, 4, 1>);
  else
    c.rows == 64 ? go(shared_main_kernel<D, E4M3, 2, 2>) : go(shared_main_kernel<D, E4M3, 4, 2>);
}

template <int D>
hipError_t launch_dim(const SharedArgs &a, const SharedCut &c, hipStream_t stream) {
  if (!c.local)
    hipLaunchKernelGGL(shared_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a, c);
  if (a.d.s.e4m3) main_typed<D, true>(a, c, stream);
  else main_typed<D, false>(a, c, stream);
  hipLaunchKernelGGL((shared_join_kernel<D>), dim3((unsigned)(a.d.s.b * a.d.n_q)), dim3(kThreads),
                     0, stream, a, c);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_decode_shared(const SharedArgs &a, hipStream_t stream) {
  const SharedCut c =
      shared_cut(a.d.s.b, a.d.n_q, a.d.s.n_k, a.d.s.d, a.d.max_len, a.n_groups);
  switch (a.d.s.d) {
    case 64: return launch_dim<64>(a, c, stream);
    case 80: return launch_dim<80>(a, c, stream);
    case 96: return launch_dim<96>(a, c, stream);
    default: return launch_dim<128>(a, c, stream);
  }
}

}  // namespace basp
