// basp_decode.hip -- attention of one new token per sequence over a paged
// key-value cache:
//   O = sum_{j < len} softmax_j(scale q . k_j) v_j,  LSE = log sum_j exp(scale q . k_j).
//
// Bound by HBM: every key and value of the cache is read once, for n_q/n_k
// operations a byte of bf16 and twice that in 8 bits (8 and 16 on 8 query heads a kv
// head; the second product of the weights, which are two bf16, is half as much
// again).  That is more than the vector units do beside such a stream and little for the
// matrix cores.
//
// The keys of all sequences are dealt out in runs: a unit is 128 keys of one kv
// head for up to 16 of its query heads (32 where it has more than 16), and each of at
// most 768 workgroups (512 of 32 heads) takes one run of units, in the order of sequences,
// heads and keys.  All runs but the last are as long, ceil(units / workgroups): even
// where there are many units, while 769 of them make runs of two, as 1536 do (one
// head in bf16, 769, 1024, 1100, 1536, 1537, 2304, 2305 units: 18.7, 20.7, 23.6, 26.1,
// 25.8, 33.7, 35.8 us).  The lengths are known on the device only, so each workgroup
// adds them up to find its run.  Its four waves take a block of 32 keys of each unit,
// each with a running maximum, sum and O of its own, joined in LDS at the end of a
// sequence's head or of the run.  Only the first and the last head of a run can be shared with other
// workgroups; their partial results are joined by a second kernel:
//   M = max_i m_i,  O = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i
// (scores in log2 units).  Splits of a fixed number of keys, one workgroup each,
// left the longest ones to run alone at the end: 64 ragged sequences of up to 32K
// tokens, 8 heads on 2 of 128, took 236 us, dealt out evenly 198.
//
// Nothing passes through LDS on the way to the matrix cores: the operands of
// v_mfma_f32_16x16x32_bf16 (lane l: 8 consecutive contraction elements
// 8(l/16).. of row or column l%16; accumulator register r: row 4(l/16) + r,
// column l%16) come straight from the pages.
//   S^T = K Q^T   rows: 16 keys of a tile, columns: query heads.  A lane loads 16
//     bytes of key l%16, the four lanes of a key 64 contiguous bytes; which
//     elements of d a step contracts does not matter as long as Q has them in the same
//     order (8 bits: a lane's 16 bytes feed two steps).
//   O^T = V^T P^T   the scores of two tiles are, lane by lane, P^T's operand: slot
//     e of the contraction is key 4(l/16) + e of the first tile, e - 4 of the
//     second.  V^T needs, for those 8 keys, one column per lane and product.  Lane
//     l loads, of each of its 8 keys, the 8 elements 8(l%16).. (four at d = 64), 16
//     lanes a whole contiguous row, and product i takes element i of each: the 8 x 8
//     elements of a lane are transposed in its own registers, 32 byte
//     permutations per 32 keys, which the vector units have room for.  Row m of
//     product i is then element 8m + i of O.
#include <math.h>

#include "basp_device.hpp"
#include "basp_ops.hpp"

namespace basp {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTiles = 2;  // of 16 keys, in a wave's block
constexpr int kBlockKeys = 16 * kTiles, kUnit = kWaves * kBlockKeys;  // a unit: a block per wave
static_assert(kUnit == kDecodeUnit, "the host's cut");
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ f32x4 mfma16x16x32(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Lanes l and l^16: v_permlane16_swap exchanges odd rows of 16 lanes of its
// first register with even rows of its second.  (Inline asm and nops as in
// lane_halves.)
__device__ __forceinline__ void lane_rows(float x, float &lo, float &hi) {
  lo = x;
  hi = x;
  asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(lo), "+v"(hi));
}
// Maximum and sum over the four lanes l%16 + 16c, in each of them.
__device__ __forceinline__ float column_max(float x) {
  float lo, hi;
  lane_rows(x, lo, hi);
  return pair_max(fmaxf(lo, hi));
}
__device__ __forceinline__ float column_sum(float x) {
  float lo, hi;
  lane_rows(x, lo, hi);
  return pair_sum(lo + hi);
}

// Low (HI = false) or high halves of two words side by side.
template <bool HI>
__device__ __forceinline__ uint32_t halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, HI ? 0x07060302u : 0x05040100u);
}

// Two e4m3 (the low or high half of a word) as two bf16, exactly.
template <bool HI>
__device__ __forceinline__ uint32_t widen(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HI));
}

__device__ __forceinline__ float pow2_of_byte(uint32_t w, int i) {
  return __builtin_bit_cast(float, ((w >> (8 * i)) & 0xFFu) << 23);
}

// What a wave loads of one block of keys.
template <int D, bool E4M3>
struct Block {
  static constexpr int kElem = E4M3 ? 1 : 2;
  static constexpr int kRowBytes = D * kElem;
  static constexpr int kLoads = (kRowBytes + 63) / 64;  // of 64 bytes per key
  static constexpr int kSteps = E4M3 ? 2 * kLoads : kLoads;
  static constexpr int kCols = D <= 64 ? 4 : 8;       // elements of d per lane of V
  static constexpr int kWords = kCols * kElem / 4;    // 32-bit words of V per key and lane
  u32x4 k[kTiles][kLoads];
  uint32_t v[8][kWords];
  uint32_t ks[kTiles], vs[kTiles];  // scale bytes of keys 4(l/16)..
  bool bad;                         // a key on no valid page (wave-uniform)
};

// Where the pages of a workgroup's kv head are.
struct Pages {
  const char *k, *v;
  const unsigned char *ks, *vs;
  const int *table;  // of the sequence
  int page_log2, n_pages, max_pages, n_k, kvh;
};

// A wave-uniform value in a scalar register.  The compiler would move address
// arithmetic that it placed in vector registers (integer division, clamps) back
// only by a loop over the lanes around every load.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A load at a scalar base plus a 32-bit offset per lane.
typedef const __attribute__((address_space(1))) char *gptr;
__device__ __forceinline__ gptr scalar_base(const void *p) {
  const uint64_t a = (uint64_t)(uintptr_t)p;
  const uint32_t lo = (uint32_t)scalar((int)(uint32_t)a), hi = (uint32_t)scalar((int)(a >> 32));
  return (gptr)(((uint64_t)hi << 32) | lo);
}
template <typename T>
__device__ __forceinline__ T load_at(gptr base, uint32_t off) {
  return *(const __attribute__((address_space(1))) T *)(base + off);
}
// The same with the non-temporal hint: for V, whose rows a load reads whole (64
// ragged sequences of up to 32K tokens: 198 -> 178 us in bf16, 115 -> 106 in 8 bits).
// K's loads read half a cache line each: with the hint 176 and 108, and K by way
// of LDS in whole rows with it 178 and 106.
template <typename T>
__device__ __forceinline__ T load_once(gptr base, uint32_t off) {
  return __builtin_nontemporal_load((const __attribute__((address_space(1))) T *)(base + off));
}

// An entry of the block table or of lens: a load through the scalar cache, which
// the counter that the pages' loads are waited by does not see (nothing writes
// either while the kernel runs).
__device__ __forceinline__ int scalar_load(const int *p, size_t i) {
  return *((const __attribute__((address_space(4))) int *)(uintptr_t)p + i);
}

// Page numbers of a block's tiles (tiles do not cross pages: both are
// multiples of 16).
__device__ __forceinline__ void load_ids(const Pages &p, int t0, int hi, int (&id)[kTiles]) {
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int at = t0 + 16 * t, pi = at >> p.page_log2;
    id[t] = -1;
    if (at < hi && pi < p.max_pages) id[t] = scalar_load(p.table, pi);
  }
}

// Loads of the block from key t0 on.  Keys from `hi` on read the last row before
// it instead (take_block drops them), tiles with no key before `hi` or on no valid
// page the first row of page 0.
template <int D, bool E4M3>
__device__ __forceinline__ void load_block(Block<D, E4M3> &b, const Pages &p, int t0, int hi,
                                           const int (&ids)[kTiles]) {
  using B = Block<D, E4M3>;
  const int lane = threadIdx.x % 64, m = lane % 16, c = lane / 16;
  b.bad = false;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int at = t0 + 16 * t;
    const int id = scalar(ids[t]);
    const bool there = id >= 0 && id < p.n_pages;
    if (!there && at < hi) b.bad = true;
    const uint32_t in_pool = there ? (uint32_t)id * p.n_k + p.kvh : 0;  // n_pages * n_k < 2^31
    const size_t row = ((size_t)in_pool << p.page_log2) +
                       (there ? at & ((1 << p.page_log2) - 1) : 0);
    const int last = scalar(there ? hi - at - 1 : 0);  // 15 or more in a full tile
    const gptr kb = scalar_base(p.k + row * B::kRowBytes);
    const gptr vb = scalar_base(p.v + row * B::kRowBytes);
    const uint32_t kr = (uint32_t)(m < last ? m : last) * B::kRowBytes;
#pragma unroll
    for (int s = 0; s < B::kLoads; ++s) {
      // past a row's end (d = 80, 96): its first bytes, which take_block drops
      const uint32_t col = 64 * s + 16 * c;
      if constexpr (B::kRowBytes % 64 == 0)
        b.k[t][s] = load_at<u32x4>(kb, kr + 16 * c + 64 * s);
      else
        b.k[t][s] = load_at<u32x4>(kb, kr + (col < (uint32_t)B::kRowBytes ? col : 0));
    }
    // past a row's end: rows of the product that are not stored
    const uint32_t vc = m * B::kCols < D ? m * B::kCols * B::kElem : 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t(&v)[B::kWords] = b.v[4 * t + e];
      const int r = 4 * c + e;
      const uint32_t o = (uint32_t)(r < last ? r : last) * B::kRowBytes + vc;
      if constexpr (B::kWords == 4) {
        const u32x4 x = load_once<u32x4>(vb, o);
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
      } else if constexpr (B::kWords == 2) {
        const u32x2 x = load_once<u32x2>(vb, o);
        v[0] = x.x, v[1] = x.y;
      } else {
        v[0] = load_once<uint32_t>(vb, o);
      }
    }
    if constexpr (E4M3) {
      b.ks[t] = load_at<uint32_t>(scalar_base(p.ks + row), 4 * c);
      b.vs[t] = load_at<uint32_t>(scalar_base(p.vs + row), 4 * c);
    }
  }
}

// One lane's state for query head l%16 of each 16 rows: its reference exponent, its
// part of the sum (keys of its quarter of the lanes), and O in kCols
// accumulators; and Q, the operand of the scores.
template <typename B>
struct State {
  float m, l;
  f32x4 o[B::kCols];
  bf16x8 q[B::kSteps];
};

// Scores of a block for 16 query heads, their maximum, and the weights (as the sum
// of two bf16, operands of the product with V): updates st.m and st.l and scales
// st.o to the new reference.
template <int D, bool E4M3>
__device__ __forceinline__ void weights(const Block<D, E4M3> &b, State<Block<D, E4M3>> &st,
                                        float scale2, int left, bf16x8 &p, bf16x8 &p2) {
  using B = Block<D, E4M3>;
  const int c = threadIdx.x % 64 / 16;
  float s[kTiles][4];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < B::kLoads; ++i) {
      u32x4 k = b.k[t][i];
      if (64 * i + 64 > B::kRowBytes && 64 * i + 16 * c >= B::kRowBytes) k = u32x4{0, 0, 0, 0};
      if constexpr (E4M3) {
        acc = mfma16x16x32(as_bf16x8(u32x4{widen<false>(k.x), widen<true>(k.x), widen<false>(k.y),
                                           widen<true>(k.y)}), st.q[2 * i], acc);
        acc = mfma16x16x32(as_bf16x8(u32x4{widen<false>(k.z), widen<true>(k.z), widen<false>(k.w),
                                           widen<true>(k.w)}), st.q[2 * i + 1], acc);
      } else {
        acc = mfma16x16x32(as_bf16x8(k), st.q[i], acc);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[t][r] = acc[r] * scale2;
      if constexpr (E4M3) s[t][r] *= pow2_of_byte(b.ks[t], r);
    }
  }
  if (left < kBlockKeys) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * t + 4 * c + r >= left) s[t][r] = -INFINITY;
  }
  if (b.bad) s[0][0] = __builtin_nanf("");
  float mx = s[0][0];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[t][r]);
  mx = fmaxf(st.m, column_max(mx));
  const float ref = mx == -INFINITY ? 0.f : mx;
  const float f = fast_exp2(st.m - ref);
  st.m = mx;
  st.l *= f;
#pragma unroll
  for (int i = 0; i < B::kCols; ++i) st.o[i] *= f;
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float w = fast_exp2(s[t][r] - ref);
      st.l += w;
      s[t][r] = w;
      if constexpr (E4M3) {
        s[t][r] *= pow2_of_byte(b.vs[t], r);
        // past the end the scale may be anything
        if (left < kBlockKeys && 16 * t + 4 * c + r >= left) s[t][r] = 0.f;
      }
    }
  // A weight as its rounding to bf16 and that of what this leaves: the matrix cores
  // have room for two products, and O is as exact as its fp32 sums.
  u32x4 hi, lo;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float *x = &s[i / 2][i % 2 * 2];
    hi[i] = pack_bf16x2(x[0], x[1]);
    lo[i] = pack_bf16x2(x[0] - __builtin_bit_cast(float, hi[i] << 16),
                        x[1] - __builtin_bit_cast(float, hi[i] & 0xFFFF0000u));
  }
  p = as_bf16x8(hi);
  p2 = as_bf16x8(lo);
}

// One block.  `left`: keys of the sequence from the block's first on (less than a
// block only in its last).
template <int D, bool E4M3, int RG>
__device__ __forceinline__ void take_block(Block<D, E4M3> &b, State<Block<D, E4M3>> (&st)[RG],
                                           float scale2, int left) {
  using B = Block<D, E4M3>;
  bf16x8 p[RG], p2[RG];
#pragma unroll
  for (int g = 0; g < RG; ++g) weights<D, E4M3>(b, st[g], scale2, left, p[g], p2[g]);
  if (left < kBlockKeys) {  // weights of 0 there; V may be anything
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (16 * (e / 4) + 4 * (int)(threadIdx.x % 64 / 16) + e % 4 >= left)
#pragma unroll
        for (int w = 0; w < B::kWords; ++w) b.v[e][w] = 0;
  }
#pragma unroll
  for (int i = 0; i < B::kCols / 2; ++i) {  // elements 2i, 2i + 1
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (E4M3)
        w[e] = i % 2 ? widen<true>(b.v[e][i / 2]) : widen<false>(b.v[e][i / 2]);
      else
        w[e] = b.v[e][i];
    }
    const bf16x8 even = as_bf16x8(u32x4{halves<false>(w[0], w[1]), halves<false>(w[2], w[3]),
                                        halves<false>(w[4], w[5]), halves<false>(w[6], w[7])});
    const bf16x8 odd = as_bf16x8(u32x4{halves<true>(w[0], w[1]), halves<true>(w[2], w[3]),
                                       halves<true>(w[4], w[5]), halves<true>(w[6], w[7])});
#pragma unroll
    for (int g = 0; g < RG; ++g) {
      f32x4 *o = st[g].o;
      o[2 * i] = mfma16x16x32(even, p[g], mfma16x16x32(even, p2[g], o[2 * i]));
      o[2 * i + 1] = mfma16x16x32(odd, p[g], mfma16x16x32(odd, p2[g], o[2 * i + 1]));
    }
  }
}

// What a workgroup leaves for the join, in the workspace: for its first (0) and
// last (1) head, of up to `rows` rows, O not divided by l [g][2][rows][D] and (m, l)
// [g][2][rows]; and, of each head that starts in its run, where its partial
// results lie if it ends past the run: `count` of them (else 0), the first in slot
// first % 2 of workgroup first / 2, the others in slot 0 of the next ones.  These
// descriptors are indexed by the head; where there are more heads than workgroups
// by the workgroup, whose last head alone can end past its run.
struct Partials {
  DecodeOpen *open;
  f32x2 *ml;
  float *o;
};
__device__ __forceinline__ Partials partials_at(void *ws, int opens, int groups, int rows) {
  Partials p;
  p.open = static_cast<DecodeOpen *>(ws);
  p.ml = reinterpret_cast<f32x2 *>(p.open + opens);
  p.o = reinterpret_cast<float *>(p.ml + (size_t)groups * 2 * rows);
  return p;
}

__device__ __forceinline__ int units_of(int len, int max_len) {
  return len <= 0 || len > max_len ? 0 : (len - 1) / kUnit + 1;
}

__device__ __forceinline__ int wave_scan(int x) {  // inclusive
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// RG: rows of 16 query heads that a workgroup serves, two where a kv head has more
// than 16, so that K and V are read once for 32 (32 ragged sequences of up to 16K
// tokens, 64 heads on 2: 85 us with 16 to a workgroup, 58 with 32).
template <int D, bool E4M3, int RG>
__global__ __launch_bounds__(kThreads, RG == 1 ? 3 : 2) void decode_kernel(const DecodeArgs a,
                                                                          int opens) {
  using B = Block<D, E4M3>;
  constexpr int kRows = 16 * RG;
  const int rep = scalar(a.n_q / a.s.n_k), row_groups = (rep + kRows - 1) / kRows;
  const int R = scalar(a.s.n_k * row_groups);  // heads, as dealt out, of a sequence
  const int b = a.s.b, G = gridDim.x, g = blockIdx.x;
  const int wave = scalar(threadIdx.x / 64);
  const int lane = threadIdx.x % 64, m = lane % 16, c = lane / 16;
  __shared__ float so[kWaves][kRows][D + 4], sm[kWaves][kRows], sl[kWaves][kRows];
  __shared__ int sums[kWaves], found[3];

  const Partials ps = partials_at(a.workspace, opens, G, kRows);
  const bool joins = a.workspace != nullptr, by_head = joins && opens != G;

  // Sequences without keys, or with more than the call allows, are shared out.
  auto write_empty = [&]() {
    for (int s = g; s < b; s += G) {
      const int len = scalar_load(a.lens, s);
      if (units_of(len, a.max_len) > 0) continue;
      uint16_t *o = static_cast<uint16_t *>(a.o) + (size_t)s * a.n_q * D;
      for (int i = threadIdx.x; i < a.n_q * D; i += kThreads) o[i] = len <= 0 ? 0 : 0x7FFF;
      if (a.lse)
        for (int i = threadIdx.x; i < a.n_q; i += kThreads)
          a.lse[(size_t)s * a.n_q + i] = len <= 0 ? -INFINITY : __builtin_nanf("");
      if (by_head)
        for (int i = threadIdx.x; i < R; i += kThreads) ps.open[(size_t)s * R + i].count = 0;
    }
  };

  // All units, and this workgroup's run [begin, end).
  const int len0 = (int)threadIdx.x < b ? a.lens[threadIdx.x] : 0;
  const int n0 = units_of(len0, a.max_len);
  int mine = n0;
  for (int s = threadIdx.x + kThreads; s < b; s += kThreads)
    mine += units_of(a.lens[s], a.max_len);
  mine = wave_scan(mine);
  if (lane == 63) sums[wave] = mine;
  __syncthreads();
  const int total = scalar(R * (sums[0] + sums[1] + sums[2] + sums[3]));
  const int quota = scalar((total + G - 1) / G);
  const long long first = (long long)g * quota;
  if (first >= total) {
    if (joins && !by_head && threadIdx.x == 0) ps.open[g].count = 0;
    write_empty();
    return;
  }
  const int begin = (int)first, end = total - begin < quota ? total : begin + quota;
  // The sequence of unit `begin`: chunks of 256 sequences, each thread one.
  int base = 0;
  for (int s0 = 0;; s0 += kThreads) {
    const int s = s0 + threadIdx.x;
    int len = len0, n = n0, x = mine;
    if (b > kThreads) {  // else the sums above are those of the one chunk
      __syncthreads();   // sums, read above or in the last turn
      if (s0 > 0) len = s < b ? a.lens[s] : 0, n = units_of(len, a.max_len);
      x = wave_scan(n);
      if (lane == 63) sums[wave] = x;
      __syncthreads();
    }
    x += base;
    for (int w = 0; w < wave; ++w) x += sums[w];
    if (begin >= R * (x - n) && begin < R * x)
      found[0] = s, found[1] = begin - R * (x - n), found[2] = len;
    base += sums[0] + sums[1] + sums[2] + sums[3];
    if (begin < R * base) break;  // some thread of this chunk has found it
    if (s0 + kThreads >= b) return;  // not reached while lens stays as it is
  }
  __syncthreads();
  int seq = scalar(found[0]);
  int len = scalar(found[2]), n = units_of(len, a.max_len);  // n: units of a head of it
  int head = scalar(found[1] / n), u = scalar(found[1] % n);

  Pages pg;
  pg.k = static_cast<const char *>(a.k_pages);
  pg.v = static_cast<const char *>(a.v_pages);
  pg.ks = a.k_scales;
  pg.vs = a.v_scales;
  pg.page_log2 = a.s.page_log2;
  pg.n_pages = a.s.n_pages;
  pg.max_pages = a.s.max_pages;
  pg.n_k = a.s.n_k;
  const float scale2 = a.scale * kLog2e;
  DecodeOpen open = {0, 0, 0, 0};

  for (int pos = begin; pos < end;) {
    const int take = n - u < end - pos ? n - u : end - pos;  // units of this head
    const int lo = u * kUnit;
    const int hi = (u + take) * kUnit < len ? (u + take) * kUnit : len;
    const int kvh = scalar(head / row_groups), grp = scalar(head % row_groups);
    const int h0 = kvh * rep + grp * kRows;  // first query head
    const int heads = rep - grp * kRows < kRows ? rep - grp * kRows : kRows;
    pg.table = a.table + (size_t)seq * a.s.max_pages;
    pg.kvh = kvh;

    // Blocks lo + (4j + wave) * kBlockKeys, one in flight per wave, the next one's
    // page numbers with it.  (A second block in flight in registers of its own
    // leaves two waves per SIMD, and the time as it is.)
    int t = lo + wave * kBlockKeys;
    Block<D, E4M3> x;
    int ids[kTiles];
    load_ids(pg, t, hi, ids);
    State<B> st[RG];
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      const int h = 16 * rg + m;
      const uint16_t *qp = static_cast<const uint16_t *>(a.q) + (long long)seq * a.q_row +
                           (size_t)(h0 + h) * D;
#pragma unroll
      for (int s = 0; s < B::kSteps; ++s) {
        const int e = E4M3 ? 64 * (s / 2) + 16 * c + 8 * (s % 2) : 32 * s + 8 * c;
        u32x4 w = {0, 0, 0, 0};
        if (h < heads && e < D) w = *reinterpret_cast<const u32x4 *>(qp + e);
        st[rg].q[s] = as_bf16x8(w);
      }
      st[rg].m = -INFINITY;
      st[rg].l = 0.f;
#pragma unroll
      for (int i = 0; i < B::kCols; ++i) st[rg].o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    while (t < hi) {
      load_block<D, E4M3>(x, pg, t, hi, ids);
      load_ids(pg, t + kUnit, hi, ids);
      take_block<D, E4M3, RG>(x, st, scale2, hi - t);
      t += kUnit;
    }

    // The four waves.
    __syncthreads();  // the last head's
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      const float l = column_sum(st[rg].l);
      if (c == 0) sm[wave][16 * rg + m] = st[rg].m, sl[wave][16 * rg + m] = l;
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
        if (B::kCols * (4 * c + r) < D) {
#pragma unroll
          for (int i = 0; i < B::kCols; i += 4)
            *reinterpret_cast<f32x4 *>(&so[wave][h][B::kCols * (4 * c + r) + i]) =
                f32x4{acc[i][r] * f, acc[i + 1][r] * f, acc[i + 2][r] * f, acc[i + 3][r] * f};
        }
    }
    __syncthreads();
    const size_t row0 = (size_t)seq * a.n_q + h0;
    const bool whole = take == n;
    const int slot = pos != begin;
    if (u == 0) {
      open = DecodeOpen{(int)row0, heads, whole ? 0 : (pos + n - 1) / quota - g + 1, 2 * g + slot};
      if (by_head && threadIdx.x == 0) ps.open[(size_t)seq * R + head] = open;
    }
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
      if (whole) {
        O *= 1.f / L;
        *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.o) + (row0 + h) * D + e) =
            u32x2{pack_bf16x2(O.x, O.y), pack_bf16x2(O.z, O.w)};
        if (e == 0 && a.lse) a.lse[row0 + h] = (mx + fast_log2(L)) * kLn2;
      } else {
        const size_t p = ((size_t)g * 2 + slot) * kRows + h;
        *reinterpret_cast<f32x4 *>(ps.o + p * D + e) = O;
        if (e == 0) ps.ml[p] = f32x2{mx, L};
      }
    }
    pos += take;
    if (pos < end) {  // the next head, of the next sequence that has keys
      u = 0;
      if (++head == R) {
        head = 0;
        n = 0;
        while (n == 0 && ++seq < b) {
          len = scalar_load(a.lens, seq);
          n = units_of(len, a.max_len);
        }
        if (n == 0) break;  // not reached while lens stays as it is
      }
    }
  }
  if (joins && !by_head && threadIdx.x == 0) ps.open[g] = open;
  write_empty();
}

// One row of one head with several partial results: these in turn over 8 C groups of
// 32 / C threads, 4 elements of d a thread, each group with a running maximum; C
// workgroups share the row's elements.
template <int D, int C>
__global__ __launch_bounds__(kThreads) void decode_join_kernel(const DecodeArgs a, int opens,
                                                               int groups, int rows) {
  constexpr int L = 32 / C, R = kThreads / L, kAtOnce = 4;
  const Partials p = partials_at(a.workspace, opens, groups, rows);
  const DecodeOpen open = p.open[blockIdx.x];
  const int h = blockIdx.y;
  if (h >= open.heads || open.count == 0) return;
  const int n = open.count;
  auto at = [&](int i) {
    return (size_t)(i ? (open.first | 1) - 1 + 2 * i : open.first) * rows + h;
  };
  const int g = threadIdx.x / L, col = blockIdx.z * (4 * L) + threadIdx.x % L * 4;
  __shared__ float so[kWaves][4 * L + 4], sm[kWaves], sl[kWaves];
  f32x4 O = {0.f, 0.f, 0.f, 0.f};
  float M = -INFINITY, l = 0.f;
  for (int i0 = g; i0 < n; i0 += kAtOnce * R) {
    f32x2 x[kAtOnce];
    f32x4 o[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = i0 + u * R < n ? i0 + u * R : i0;  // again the first: dropped below
      x[u] = p.ml[at(i)];
      o[u] = *reinterpret_cast<const f32x4 *>(p.o + at(i) * D + (col < D ? col : 0));
    }
    float mx = fmaxf(M, x[0].x);
#pragma unroll
    for (int u = 1; u < kAtOnce; ++u) mx = fmaxf(mx, x[u].x);
    const float ref = mx == -INFINITY ? 0.f : mx, f = fast_exp2(M - ref);
    M = mx;
    l *= f;
    O *= f;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      if (i0 + u * R < n) {
        const float w = fast_exp2(x[u].x - ref);
        l += w * x[u].y;
        O += w * o[u];
      }
  }
  // the groups of a wave, then the waves
  float mx = M;
#pragma unroll
  for (int x = 32; x >= L; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
  const float f = fast_exp2(M - (mx == -INFINITY ? 0.f : mx));
  l *= f;
  O *= f;
#pragma unroll
  for (int x = 32; x >= L; x >>= 1) {
    l += __shfl_xor(l, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) O[i] += __shfl_xor(O[i], x);
  }
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  if (lane < L) *reinterpret_cast<f32x4 *>(&so[wave][4 * lane]) = O;
  if (lane == 0) sm[wave] = mx, sl[wave] = l;
  __syncthreads();
  const int e = blockIdx.z * (4 * L) + threadIdx.x * 2;
  if (threadIdx.x < 2 * L && e < D) {
    M = sm[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm[w]);
    float A = 0.f, Bb = 0.f;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float fw = fast_exp2(sm[w] - (M == -INFINITY ? 0.f : M));
      A += fw * so[w][threadIdx.x * 2];
      Bb += fw * so[w][threadIdx.x * 2 + 1];
      l += fw * sl[w];
    }
    const float inv = 1.f / l;
    const size_t r = (size_t)open.row0 + h;
    static_cast<uint32_t *>(a.o)[(r * D + e) / 2] = pack_bf16x2(A * inv, Bb * inv);
    if (e == 0 && a.lse) a.lse[r] = (M + fast_log2(l)) * kLn2;
  }
}

template <int D, bool E4M3>
hipError_t decode_typed(const DecodeArgs &a, hipStream_t stream) {
  const DecodeCut s = decode_cut(a.s.b, a.n_q, a.s.n_k, D, a.max_len);
  if (s.rows == 16)
    hipLaunchKernelGGL((decode_kernel<D, E4M3, 1>), dim3(s.groups), dim3(kThreads), 0, stream, a,
                       s.opens);
  else
    hipLaunchKernelGGL((decode_kernel<D, E4M3, 2>), dim3(s.groups), dim3(kThreads), 0, stream, a,
                       s.opens);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.workspace) return e;
  const int rep = a.n_q / a.s.n_k, rows = rep < s.rows ? rep : s.rows;
  if (s.groups >= 16 * s.opens)
    hipLaunchKernelGGL((decode_join_kernel<D, 8>), dim3(s.opens, rows, 8), dim3(kThreads), 0,
                       stream, a, s.opens, s.groups, s.rows);
  else
    hipLaunchKernelGGL((decode_join_kernel<D, 1>), dim3(s.opens, rows), dim3(kThreads), 0, stream,
                       a, s.opens, s.groups, s.rows);
  return hipGetLastError();
}

template <int D>
hipError_t decode_dim(const DecodeArgs &a, hipStream_t stream) {
  return a.s.e4m3 ? decode_typed<D, true>(a, stream) : decode_typed<D, false>(a, stream);
}

}  // namespace

hipError_t launch_attn_decode(const DecodeArgs &a, hipStream_t stream) {
  switch (a.s.d) {
    case 64: return decode_dim<64>(a, stream);
    case 80: return decode_dim<80>(a, stream);
    case 96: return decode_dim<96>(a, stream);
    default: return decode_dim<128>(a, stream);
  }
}

}  // namespace basp
