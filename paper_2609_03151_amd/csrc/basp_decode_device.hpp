// basp_decode_device.hpp -- what attention of one new token loads and computes per
// block of keys, for the kernels that do so (basp_decode.hip, basp_shared.hip): the
// operands' way from the pages to the matrix cores is described at the top of the former.
#pragma once

#include "basp_device.hpp"
#include "basp_ops.hpp"

namespace basp {
namespace {

constexpr int kTiles = 2;  // of 16 keys, in a wave's block
constexpr int kBlockKeys = 16 * kTiles;
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

// What capped and biased scores (basp_span.hpp) and a first key past 0 need.
struct KeyRule {
  bool capped;
  float c1, cap2;  // of cap_r; the cap in log2 units
  int at;          // the query's position; distances are taken in whole numbers, since fp32 does
                   // not hold positions past 2^24
  int lo;          // its first key
};

// Scores of a block for 16 query heads, their maximum, and the weights (as the sum
// of two bf16, operands of the product with V): updates st.m and st.l and scales
// st.o to the new reference.
template <int D, bool E4M3, bool RULE>
__device__ __forceinline__ void weights(const Block<D, E4M3> &b, State<Block<D, E4M3>> &st,
                                        float scale2, int left, bf16x8 &p, bf16x8 &p2,
                                        const KeyRule &rule, float sl, int t0) {
  using B = Block<D, E4M3>;
  const int c = threadIdx.x % 64 / 16;
  float s[kTiles][4];
  const float away = RULE ? (float)(rule.at - (t0 + 4 * c)) : 0.f;  // the lane's first key
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
      if constexpr (RULE) {
        float x = acc[r];
        if constexpr (E4M3) x *= pow2_of_byte(b.ks[t], r);
        x = rule.capped ? fmaf(cap_r(x, rule.c1), -2.f * rule.cap2, rule.cap2) : x * scale2;
        s[t][r] = fmaf(-sl, away - (float)(16 * t + r), x);
      } else {
        s[t][r] = acc[r] * scale2;
        if constexpr (E4M3) s[t][r] *= pow2_of_byte(b.ks[t], r);
      }
    }
  }
  if constexpr (RULE) {
    if (t0 < rule.lo) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (t0 + 16 * t + 4 * c + r < rule.lo) s[t][r] = -INFINITY;
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
        if (RULE && t0 + 16 * t + 4 * c + r < rule.lo) s[t][r] = 0.f;
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
// block only in its last).  With RULE: key t0 is its first, sl the slopes (in log2 units)
// of the lane's query heads.
template <int D, bool E4M3, int RG, bool RULE = false>
__device__ __forceinline__ void take_block(Block<D, E4M3> &b, State<Block<D, E4M3>> (&st)[RG],
                                           float scale2, int left, const KeyRule &rule = {},
                                           const float *sl = nullptr, int t0 = 0) {
  using B = Block<D, E4M3>;
  bf16x8 p[RG], p2[RG];
#pragma unroll
  for (int g = 0; g < RG; ++g)
    weights<D, E4M3, RULE>(b, st[g], scale2, left, p[g], p2[g], rule, RULE ? sl[g] : 0.f, t0);
  if constexpr (RULE) {
    if (t0 < rule.lo) {  // as past the end, below
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (t0 + 16 * (e / 4) + 4 * (int)(threadIdx.x % 64 / 16) + e % 4 < rule.lo)
#pragma unroll
          for (int w = 0; w < B::kWords; ++w) b.v[e][w] = 0;
    }
  }
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

__device__ __forceinline__ int wave_scan(int x) {  // inclusive
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

}  // namespace
}  // namespace basp
