// basp_decode.hip -- attention of one new token per sequence over a paged
// key-value cache:
//   O = sum_{j < len} softmax_j(scale q . k_j) v_j,  LSE = log sum_j exp(scale q . k_j).
//
// Bound by HBM: every key and value of the cache is read once, for 4 n_q/n_k
// operations a byte of bf16 (16 on 8 query heads a kv head), which is more than
// the vector units do beside such a stream and little for the matrix cores.
//
// A workgroup takes one split of a sequence's keys for the (up to 16) query
// heads of one kv head; its four waves take blocks of 32 keys (64 in 8 bits)
// in turn, each with a running maximum, sum and O of its own, joined in LDS at
// the end.  Splits of one sequence are joined by a second kernel:
//   M = max_i m_i,  O = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i
// (scores in log2 units).
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
constexpr int kRows = 16;  // query heads of a workgroup
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

// What a wave loads of one block of keys.  W: words of V per key and lane
// before widening.
template <int D, bool E4M3>
struct Block {
  static constexpr int kElem = E4M3 ? 1 : 2;
  static constexpr int kRowBytes = D * kElem;
  static constexpr int kTiles = E4M3 ? 4 : 2;         // 16 keys each
  static constexpr int kKeys = 16 * kTiles;
  static constexpr int kLoads = (kRowBytes + 63) / 64;  // of 64 bytes per key
  static constexpr int kSteps = E4M3 ? 2 * kLoads : kLoads;
  static constexpr int kCols = D <= 64 ? 4 : 8;       // elements of d per lane of V
  static constexpr int kWords = kCols * kElem / 4;
  u32x4 k[kTiles][kLoads];
  uint32_t v[kTiles / 2][8][kWords];
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

// Page numbers of a block's tiles (tiles do not cross pages: both are
// multiples of 16).
template <typename B>
__device__ __forceinline__ void load_ids(const Pages &p, int t0, int hi, int (&id)[B::kTiles]) {
#pragma unroll
  for (int t = 0; t < B::kTiles; ++t) {
    const int at = t0 + 16 * t, pi = at >> p.page_log2;
    id[t] = -1;
    if (at < hi && pi < p.max_pages) id[t] = p.table[pi];
  }
}

template <int D, bool E4M3>
__device__ __forceinline__ void load_block(Block<D, E4M3> &b, const Pages &p, int t0, int hi,
                                           const int (&ids)[Block<D, E4M3>::kTiles]) {
  using B = Block<D, E4M3>;
  const int lane = threadIdx.x % 64, m = lane % 16, c = lane / 16;
  uint32_t ko[B::kLoads];
#pragma unroll
  for (int s = 0; s < B::kLoads; ++s) {
    const uint32_t at = 64 * s + 16 * c;
    ko[s] = at < (uint32_t)B::kRowBytes ? m * B::kRowBytes + at : kZeroOffset;
  }
  const uint32_t vo = m * B::kCols < D ? 4 * c * B::kRowBytes + m * B::kCols * B::kElem
                                       : kZeroOffset;
  b.bad = false;
#pragma unroll
  for (int t = 0; t < B::kTiles; ++t) {
    const int at = t0 + 16 * t;
    const int id = __builtin_amdgcn_readfirstlane(ids[t]);
    const bool there = id >= 0 && id < p.n_pages;
    int rows = hi - at;
    rows = rows < 0 ? 0 : rows > 16 ? 16 : rows;
    if (!there && rows > 0) b.bad = true;
    if (!there) rows = 0;
    const size_t row = (((size_t)(there ? id : 0) * p.n_k + p.kvh) << p.page_log2) +
                       (at & ((1 << p.page_log2) - 1));
    const rsrc_t kr = make_rsrc(p.k + row * B::kRowBytes, rows * B::kRowBytes);
    const rsrc_t vr = make_rsrc(p.v + row * B::kRowBytes, rows * B::kRowBytes);
#pragma unroll
    for (int s = 0; s < B::kLoads; ++s) b.k[t][s] = buf_load16(kr, ko[s]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t(&v)[B::kWords] = b.v[t / 2][4 * (t % 2) + e];
      const uint32_t o = vo + e * B::kRowBytes;
      if constexpr (B::kWords == 4) {
        const u32x4 x = buf_load16(vr, o);
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
      } else if constexpr (B::kWords == 2) {
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(vr, o, 0, 0));
        v[0] = x.x, v[1] = x.y;
      } else {
        v[0] = __builtin_amdgcn_raw_buffer_load_b32(vr, o, 0, 0);
      }
    }
    if constexpr (E4M3) {
      const uint32_t bytes = rows > 0 ? 16 : 0;
      b.ks[t] = __builtin_amdgcn_raw_buffer_load_b32(make_rsrc(p.ks + row, bytes), 4 * c, 0, 0);
      b.vs[t] = __builtin_amdgcn_raw_buffer_load_b32(make_rsrc(p.vs + row, bytes), 4 * c, 0, 0);
    }
  }
}

// One lane's state: query head l%16, its reference exponent, its part of the
// sum (keys of its quarter of the lanes), and O in kCols accumulators.
template <typename B>
struct State {
  float m, l;
  f32x4 o[B::kCols];
};

// Maximum, weights and O of one block.  `left`: keys of the sequence from the
// block's first on (less than a block only in its last).
template <int D, bool E4M3>
__device__ __forceinline__ void take_block(const Block<D, E4M3> &b, State<Block<D, E4M3>> &st,
                                           const bf16x8 (&q)[Block<D, E4M3>::kSteps], float scale2,
                                           int left) {
  using B = Block<D, E4M3>;
  const int c = threadIdx.x % 64 / 16;
  float s[B::kTiles][4];
#pragma unroll
  for (int t = 0; t < B::kTiles; ++t) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < B::kLoads; ++i) {
      const u32x4 k = b.k[t][i];
      if constexpr (E4M3) {
        acc = mfma16x16x32(as_bf16x8(u32x4{widen<false>(k.x), widen<true>(k.x), widen<false>(k.y),
                                           widen<true>(k.y)}), q[2 * i], acc);
        acc = mfma16x16x32(as_bf16x8(u32x4{widen<false>(k.z), widen<true>(k.z), widen<false>(k.w),
                                           widen<true>(k.w)}), q[2 * i + 1], acc);
      } else {
        acc = mfma16x16x32(as_bf16x8(k), q[i], acc);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[t][r] = acc[r] * scale2;
      if constexpr (E4M3) s[t][r] *= pow2_of_byte(b.ks[t], r);
    }
  }
  if (left < B::kKeys) {
#pragma unroll
    for (int t = 0; t < B::kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * t + 4 * c + r >= left) s[t][r] = -INFINITY;
  }
  if (b.bad) s[0][0] = __builtin_nanf("");
  float mx = s[0][0];
#pragma unroll
  for (int t = 0; t < B::kTiles; ++t)
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
  for (int t = 0; t < B::kTiles; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float p = fast_exp2(s[t][r] - ref);
      st.l += p;
      s[t][r] = p;
      if constexpr (E4M3) {
        s[t][r] *= pow2_of_byte(b.vs[t], r);
        // past the end the scale may be anything
        if (left < B::kKeys && 16 * t + 4 * c + r >= left) s[t][r] = 0.f;
      }
    }
#pragma unroll
  for (int g = 0; g < B::kTiles / 2; ++g) {
    // P rounded to bf16 for the matrix cores; its sum above is of the unrounded
    const bf16x8 p = as_bf16x8(u32x4{pack_bf16x2(s[2 * g][0], s[2 * g][1]),
                                     pack_bf16x2(s[2 * g][2], s[2 * g][3]),
                                     pack_bf16x2(s[2 * g + 1][0], s[2 * g + 1][1]),
                                     pack_bf16x2(s[2 * g + 1][2], s[2 * g + 1][3])});
#pragma unroll
    for (int i = 0; i < B::kCols / 2; ++i) {  // elements 2i, 2i + 1
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (E4M3)
          w[e] = i % 2 ? widen<true>(b.v[g][e][i / 2]) : widen<false>(b.v[g][e][i / 2]);
        else
          w[e] = b.v[g][e][i];
      }
      st.o[2 * i] = mfma16x16x32(as_bf16x8(u32x4{halves<false>(w[0], w[1]), halves<false>(w[2], w[3]),
                                                 halves<false>(w[4], w[5]), halves<false>(w[6], w[7])}),
                                 p, st.o[2 * i]);
      st.o[2 * i + 1] = mfma16x16x32(as_bf16x8(u32x4{halves<true>(w[0], w[1]), halves<true>(w[2], w[3]),
                                                     halves<true>(w[4], w[5]), halves<true>(w[6], w[7])}),
                                     p, st.o[2 * i + 1]);
    }
  }
}

// Partial results of split i of (sequence, query head) r, n splits a row:
// o [rows][n][d] (not divided by l), then (m, l) [rows][n].
struct Partials {
  float *o;
  f32x2 *ml;
};
__device__ __forceinline__ Partials partials_at(void *ws, size_t rows, int n, int d) {
  Partials p;
  p.o = static_cast<float *>(ws);
  p.ml = reinterpret_cast<f32x2 *>(p.o + rows * n * d);
  return p;
}

template <int D, bool E4M3>
__global__ __launch_bounds__(kThreads, 2) void decode_split_kernel(const DecodeArgs a,
                                                                   const DecodeSplit sp) {
  using B = Block<D, E4M3>;
  const int rep = a.n_q / a.s.n_k, groups = (rep + kRows - 1) / kRows;
  int at = blockIdx.x;
  const int split = at % sp.splits;
  at /= sp.splits;
  const int grp = at % groups;
  at /= groups;
  const int kvh = at % a.s.n_k, seq = at / a.s.n_k;
  const int h0 = kvh * rep + grp * kRows;  // first query head
  const int heads = rep - grp * kRows < kRows ? rep - grp * kRows : kRows;
  const int len = a.lens[seq], lo = split * sp.keys;
  const size_t row0 = (size_t)seq * a.n_q + h0;
  uint16_t *o = static_cast<uint16_t *>(a.o) + row0 * D;
  if (len <= 0 || len > a.max_len) {  // no keys, or more than the call allows
    if (split > 0) return;
    for (int i = threadIdx.x; i < heads * D; i += kThreads) o[i] = len <= 0 ? 0 : 0x7FFF;
    if (threadIdx.x < heads && a.lse)
      a.lse[row0 + threadIdx.x] = len <= 0 ? -INFINITY : __builtin_nanf("");
    return;
  }
  if (lo >= len) return;
  const int hi = len - lo < sp.keys ? len : lo + sp.keys;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x % 64, m = lane % 16, c = lane / 16;

  Pages pg;
  pg.k = static_cast<const char *>(a.k_pages);
  pg.v = static_cast<const char *>(a.v_pages);
  pg.ks = a.k_scales;
  pg.vs = a.v_scales;
  pg.table = a.table + (size_t)seq * a.s.max_pages;
  pg.page_log2 = a.s.page_log2;
  pg.n_pages = a.s.n_pages;
  pg.max_pages = a.s.max_pages;
  pg.n_k = a.s.n_k;
  pg.kvh = kvh;

  bf16x8 q[B::kSteps];
  const uint16_t *qp = static_cast<const uint16_t *>(a.q) + (long long)seq * a.q_row +
                       (size_t)(h0 + m) * D;
#pragma unroll
  for (int s = 0; s < B::kSteps; ++s) {
    const int e = E4M3 ? 64 * (s / 2) + 16 * c + 8 * (s % 2) : 32 * s + 8 * c;
    u32x4 w = {0, 0, 0, 0};
    if (m < heads && e < D) w = *reinterpret_cast<const u32x4 *>(qp + e);
    q[s] = as_bf16x8(w);
  }
  const float scale2 = a.scale * kLog2e;

  State<B> st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int i = 0; i < B::kCols; ++i) st.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Blocks lo + (4j + wave) * kKeys: the next one's loads are in flight while
  // one is taken, and the one after's page numbers.
  constexpr int kStep = kWaves * B::kKeys;
  int t = lo + wave * B::kKeys;
  Block<D, E4M3> x, y;
  int ids[B::kTiles];
  load_ids<B>(pg, t, hi, ids);
  load_block<D, E4M3>(x, pg, t, hi, ids);
  load_ids<B>(pg, t + kStep, hi, ids);
  while (t < hi) {
    load_block<D, E4M3>(y, pg, t + kStep, hi, ids);
    load_ids<B>(pg, t + 2 * kStep, hi, ids);
    take_block<D, E4M3>(x, st, q, scale2, hi - t);
    t += kStep;
    if (t >= hi) break;
    load_block<D, E4M3>(x, pg, t + kStep, hi, ids);
    load_ids<B>(pg, t + 2 * kStep, hi, ids);
    take_block<D, E4M3>(y, st, q, scale2, hi - t);
    t += kStep;
  }
  st.l = column_sum(st.l);

  // The four waves.
  __shared__ float so[kWaves][kRows][D + 4], sm[kWaves][kRows], sl[kWaves][kRows];
  if (c == 0) sm[wave][m] = st.m, sl[wave][m] = st.l;
  __syncthreads();
  float M = sm[0][m];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm[w][m]);
  const float f = fast_exp2(st.m - (M == -INFINITY ? 0.f : M));
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (B::kCols * (4 * c + r) < D) {
#pragma unroll
      for (int i = 0; i < B::kCols; i += 4)
        *reinterpret_cast<f32x4 *>(&so[wave][m][B::kCols * (4 * c + r) + i]) =
            f32x4{st.o[i][r] * f, st.o[i + 1][r] * f, st.o[i + 2][r] * f, st.o[i + 3][r] * f};
    }
  __syncthreads();
  const bool whole = len <= sp.keys;  // the sequence's only split
  const Partials ps = partials_at(a.workspace, (size_t)a.s.b * a.n_q, sp.splits, D);
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
      *reinterpret_cast<u32x2 *>(o + h * D + e) = u32x2{pack_bf16x2(O.x, O.y), pack_bf16x2(O.z, O.w)};
      if (e == 0 && a.lse) a.lse[row0 + h] = (mx + fast_log2(L)) * kLn2;
    } else {
      const size_t p = (row0 + h) * sp.splits + split;
      *reinterpret_cast<f32x4 *>(ps.o + p * D + e) = O;
      if (e == 0) ps.ml[p] = f32x2{mx, L};
    }
  }
}

// One (sequence, query head) with several splits: its splits in turn over 8
// groups of 32 threads, 4 elements of d a thread.
template <int D>
__global__ __launch_bounds__(kThreads) void decode_join_kernel(const DecodeArgs a,
                                                               const DecodeSplit sp) {
  const int r = blockIdx.x;
  const int len = a.lens[r / a.n_q];
  if (len <= sp.keys || len > a.max_len) return;  // written by the split itself
  const int n = (len + sp.keys - 1) / sp.keys;
  const Partials p = partials_at(a.workspace, gridDim.x, sp.splits, D);
  const f32x2 *ml = p.ml + (size_t)r * sp.splits;
  const float *po = p.o + (size_t)r * sp.splits * D;
  const int g = threadIdx.x / 32, e = threadIdx.x % 32 * 4;
  __shared__ float so[8][D + 4], sl[8], sm[kWaves];
  float M = -INFINITY;
  for (int i = threadIdx.x; i < n; i += kThreads) M = fmaxf(M, ml[i].x);
#pragma unroll
  for (int x = 32; x; x >>= 1) M = fmaxf(M, __shfl_xor(M, x));
  if (threadIdx.x % 64 == 0) sm[threadIdx.x / 64] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm[w]);
  const float ref = M == -INFINITY ? 0.f : M;
  f32x4 O = {0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
#pragma unroll 4
  for (int i = g; i < n; i += 8) {
    const f32x2 x = ml[i];
    const float f = fast_exp2(x.x - ref);
    L += f * x.y;
    if (e < D) O += f * *reinterpret_cast<const f32x4 *>(po + (size_t)i * D + e);
  }
  if (e < D) *reinterpret_cast<f32x4 *>(&so[g][e]) = O;
  if (e == 0) sl[g] = L;
  __syncthreads();
  if (threadIdx.x < D / 2) {
    const int x = threadIdx.x * 2;
    float A = 0.f, Bb = 0.f;
    L = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) A += so[i][x], Bb += so[i][x + 1], L += sl[i];
    const float inv = 1.f / L;
    static_cast<uint32_t *>(a.o)[(size_t)r * (D / 2) + threadIdx.x] = pack_bf16x2(A * inv, Bb * inv);
    if (threadIdx.x == 0 && a.lse) a.lse[r] = (M + fast_log2(L)) * kLn2;
  }
}

template <int D>
hipError_t decode_dim(const DecodeArgs &a, hipStream_t stream) {
  const DecodeSplit sp = decode_split(a.s.b, a.n_q, a.s.n_k, a.max_len);
  const int rep = a.n_q / a.s.n_k;
  const unsigned blocks =
      (unsigned)a.s.b * a.s.n_k * ((rep + kRows - 1) / kRows) * (unsigned)sp.splits;
  if (a.s.e4m3)
    hipLaunchKernelGGL((decode_split_kernel<D, true>), dim3(blocks), dim3(kThreads), 0, stream, a,
                       sp);
  else
    hipLaunchKernelGGL((decode_split_kernel<D, false>), dim3(blocks), dim3(kThreads), 0, stream, a,
                       sp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.splits == 1) return e;
  hipLaunchKernelGGL((decode_join_kernel<D>), dim3((unsigned)a.s.b * a.n_q), dim3(kThreads), 0,
                     stream, a, sp);
  return hipGetLastError();
}

}  // namespace

DecodeSplit decode_split(int b, int n_q, int n_k, int max_len) {
  const int rep = n_q / n_k;
  const long long rows = (long long)b * n_k * ((rep + kRows - 1) / kRows);
  const long long want = (4096 + rows - 1) / rows;  // splits
  DecodeSplit sp;
  sp.keys = (int)((max_len + want * 256 - 1) / (want * 256)) * 256;
  sp.splits = (max_len + sp.keys - 1) / sp.keys;
  return sp;
}

size_t decode_workspace_bytes(int b, int n_q, int n_k, int d, int max_len) {
  const DecodeSplit sp = decode_split(b, n_q, n_k, max_len);
  return sp.splits == 1 ? 0 : (size_t)b * n_q * sp.splits * (d + 2) * sizeof(float);
}

hipError_t launch_attn_decode(const DecodeArgs &a, hipStream_t stream) {
  switch (a.s.d) {
    case 64: return decode_dim<64>(a, stream);
    case 80: return decode_dim<80>(a, stream);
    case 96: return decode_dim<96>(a, stream);
    default: return decode_dim<128>(a, stream);
  }
}

}  // namespace basp
