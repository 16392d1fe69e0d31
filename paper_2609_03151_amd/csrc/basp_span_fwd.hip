// basp_span_fwd.hip -- forward of attention over spans.
//
// Every query row sees one run of keys [lo, hi); scores may be capped by a
// tanh and biased by distance (basp_span.hpp).  Bound by the matrix cores
// (4 d operations a seen pair) and, with a cap, by the vector units, which form
// three exponentials or reciprocals a score instead of one.  On MI355X: one document of
// 32K tokens with a cap, 4 heads on 1 of 128, 1155 us, 950 TFLOP/s (a large matrix product
// reaches 1600); 16K tokens in documents of some 2K with a bias, 8 heads on 2, 172 us, 517
// TFLOP/s, the ends of uneven workgroups; no rule, 16K, 8 heads on 2, 488 us.
//
// gfx950 mapping, as the causal forward's: a workgroup owns 32 R query rows of one
// head, its waves R row groups times P key parts; S^T = K Q^T
// and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16, with Q in registers, P
// straight from the score accumulator, and K and V copied HBM -> LDS into a
// ring of stages.  A lane holds one row's scores of 16 keys per 32.
//
// Masks cost what lies on their edges: the workgroup visits the tiles between
// its rows' least lo and largest hi, a wave skips tiles that none of its 32 rows sees,
// and only where some row sees some keys of a tile are its scores masked one by one,
// in place behind one branch: two forms of a whole tile would fill the registers.
#include <math.h>

#include <type_traits>

#include "basp_span_device.hpp"

namespace basp {
namespace {

constexpr int kMaxWaves = 8;
constexpr float kRescaleSlack = 8.f;  // log2 headroom before the reference max moves
// A lane's sum of a tile's P past which the pipelined loop moves the reference.
constexpr float kFollowSum = 65536.f;
constexpr int kFewKeys = 16;
// With a fixed reference, the sums of a row's P between which its products with V stay
// in fp32's range, since they are at most the sum times the largest |V| (2^104 / 2^24),
// and those that come out 0 are less than 2^-86 a key.
constexpr float kLowSum = 0x1p-40f, kHighSum = 0x1p24f;
constexpr int kSchedMfma = 0x008;
constexpr int kSchedDsRead = 0x100;

// WAVES waves: RG row groups of 32 query rows times WAVES / RG parts of KEYS keys each.
template <int D, int WAVES, int RG, int KEYS>
struct Cfg {
  static constexpr int R = RG, P = WAVES / R, THREADS = 64 * WAVES;
  static constexpr int DC = HeadDim<D>::DC;
  static constexpr int LW = HeadDim<D>::LW;
  static constexpr int BM = 32 * R;               // query rows per workgroup
  static constexpr int KM = KEYS / 32;            // 32-key blocks per wave and tile
  static constexpr int BN = 32 * KM * P;          // keys per tile
  static constexpr int TILE_BYTES = BN * LW * 2;
  // 128 KB of ring for 8 waves, one workgroup a CU; 64 KB for 4, two of them.
  static constexpr int STAGES = 16384 * WAVES >= 8 * TILE_BYTES ? 4 : 2;
  static constexpr int LDS_BYTES = STAGES * 2 * TILE_BYTES;
  static constexpr int NS = D / 16;               // 16-deep steps over the head dim
  static constexpr int NE = DC / 32;              // 32-wide head-dim subtiles of O
  static constexpr int CPR = LW / 8;              // 16-byte chunks per LDS row
  static constexpr int DMA_PER_WAVE = BN * CPR / THREADS;
  static constexpr int PART_BYTES = NE * 4 * 1024 + 768;
  static_assert((P - 1) * R * PART_BYTES <= LDS_BYTES, "the merge area fits the ring");
};

// The key parts of a row group brought together: parts 1 .. P-1 put their
// reference, row sum and O in LDS (every copy landed, nothing left to read in the
// ring), part 0 takes them into its own in order.  True in part 0.
template <class C>
__device__ __forceinline__ bool merge_parts(unsigned char *smem, int rg, int part, int lane,
                                            float &m_ref, float &l_tot, float &l_fix,
                                            f32x16 (&oacc)[C::NE]) {
  auto area = [&](int p) __attribute__((always_inline)) {
    return smem + ((p - 1) * C::R + rg) * C::PART_BYTES;
  };
  constexpr int kScalars = C::NE * 4 * 1024;
  __syncthreads();
  if (part > 0) {
    unsigned char *a = area(part);
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(a + (n * 4 + g) * 1024 + 16 * lane) =
            f32x4{oacc[n][4 * g], oacc[n][4 * g + 1], oacc[n][4 * g + 2], oacc[n][4 * g + 3]};
    *reinterpret_cast<float *>(a + kScalars + 4 * lane) = m_ref;
    *reinterpret_cast<float *>(a + kScalars + 256 + 4 * lane) = l_tot;
    *reinterpret_cast<float *>(a + kScalars + 512 + 4 * lane) = l_fix;
  }
  __syncthreads();
  if (part > 0) return false;
  float m_all = m_ref, wt[C::P];
  wt[0] = m_ref;
#pragma unroll
  for (int p = 1; p < C::P; ++p) {
    wt[p] = *reinterpret_cast<const float *>(area(p) + kScalars + 4 * lane);
    m_all = fmaxf(m_all, wt[p]);
  }
#pragma unroll
  for (int p = 0; p < C::P; ++p) wt[p] = wt[p] == -INFINITY ? 0.f : fast_exp2(wt[p] - m_all);
  m_ref = m_all;
  // A part that saw no key of the row holds zeros; one whose V had infinities
  // or NaN must not meet a weight of 0 only for that.
  l_tot *= wt[0];
  l_fix *= wt[0];
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[n][r] *= wt[0];
#pragma unroll
  for (int p = 1; p < C::P; ++p) {
    l_tot = fmaf(wt[p], *reinterpret_cast<const float *>(area(p) + kScalars + 256 + 4 * lane),
                 l_tot);
    l_fix = fmaf(wt[p], *reinterpret_cast<const float *>(area(p) + kScalars + 512 + 4 * lane),
                 l_fix);
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 z =
            *reinterpret_cast<const f32x4 *>(area(p) + (n * 4 + g) * 1024 + 16 * lane);
#pragma unroll
        for (int y = 0; y < 4; ++y) oacc[n][4 * g + y] = fmaf(wt[p], z[y], oacc[n][4 * g + y]);
      }
  }
  return true;
}

// What the workgroup and this lane work on: one head's rows q0 .. q0 + BM - 1, the
// lane's row (with lane l ^ 32) and its rule.
template <class C>
struct Work {
  int beta, h, wrow0, row, lo, hi;
  int t0, nt;            // the tiles some row sees
  SpanHull hull;         // of the wave's rows
  float sl, c, rc, c1, cap2;
  bool fixed;            // the reference stands still (kSpanFixedCap)
  bool stays;            // this row's, where not all rows' do
  float m_ref, l_run;
  // With a fixed reference, where some row of the wave sees few keys (`few`): what rounding
  // P to bf16 on edges added to the row's sum.  Its largest P is not 1, and O is divided
  // by the sum of what it was formed from (one key: O is that key's V).  With more keys the
  // roundings even out (3 x 1537 rows of 7 heads in documents of some 300 tokens: 24.9 us
  // on every edge, 23.7 with `few`, 22.7 without; the small calls' kernel the same).
  float l_fix;
  bool few;
  u32x4 rk, rv;
  uint32_t k_row_bytes, v_row_bytes;

  // First key of the wave in tile u.
  __device__ __forceinline__ int first_key(int u, int part) const {
    return (t0 + u) * C::BN + 32 * C::KM * part;
  }
  __device__ __forceinline__ bool none(int u, int part) const {
    return hull.none(first_key(u, part), 32 * C::KM);
  }
  // Some row sees only some of the keys, or the bias changes its sign among them.
  template <bool BIAS>
  __device__ __forceinline__ bool edge(int u, int part) const {
    const int j0 = first_key(u, part), n = 32 * C::KM;
    return !hull.full(j0, n) || (BIAS && j0 + n - 1 > wrow0 && j0 < wrow0 + 31);
  }
  // Scores of the keys from j0 on (32 of them) of an edge: the bias goes into them,
  // and what the row does not see becomes -inf.
  template <bool BIAS>
  __device__ __forceinline__ void fix_scores(f32x16 &sc, int jl) const {
    asm volatile("" ::: "memory");
    const float ahead = (float)(row - jl);
    const int past = jl - lo;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int jo = 8 * (r >> 2) + (r & 3);
      const bool vis = (uint32_t)(past + jo) < (uint32_t)(hi - lo);
      const float x = BIAS ? fmaf(-sl * rc, fabsf(ahead - (float)jo), sc[r]) : sc[r];
      sc[r] = vis ? x : -INFINITY;
    }
    asm volatile("" ::: "memory");
  }
};

template <class C, int D, bool CAP, bool BIAS>
__device__ __forceinline__ void enter(Work<C> &wk, bf16x8 (&qf)[C::NS], const SpanArgs &a,
                                      int heads_total, int qtiles, int (&hulls)[2][kMaxWaves]) {
  const int S = a.S, Hl = a.Hl, lane = threadIdx.x & 63, hh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int L = blockIdx.x, qt = qtiles - 1 - L / heads_total, hb = L % heads_total;
  wk.beta = hb / Hl, wk.h = hb % Hl;
  const int kvh = wk.h / (Hl / a.Hkl), q0 = qt * C::BM;
  wk.wrow0 = q0 + 32 * (w % C::R);
  wk.row = wk.wrow0 + (lane & 31);
  const uint32_t q_row_bytes = a.q.row_elems * 2;
  wk.k_row_bytes = a.k.row_elems * 2;
  wk.v_row_bytes = a.v.row_elems * 2;
  const size_t first = (size_t)wk.beta * S;
  const rsrc_t rq = make_rsrc(a.q.p + (first + q0) * a.q.row_elems + (size_t)wk.h * D,
                              (uint32_t)(S - q0) * q_row_bytes);
  wk.rk = make_rsrc_words(a.k.p + first * a.k.row_elems + (size_t)kvh * D,
                          (uint32_t)S * wk.k_row_bytes);
  wk.rv = make_rsrc_words(a.v.p + first * a.v.row_elems + (size_t)kvh * D,
                          (uint32_t)S * wk.v_row_bytes);
#pragma unroll
  for (int s = 0; s < C::NS; ++s)
    qf[s] = as_bf16x8(
        buf_load16(rq, (uint32_t)(wk.row - q0) * q_row_bytes + (2 * s + hh) * 16));
  wk.lo = wk.hi = 0;
  if (wk.row < S) span_of(a.spans, wk.beta, S, wk.row, wk.lo, wk.hi);
  wk.sl = BIAS ? a.slopes[wk.h] * kSpanLog2e : 0.f;  // in log2 units
  wk.hull = wave_hull(hull_of(wk.lo, wk.hi, wk.row < S));
  if (lane == 0) hulls[0][w] = wk.hull.any_lo, hulls[1][w] = wk.hull.any_hi;
  wait_vmcnt<0>();  // retire the tracked loads before untracked copies start
  __syncthreads();
  int lo = hulls[0][0], hi = hulls[1][0];
#pragma unroll
  for (int i = 1; i < C::R; ++i) {
    lo = min(lo, hulls[0][i]);
    hi = max(hi, hulls[1][i]);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  wk.t0 = lo < hi ? lo / C::BN : 0;
  wk.nt = lo < hi ? (hi + C::BN - 1) / C::BN - wk.t0 : 0;
  wk.c = a.scale * kSpanLog2e;
  wk.rc = 1.f / wk.c;
  wk.c1 = CAP ? 2.f * wk.c / a.cap : 0.f;
  wk.cap2 = CAP ? a.cap * kSpanLog2e : 0.f;
  wk.fixed = CAP && a.cap <= kSpanFixedCap;
  wk.few = wk.fixed && __builtin_amdgcn_ballot_w64(wk.hi > wk.lo && wk.hi - wk.lo <= kFewKeys) != 0;
  wk.l_run = wk.l_fix = 0.f;
  wk.stays = false;
  wk.m_ref = -INFINITY;
  if (wk.fixed) {  // the largest bias of the row, at its nearest or farthest key
    const int near = wk.row < wk.lo ? wk.lo - wk.row : wk.row >= wk.hi ? wk.row - wk.hi + 1 : 0;
    const int far = max(abs(wk.row - wk.lo), abs(wk.row - wk.hi + 1));
    wk.m_ref = BIAS && wk.hi > wk.lo ? fmaxf(-wk.sl * (float)near, -wk.sl * (float)far) : 0.f;
  }
}

// O and LSE of the lane's row.  oacc[n][r] = O^T[e = 32n + 8(r/4) + 4hh + r%4][row],
// not divided by the row's sum.
template <class C, int D>
__device__ __forceinline__ void leave(const Work<C> &wk, const SpanArgs &a, uint16_t *o,
                                      float *lse, float l_tot, float l_fix,
                                      const f32x16 (&oacc)[C::NE]) {
  if (wk.row >= a.S) return;
  const int hh = (threadIdx.x & 63) >> 5;
  const bool empty = wk.hi <= wk.lo;
  const float inv = empty ? 0.f : 1.f / (l_tot + l_fix);
  uint16_t *ob = o + (((size_t)wk.beta * a.S + wk.row) * a.Hl + wk.h) * D;
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (32 * n + 8 * g >= D) continue;  // padding columns
      u32x2 val = {pack_bf16x2(oacc[n][4 * g] * inv, oacc[n][4 * g + 1] * inv),
                   pack_bf16x2(oacc[n][4 * g + 2] * inv, oacc[n][4 * g + 3] * inv)};
      if (empty) val = u32x2{0, 0};
      *reinterpret_cast<u32x2 *>(ob + 32 * n + 8 * g + 4 * hh) = val;
    }
  if (hh == 0)
    lse[((size_t)wk.beta * a.Hl + wk.h) * a.S + wk.row] =
        empty ? -INFINITY : (wk.m_ref + fast_log2(l_tot)) * kSpanLn2;
}

template <int NE>
__device__ __forceinline__ void clear(f32x16 (&acc)[NE]) {
#pragma unroll
  for (int n = 0; n < NE; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[n][r] = 0.f;
}
template <int NE>
__device__ __forceinline__ bool finite(const f32x16 (&acc)[NE], float z) {
#pragma unroll
  for (int n = 0; n < NE; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = fmaf(0.f, acc[n][r], z);
  return z == 0.f;
}

// Maximum `mx` of new scores (log2 units) against the row's reference.
template <class C>
__device__ __forceinline__ void move_reference(Work<C> &wk, f32x16 (&oacc)[C::NE], float mx) {
  const bool grow = mx > wk.m_ref + kRescaleSlack;
  if (__builtin_amdgcn_ballot_w64(grow)) {  // wave-uniform, rare after the first tiles
    asm volatile("" ::: "memory");
    const float alpha = grow ? fast_exp2(wk.m_ref - mx) : 1.f;
    wk.m_ref = grow ? mx : wk.m_ref;
    wk.l_run *= alpha;
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[n][r] *= alpha;
  }
}

__device__ __forceinline__ u32x4 pack8(const f32x16 &x, int b8) {
  return u32x4{pack_bf16x2(x[b8 + 0], x[b8 + 1]), pack_bf16x2(x[b8 + 2], x[b8 + 3]),
               pack_bf16x2(x[b8 + 4], x[b8 + 5]), pack_bf16x2(x[b8 + 6], x[b8 + 7])};
}

// Sum of the eight bf16 of an operand.
__device__ __forceinline__ float sum8(u32x4 x) {
  float s = 0.f;
#pragma unroll
  for (int y = 0; y < 4; ++y)
    s += __builtin_bit_cast(float, x[y] << 16) + __builtin_bit_cast(float, x[y] & 0xFFFF0000u);
  return s;
}

// LDS offsets of the lane's operand reads.
template <class C, int D>
struct Offsets {
  using T = LdsTile<C::LW>;
  int k[C::NS], v[C::NE][2];
  __device__ __forceinline__ Offsets(int part) {
    const int lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5;
    const int part_off = part * 32 * C::KM * T::ROW_BYTES;
#pragma unroll
    for (int s = 0; s < C::NS; ++s) {
      k[s] = T::off(l32, 2 * s + hh) + part_off;
      asm volatile("" : "+v"(k[s]));
    }
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        v[n][x] = C::STAGES * C::TILE_BYTES + part_off +
                  tr_piece_off<C::LW>(4 * hh + 8 * x, 32 * n + 16 * ((lane >> 4) & 1), lane);
        asm volatile("" : "+v"(v[n][x]));
      }
  }
};

// Tile u's K and V of the workgroup into stage u % STAGES.
template <class C, int D>
struct Copies {
  uint32_t gk[C::DMA_PER_WAVE], gv[C::DMA_PER_WAVE], base;
  __device__ __forceinline__ Copies(const Work<C> &wk, const void *smem) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < C::DMA_PER_WAVE; ++i) {
      const int pos = (w * C::DMA_PER_WAVE + i) * 64 + lane;
      gk[i] = dma_src_off<C::LW, D>(pos, wk.k_row_bytes);
      gv[i] = dma_src_off<C::LW, D>(pos, wk.v_row_bytes);
    }
    base = lds_addr_of(smem) + w * C::DMA_PER_WAVE * 1024;
  }
  __device__ __forceinline__ void load_k(const Work<C> &wk, int u) const {
    const uint32_t ks = base + (u % C::STAGES) * C::TILE_BYTES;
    const uint32_t kb = (uint32_t)((wk.t0 + u) * C::BN) * wk.k_row_bytes;
#pragma unroll
    for (int i = 0; i < C::DMA_PER_WAVE; ++i) copy16_to_lds(wk.rk, kb + gk[i], ks + i * 1024);
  }
  __device__ __forceinline__ void load_v(const Work<C> &wk, int u) const {
    const uint32_t vs = base + (C::STAGES + u % C::STAGES) * C::TILE_BYTES;
    const uint32_t vb = (uint32_t)((wk.t0 + u) * C::BN) * wk.v_row_bytes;
#pragma unroll
    for (int i = 0; i < C::DMA_PER_WAVE; ++i) copy16_to_lds(wk.rv, vb + gv[i], vs + i * 1024);
  }
  __device__ __forceinline__ void load(const Work<C> &wk, int u) const {
    load_k(wk, u);
    load_v(wk, u);
  }
};

// One tile by itself: scores, reference, exponentials, P V, 32 keys at a time.  CAREFUL: V
// holds infinities or NaN somewhere, which must not reach a row through a weight of 0.
template <class C, int D, bool CAP, bool BIAS, bool CAREFUL>
__device__ __forceinline__ void one_tile(Work<C> &wk, const Offsets<C, D> &off,
                                         const bf16x8 (&qf)[C::NS], f32x16 (&oacc)[C::NE],
                                         const unsigned char *Ks, int u, int part) {
  using T = LdsTile<C::LW>;
  const int hh = (threadIdx.x & 63) >> 5;
  const bool edge = wk.template edge<BIAS>(u, part);
  const int j0 = wk.first_key(u, part);
#pragma unroll
  for (int m = 0; m < C::KM; ++m) {
    f32x16 sc;
    wave_priority<1>();
#pragma unroll
    for (int s = 0; s < C::NS; ++s) {
      const bf16x8 x = *reinterpret_cast<const bf16x8 *>(Ks + off.k[s] + m * 32 * T::ROW_BYTES);
      sc = mfma32x32x16(x, qf[s], s == 0 ? f32x16{} : sc);
    }
    wave_priority<0>();
    // sc[r] = (q . k) of key jl + 8(r/4) + r%4 for this lane's row
    const int jl = j0 + 32 * m + 4 * hh;
    const float slp = edge ? 0.f : j0 + 32 * m > wk.wrow0 ? -wk.sl : wk.sl;
    const float base = BIAS ? -slp * (float)(wk.row - jl) : 0.f;
    u32x4 seen[2] = {};
    if (CAREFUL) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if ((uint32_t)(jl + 8 * (r >> 2) + (r & 3) - wk.lo) < (uint32_t)(wk.hi - wk.lo))
          seen[r / 8][r % 8 / 2] |= r % 2 ? 0x3F800000u : 0x3F80u;
    }
    if constexpr (CAP) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = fmaf(cap_r(sc[r], wk.c1), -2.f * wk.cap2, wk.cap2) * wk.rc;
    }
    if (edge) wk.template fix_scores<BIAS>(sc, jl);  // wave-uniform
#pragma unroll
    for (int r = 0; r < 16; ++r)
      sc[r] = fmaf(sc[r], wk.c, BIAS ? fmaf(slp, (float)(8 * (r >> 2) + (r & 3)), base) : base);
    if (!wk.fixed) {
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
      if (CAP && CAREFUL && wk.stays) mx = -INFINITY;
      move_reference<C>(wk, oacc, pair_max(mx));
    }
    // A row of which no key has come yet: every score is -inf, P = 0.
    const float m_use = wk.m_ref == -INFINITY ? 0.f : wk.m_ref;
    float psum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = fast_exp2(sc[r] - m_use);
      psum += sc[r];
    }
    wk.l_run += psum;
    const u32x4 p8[2] = {pack8(sc, 0), pack8(sc, 8)};
    if (CAP && edge && wk.few) {  // wave-uniform
      const float fix = sum8(p8[0]) + sum8(p8[1]) - psum;
      wk.l_fix += CAREFUL && !wk.stays ? 0.f : fix;  // a reference that moves does not move it
    }
    const bf16x8 pf[2] = {as_bf16x8(p8[0]), as_bf16x8(p8[1])};
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const int ro = (2 * m + s2) * 16 * T::ROW_BYTES;
        bf16x8 x = tr_operand(Ks, off.v[n][0] + ro, off.v[n][1] + ro);
        if constexpr (CAREFUL) x = finite_operand(x, seen[s2], oacc[n]);
        oacc[n] = mfma32x32x16(x, pf[s2], oacc[n]);
      }
    if constexpr (!CAREFUL) {
      __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 4, 0);
#pragma unroll
      for (int i = 0; i < 2 * C::NE - 2; ++i) {
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kSchedMfma, 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// O of no finite value anywhere in the workgroup: infinities or NaN in V, which 0 * V
// may have carried to rows that do not see them, or P, or its products, past fp32's range.
// Or a row whose sum is low with a fixed reference (P of all its keys down to 2^-92): its
// products with small values have come out 0.  All rows again, tile by tile, those whose
// sum is far from 1 against their maximum (the others keep their reference, and so their
// bits, whatever is in rows beside them).
template <class C, int D, bool CAP, bool BIAS>
__device__ __forceinline__ void again_if_needed(Work<C> &wk, const Offsets<C, D> &off,
                                                const Copies<C, D> &copies,
                                                const bf16x8 (&qf)[C::NS], f32x16 (&oacc)[C::NE],
                                                const unsigned char *smem,
                                                uint32_t (&votes)[3][kMaxWaves], int part) {
  const bool bad = !finite<C::NE>(oacc, 0.f * wk.l_run);
  if constexpr (CAP) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool sees = wk.fixed && wk.hi > wk.lo;
    const float l = pair_sum(wk.l_run);
    const uint32_t any = __builtin_amdgcn_ballot_w64(bad) != 0;
    const uint32_t low = (uint32_t)__builtin_amdgcn_ballot_w64(sees && l < kLowSum);
    const uint32_t high = (uint32_t)__builtin_amdgcn_ballot_w64(sees && l > kHighSum);
    if ((threadIdx.x & 63) == 0) votes[0][w] = any, votes[1][w] = low, votes[2][w] = high;
    __syncthreads();
    uint32_t wrong = 0, little = 0, mine = 0;
#pragma unroll
    for (int r = 0; r < C::R; ++r) {
      uint32_t lows = ~0u, highs = 0;  // low in every part: in one, keys may well weigh nothing
#pragma unroll
      for (int p = 0; p < C::P; ++p) {
        wrong |= votes[0][p * C::R + r];
        lows &= votes[1][p * C::R + r];
        highs |= votes[2][p * C::R + r];
      }
      little |= lows;
      if (w % C::R == r) mine = lows | highs;
    }
    wrong = __builtin_amdgcn_readfirstlane(wrong);
    little = __builtin_amdgcn_readfirstlane(little);
    if (!wrong && !little) return;
    if (wk.fixed) {
      wk.stays = !((mine >> (threadIdx.x & 31)) & 1);
      if (!wk.stays) wk.m_ref = -INFINITY;
      wk.fixed = false;
    } else {
      wk.m_ref = -INFINITY;
    }
  } else {
    if (!__syncthreads_or(bad)) return;
    wk.m_ref = -INFINITY;
  }
  wk.l_run = wk.l_fix = 0.f;
  clear<C::NE>(oacc);
  for (int u = 0; u < wk.nt; ++u) {
    barrier_no_fence();  // every wave is done with the stage
    copies.load(wk, u);
    wait_vmcnt<0>();
    barrier_no_fence();
    if (!wk.none(u, part))
      one_tile<C, D, CAP, BIAS, true>(wk, off, qf, oacc,
                                      smem + (u % C::STAGES) * C::TILE_BYTES, u, part);
  }
}

// Workgroups of 64 or 128 rows, the keys of a tile shared by 4 or 2 waves.
template <int D, int R, bool CAP, bool BIAS>
__global__ __launch_bounds__(512, 1) void span_fwd_split_kernel(const SpanArgs a,
                                                                     uint16_t *__restrict__ o,
                                                                     float *__restrict__ lse,
                                                                     int heads_total, int qtiles) {
  using C = Cfg<D, 8, R, 32>;
  // LDS: the K tiles of the ring stages, then their V tiles.
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::LDS_BYTES];
  __shared__ int hulls[2][kMaxWaves];
  __shared__ uint32_t votes[3][kMaxWaves];
  constexpr int kSt = C::STAGES;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = w % R, part = w / R;  // row group, key part
  Work<C> wk;
  bf16x8 qf[C::NS];
  enter<C, D, CAP, BIAS>(wk, qf, a, heads_total, qtiles, hulls);
  const Copies<C, D> copies(wk, smem);
  // Tiles 0 .. kSt-2 are issued up front; iteration u waits for its own copies of
  // tile u, passes the barrier and issues tile u + kSt-1 into the stage of tile
  // u-1, which every wave has finished with.
  auto begin_tile = [&](int u) __attribute__((always_inline)) {
    if constexpr (kSt == 4) {
      const int ahead = min(2, wk.nt - 1 - u);
      if (ahead >= 2) wait_vmcnt<4 * C::DMA_PER_WAVE>();
      else if (ahead == 1) wait_vmcnt<2 * C::DMA_PER_WAVE>();
      else wait_vmcnt<0>();
    } else {
      wait_vmcnt<0>();
    }
    barrier_no_fence();
    if (u + kSt - 1 < wk.nt) copies.load(wk, u + kSt - 1);
  };
#pragma unroll
  for (int u = 0; u < kSt - 1; ++u)
    if (u < wk.nt) copies.load(wk, u);
  const Offsets<C, D> off(part);
  f32x16 oacc[C::NE];
  clear<C::NE>(oacc);
  for (int u0 = 0; u0 < wk.nt; u0 += kSt)
#pragma unroll
    for (int st = 0; st < kSt; ++st)
      if (u0 + st < wk.nt) {
        begin_tile(u0 + st);
        if (!wk.none(u0 + st, part))  // wave-uniform
          one_tile<C, D, CAP, BIAS, false>(wk, off, qf, oacc, smem + st * C::TILE_BYTES, u0 + st,
                                           part);
      }
  again_if_needed<C, D, CAP, BIAS>(wk, off, copies, qf, oacc, smem, votes, part);
  float l_tot = pair_sum(wk.l_run), l_fix = CAP ? pair_sum(wk.l_fix) : 0.f;
  if (!merge_parts<C>(smem, rg, part, lane, wk.m_ref, l_tot, l_fix, oacc)) return;
  leave<C, D>(wk, a, o, lse, l_tot, l_fix, oacc);
}

// Workgroups of 128 rows, of 4 waves or of 8 that share the keys, software-pipelined as
// the causal forward is: the score products of tile u+1 are issued between the
// exponentials of tile u, and the row sum of u between its P V products, one product
// per slot.
// Without a cap a row's reference starts as the maximum of the first scores that it
// sees, is checked against the maximum on edges, and on the other tiles follows the
// row sums (half a row's sum is at least its maximum); where P passes fp32's range in
// between, the workgroup is done again (above).
template <int D, int WAVES, int R, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * WAVES, 8 / WAVES) void span_fwd_kernel(const SpanArgs a,
                                                               uint16_t *__restrict__ o,
                                                               float *__restrict__ lse,
                                                               int heads_total, int qtiles) {
  using C = Cfg<D, WAVES, R, 64>;
  using T = LdsTile<C::LW>;
  // Four stages: three tiles in flight.  Two (128 keys): K runs one tile ahead of V.
  constexpr int kSt = C::STAGES, kPD = 2, kPf = 2;
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::LDS_BYTES];
  __shared__ int hulls[2][kMaxWaves];
  __shared__ uint32_t votes[3][kMaxWaves];
  const int hh = (threadIdx.x & 63) >> 5;
  Work<C> wk;
  bf16x8 qf[C::NS];
  enter<C, D, CAP, BIAS>(wk, qf, a, heads_total, qtiles, hulls);
  const int part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / R;
  const Copies<C, D> copies(wk, smem);
  const int nt = wk.nt;
  if constexpr (kSt == 4) {
    for (int u = 0; u <= kPD && u < nt; ++u) copies.load(wk, u);
  } else if (nt > 0) {
    copies.load(wk, 0);
    if (nt > 1) copies.load_k(wk, 1);
  }
  const Offsets<C, D> off(part);
  f32x16 oacc[C::NE];
  clear<C::NE>(oacc);
  if (!CAP && wk.row >= a.S) wk.m_ref = 0.f;  // waits for no first key

  auto wait_tile = [&](int ahead) __attribute__((always_inline)) {
    if (ahead >= 2) wait_vmcnt<4 * C::DMA_PER_WAVE>();
    else if (ahead == 1) wait_vmcnt<2 * C::DMA_PER_WAVE>();
    else wait_vmcnt<0>();
  };
  auto ahead_of = [&](int u, int m) __attribute__((always_inline)) {
    return (float)(wk.row - (wk.first_key(u, part) + 32 * m + 4 * hh));
  };
  auto slope_of = [&](int u, bool edge) __attribute__((always_inline)) {
    return edge ? 0.f : wk.first_key(u, part) > wk.wrow0 ? -wk.sl : wk.sl;
  };
  // Tile u's scores are there: its edge, and the reference.
  auto prepare = [&](int u, bool edge, f32x16 (&sc)[2]) __attribute__((always_inline)) {
    if constexpr (!CAP) {
      const bool first = __builtin_amdgcn_ballot_w64(wk.m_ref == -INFINITY) != 0;
      if (!edge && !first) return;  // wave-uniform
      const float slp = slope_of(u, edge);
      float mx = -INFINITY;
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        if (edge) wk.template fix_scores<BIAS>(sc[m], wk.first_key(u, part) + 32 * m + 4 * hh);
        const float base = BIAS ? -slp * ahead_of(u, m) : 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          mx = fmaxf(mx, fmaf(sc[m][r], wk.c,
                              BIAS ? fmaf(slp, (float)(8 * (r >> 2) + (r & 3)), base) : base));
      }
      move_reference<C>(wk, oacc, pair_max(mx));
    }
  };
  // With a cap, an edge's P: the exponents so far hold neither bias nor reference.
  auto fix_weights = [&](int u, f32x16 (&p)[2], u32x4 (&pf)[4]) __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float ahead = ahead_of(u, m);
      const int past = wk.first_key(u, part) + 32 * m + 4 * hh - wk.lo;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int jo = 8 * (r >> 2) + (r & 3);
        const bool vis = (uint32_t)(past + jo) < (uint32_t)(wk.hi - wk.lo);
        float x = p[m][r];
        if constexpr (BIAS) {
          // in two halves: a key's P, of up to 2^92 before its bias, may be most of the
          // row's sum where that bias alone would be below fp32's range
          const float y = fast_exp2(0.5f * fmaf(-wk.sl, fabsf(ahead - (float)jo), -wk.m_ref));
          x = x * y * y;
        }
        p[m][r] = vis ? x : 0.f;
      }
      pf[2 * m] = pack8(p[m], 0);
      pf[2 * m + 1] = pack8(p[m], 8);
    }
    asm volatile("" ::: "memory");
  };
  auto follow = [&](float psum) __attribute__((always_inline)) {
    if (__builtin_amdgcn_ballot_w64(!(psum <= kFollowSum))) {  // wave-uniform, rare
      asm volatile("" ::: "memory");
      // 2^-up in two halves: itself it can lie below fp32's normal range
      const float up = fast_log2(fmaxf(pair_max(psum), 1.f));
      const float half = fast_exp2(-0.5f * up);
      wk.m_ref += up;
      wk.l_run = wk.l_run * half * half;
#pragma unroll
      for (int n = 0; n < C::NE; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[n][r] = oacc[n][r] * half * half;
    }
  };

  bool none = nt == 0, edge = false;  // of the current tile
  f32x16 sa[2], sb[2];
  // Iteration u: `cur` holds the scores of tile u, those of tile u + 1 (where there is
  // none, of what the stage held before) go to `nxt`.
  auto turn = [&](int u, auto stage_tag, f32x16 (&cur)[2], f32x16 (&nxt)[2])
                  __attribute__((always_inline)) {
    constexpr int ST = decltype(stage_tag)::value;  // u % kSt
    // K of tile u + 1 and V of tile u are there, and the copies after those in flight go
    // into stages that every wave has finished with.
    if constexpr (kSt == 4) {
      wait_tile(min(1, nt - 2 - u));
      barrier_no_fence();
      if (u + kPD + 1 < nt) copies.load(wk, u + kPD + 1);
    } else {
      wait_vmcnt<0>();
      barrier_no_fence();
      if (u + 2 < nt) copies.load_k(wk, u + 2);
      if (u + 1 < nt) copies.load_v(wk, u + 1);
    }
    const bool none_next = u + 1 >= nt || wk.none(u + 1, part);
    const bool edge_next = !none_next && wk.template edge<BIAS>(u + 1, part);
    if (!none || !none_next) {
      asm volatile("" : "+v"(wk.m_ref));  // keep the exponent arguments here
      const float m_use = !CAP && wk.m_ref == -INFINITY ? 0.f : wk.m_ref;
      const float slp = BIAS ? slope_of(u, edge) : 0.f;
      float base[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        base[m] = CAP ? (edge && BIAS ? wk.cap2 : wk.cap2 - m_use) : -m_use;
        if constexpr (BIAS) base[m] = fmaf(-slp, ahead_of(u, m), base[m]);
      }
      u32x4 pf[4];
      // Block X: scores of tile u+1, exponentials of tile u, at raised issue
      // priority: of the two waves of a SIMD, the one in this block keeps the
      // matrix unit while the other is in block Y.
      wave_priority<1>();
      {
        constexpr int NG = 2 * C::NS;
        const unsigned char *Ks = smem + ((ST + 1) % kSt) * C::TILE_BYTES;
        bf16x8 op[NG];
        auto read = [&](int g) __attribute__((always_inline)) {
          op[g] = *reinterpret_cast<const bf16x8 *>(Ks + off.k[g / 2] + (g % 2) * 32 * T::ROW_BYTES);
        };
#pragma unroll
        for (int g = 0; g < kPf; ++g) read(g);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          if (g + kPf < NG) read(g + kPf);
          const int m = g % 2, s2 = g / 2;
          nxt[m] = mfma32x32x16(op[g], qf[s2], s2 == 0 ? f32x16{} : nxt[m]);
#pragma unroll
          for (int e = 32 * g / NG; e < 32 * (g + 1) / NG; ++e) {
            const int mm = e / 16, r = e % 16, jo = 8 * (r >> 2) + (r & 3);
            const float add = BIAS ? fmaf(slp, (float)jo, base[mm]) : base[mm];
            if constexpr (CAP)
              cur[mm][r] = fast_exp2(fmaf(cap_r(cur[mm][r], wk.c1), -2.f * wk.cap2, add));
            else
              cur[mm][r] = fast_exp2(fmaf(cur[mm][r], wk.c, add));
            if (r % 8 == 7) pf[2 * mm + r / 8] = pack8(cur[mm], r - 7);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      wave_priority<0>();
      if (CAP && edge) fix_weights(u, cur, pf);  // wave-uniform
      if (!none) {
        // Block Y: P V of tile u, its row sum.
        float psum = 0.f;
        constexpr int NG = C::NE * 4;
        const unsigned char *Vs = smem + ST * C::TILE_BYTES;
        bf16x8 op[NG];
        auto read = [&](int g) __attribute__((always_inline)) {
          const int n = g / 4, s2 = g % 4;
          op[g] = tr_operand(Vs, off.v[n][0] + s2 * 16 * T::ROW_BYTES,
                             off.v[n][1] + s2 * 16 * T::ROW_BYTES);
        };
#pragma unroll
        for (int g = 0; g < kPf; ++g) read(g);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          if (g + kPf < NG) read(g + kPf);
          const int n = g / 4, s2 = g % 4;
          oacc[n] = mfma32x32x16(op[g], as_bf16x8(pf[s2]), oacc[n]);
#pragma unroll
          for (int e = 32 * g / NG; e < 32 * (g + 1) / NG; ++e) psum += cur[e / 16][e % 16];
          __builtin_amdgcn_sched_barrier(0);
        }
        wk.l_run += psum;
        if constexpr (!CAP) follow(psum);
        if (CAP && edge && wk.few) {  // wave-uniform
          asm volatile("" ::: "memory");
          wk.l_fix += sum8(pf[0]) + sum8(pf[1]) + sum8(pf[2]) + sum8(pf[3]) - psum;
        }
      }
      if (!none_next) prepare(u + 1, edge_next, nxt);
    }
    none = none_next;
    edge = edge_next;
  };
  if (nt > 0) {
    if constexpr (kSt == 4) wait_tile(min(kPD, nt - 1));
    else wait_vmcnt<0>();
    barrier_no_fence();
    none = wk.none(0, part);
    edge = !none && wk.template edge<BIAS>(0, part);
    if (!none) {
#pragma unroll
      for (int s = 0; s < C::NS; ++s)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const bf16x8 x =
              *reinterpret_cast<const bf16x8 *>(smem + off.k[s] + m * 32 * T::ROW_BYTES);
          sa[m] = mfma32x32x16(x, qf[s], s == 0 ? f32x16{} : sa[m]);
        }
      prepare(0, edge, sa);
    } else {
#pragma unroll
      for (int m = 0; m < 2; ++m) sa[m] = f32x16{};
    }
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2 % kSt>;
    using I3 = std::integral_constant<int, 3 % kSt>;
    for (int u = 0; u < nt; u += kSt) {  // every stage offset a constant
      turn(u, I0{}, sa, sb);
      if (u + 1 < nt) turn(u + 1, I1{}, sb, sa);
      if constexpr (kSt == 4) {
        if (u + 2 < nt) turn(u + 2, I2{}, sa, sb);
        if (u + 3 < nt) turn(u + 3, I3{}, sb, sa);
      }
    }
  }
  again_if_needed<C, D, CAP, BIAS>(wk, off, copies, qf, oacc, smem, votes, part);
  float l_tot = pair_sum(wk.l_run), l_fix = CAP ? pair_sum(wk.l_fix) : 0.f;
  if constexpr (C::P > 1) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (!merge_parts<C>(smem, w % R, part, threadIdx.x & 63, wk.m_ref, l_tot, l_fix, oacc))
      return;
  }
  leave<C, D>(wk, a, o, lse, l_tot, l_fix, oacc);
}

// The workgroup of a call, by its query rows W = b Hl S: few rows need small ones
// to fill the GPU, and many let a K or V tile feed more products.  Three kinds, us on
// MI355X (8 heads on 2 of 128; one document | documents of some S / 8 tokens, one draw | of 300):
//   64 rows, 8 waves; 128 rows, 8 waves, pipelined; 128 rows, 4 waves, pipelined, two a CU
//   W = 16K, S = 2048  29, 34, -    15, 18, -     15, 19, -
//   32K, 4096          58, 61, 73   31, 29, 34    25, 22, 24
//   46K, 6000          115, 91, 112 40, 39, 37    38, 36, 32
//   64K, 8192          195, 149, 175  64, 53, 49  51, 40, 38
//   96K, 48 x 256      62, 43, 29
//   93K, 2 x 6000      227, 179, 153  98, 73, 66  70, 53, 39
//   128K, 16384        717, 521, 483  393, 306, 354  91, 70, 55
//   512K, 65536 on 1   9984, 7830, 7413  1685, 1286, 1253  364, 257, 178
// (256 rows and 8 waves, one workgroup a CU, 493, 300 and 66 at W = 128K, lost to the
// last kind wherever the others did.)  Documents of thousands of tokens end with a few long
// workgroups, which 8 waves do in half the time; which kind wins past 72K rows is then a
// matter of the draw, us of three each, 8 waves and 4:
//   W = 96K   of 1000  77 75, 90 98, 103 135     of 4096  178 212, 314 300, 118 107
//   128K      of 1000  102 93, 107 109, 121 142  of 2048  126 140, 213 235, 130 118
//   256K      of 1000  184 155, 226 203, 218 210  of 4096  379 391, 725 720, 407 376
// Caps past kSpanFixedCap take the tiles that follow the running maximum, not pipelined, past
// the first line in 128-row workgroups (one document of 32K tokens, 4 heads on 1: 1494 us, 1137
// with a cap of 50; 16K tokens of documents of 2K, 8 on 2: 184, 167).
enum class Kind { k64, k128, k128Narrow, k128Running };
Kind kind_of(const SpanArgs &a) {
  const long long rows = (long long)a.b * a.Hl * a.S;
  if (rows <= 28672) return Kind::k64;
  if (a.cap > kSpanFixedCap) return Kind::k128Running;
  return rows <= 73728 && a.S > 512 ? Kind::k128 : Kind::k128Narrow;
}

}  // namespace

hipError_t launch_span_fwd(const SpanArgs &a, uint16_t *o, float *lse, hipStream_t stream) {
  const Kind kind = kind_of(a);
  const int rows = kind == Kind::k64 ? 64 : 128;
  const int qtiles = (a.S + rows - 1) / rows;
  const int heads_total = a.b * a.Hl;
  const long long blocks = (long long)qtiles * heads_total;
  auto by_rule = [&](auto dim, auto cap, auto bias) {
    constexpr int D = decltype(dim)::value;
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    auto go = [&](auto kernel, int threads) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, stream, a, o, lse,
                         heads_total, qtiles);
    };
    switch (kind) {
      case Kind::k64: go(span_fwd_split_kernel<D, 2, CAP, BIAS>, 512); break;
      case Kind::k128: go(span_fwd_kernel<D, 8, 4, CAP, BIAS>, 512); break;
      case Kind::k128Narrow: go(span_fwd_kernel<D, 4, 4, CAP, BIAS>, 256); break;
      case Kind::k128Running:
        if constexpr (CAP) go(span_fwd_split_kernel<D, 4, CAP, BIAS>, 512);
        break;
    }
  };
  auto by_dim = [&](auto dim) {
    using No = std::false_type;
    using Yes = std::true_type;
    if (a.cap > 0.f) a.slopes ? by_rule(dim, Yes{}, Yes{}) : by_rule(dim, Yes{}, No{});
    else a.slopes ? by_rule(dim, No{}, Yes{}) : by_rule(dim, No{}, No{});
  };
  switch (a.d) {
    case 64: by_dim(std::integral_constant<int, 64>{}); break;
    case 80: by_dim(std::integral_constant<int, 80>{}); break;
    case 96: by_dim(std::integral_constant<int, 96>{}); break;
    default: by_dim(std::integral_constant<int, 128>{}); break;
  }
  return hipGetLastError();
}

}  // namespace basp
