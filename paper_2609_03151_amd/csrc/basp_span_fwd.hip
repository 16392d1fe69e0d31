// basp_span_fwd.hip -- forward of attention over spans.
//
// Every query row sees one run of keys [lo, hi); scores may be capped by a
// tanh and biased by distance (basp_span.hpp).  Bound by the matrix cores
// (4 d operations a seen pair) and, with a cap, by the vector units, which form
// three exponentials or reciprocals a score instead of one.
//
// gfx950 mapping, as the causal forward's: a workgroup of 8 waves owns 32 R
// query rows of one head, R row groups times P = 8 / R key parts; S^T = K Q^T
// and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16, with Q in registers, P
// straight from the score accumulator, and K and V copied HBM -> LDS into a
// ring of stages.  A lane holds one row's scores of 16 keys per 32.
//
// Masks cost what lies on their edges: the workgroup visits the tiles between
// its rows' least lo and largest hi, and a wave skips tiles that none of its 32
// rows sees and takes tiles that all of them see without any mask.
#include <math.h>

#include <type_traits>

#include "basp_span_device.hpp"

namespace basp {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = 8;
constexpr float kRescaleSlack = 8.f;  // log2 headroom before the reference max moves
constexpr int kSchedMfma = 0x008;
constexpr int kSchedDsRead = 0x100;

template <int D, int RG>
struct Cfg {
  static constexpr int R = RG, P = kWaves / R;
  static constexpr int DC = HeadDim<D>::DC;
  static constexpr int LW = HeadDim<D>::LW;
  static constexpr int BM = 32 * R;               // query rows per workgroup
  static constexpr int KM = P == 1 ? 2 : 1;       // 32-key blocks per wave and tile
  static constexpr int BN = 32 * KM * P;          // keys per tile
  static constexpr int TILE_BYTES = BN * LW * 2;
  static constexpr int STAGES = 2 * TILE_BYTES > 32768 ? 2 : 4;
  static constexpr int LDS_BYTES = STAGES * 2 * TILE_BYTES;
  static constexpr int NS = D / 16;               // 16-deep steps over the head dim
  static constexpr int NE = DC / 32;              // 32-wide head-dim subtiles of O
  static constexpr int CPR = LW / 8;              // 16-byte chunks per LDS row
  static constexpr int DMA_PER_WAVE = BN * CPR / kThreads;
  static constexpr int PART_BYTES = NE * 4 * 1024 + 512;
  static_assert((P - 1) * R * PART_BYTES <= LDS_BYTES, "the merge area fits the ring");
};

// The key parts of a row group brought together: parts 1 .. P-1 put their
// reference, row sum and O in LDS (every copy landed, nothing left to read in the
// ring), part 0 takes them into its own in order.  True in part 0.
template <class C>
__device__ __forceinline__ bool merge_parts(unsigned char *smem, int rg, int part, int lane,
                                            float &m_ref, float &l_tot, f32x16 (&oacc)[C::NE]) {
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
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[n][r] *= wt[0];
#pragma unroll
  for (int p = 1; p < C::P; ++p) {
    l_tot = fmaf(wt[p], *reinterpret_cast<const float *>(area(p) + kScalars + 256 + 4 * lane),
                 l_tot);
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

template <int D, int R, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 1) void span_fwd_kernel(const SpanArgs a,
                                                               uint16_t *__restrict__ o,
                                                               float *__restrict__ lse,
                                                               int heads_total, int qtiles) {
  using C = Cfg<D, R>;
  using T = LdsTile<C::LW>;
  // LDS: the K tiles of the ring stages, then their V tiles.
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::LDS_BYTES];
  __shared__ int hulls[2][kWaves];
  constexpr int kSt = C::STAGES, kVRegion = kSt * C::TILE_BYTES;

  const int S = a.S, Hl = a.Hl;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const int rg = w % R, part = w / R;  // row group, key part

  const int L = blockIdx.x;
  const int qt = qtiles - 1 - L / heads_total;
  const int hb = L % heads_total;
  const int beta = hb / Hl, h = hb % Hl, kvh = h / (Hl / a.Hkl);
  const int q0 = qt * C::BM;
  const int wrow0 = q0 + 32 * rg;
  const int row = wrow0 + l32;

  const uint32_t q_row_bytes = a.q.row_elems * 2;
  const uint32_t k_row_bytes = a.k.row_elems * 2, v_row_bytes = a.v.row_elems * 2;
  const rsrc_t rq = make_rsrc(a.q.p + ((size_t)beta * S + q0) * a.q.row_elems + (size_t)h * D,
                              (uint32_t)(S - q0) * q_row_bytes);
  const u32x4 rk = make_rsrc_words(a.k.p + (size_t)beta * S * a.k.row_elems + (size_t)kvh * D,
                                   (uint32_t)S * k_row_bytes);
  const u32x4 rv = make_rsrc_words(a.v.p + (size_t)beta * S * a.v.row_elems + (size_t)kvh * D,
                                   (uint32_t)S * v_row_bytes);
  const uint32_t smem_lds = lds_addr_of(smem);

  bf16x8 qf[C::NS];
#pragma unroll
  for (int s = 0; s < C::NS; ++s)
    qf[s] = as_bf16x8(buf_load16(rq, (uint32_t)(row - q0) * q_row_bytes + (2 * s + hh) * 16));
  int lo = 0, hi = 0;
  if (row < S) span_of(a.spans, beta, S, row, lo, hi);
  float sl = 0.f;  // the slope in log2 units
  if constexpr (BIAS) sl = a.slopes[h] * kSpanLog2e;
  const SpanHull wh = wave_hull(hull_of(lo, hi, row < S));
  if (lane == 0) hulls[0][w] = wh.any_lo, hulls[1][w] = wh.any_hi;
  wait_vmcnt<0>();  // retire the tracked loads before untracked copies start
  __syncthreads();
  int all_lo = hulls[0][0], all_hi = hulls[1][0];
#pragma unroll
  for (int i = 1; i < R; ++i) {
    all_lo = min(all_lo, hulls[0][i]);
    all_hi = max(all_hi, hulls[1][i]);
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  const int t0 = all_lo < all_hi ? all_lo / C::BN : 0;
  const int nt = all_lo < all_hi ? (all_hi + C::BN - 1) / C::BN - t0 : 0;  // tiles t0 .. t0+nt-1

  uint32_t gk[C::DMA_PER_WAVE], gv[C::DMA_PER_WAVE];
#pragma unroll
  for (int i = 0; i < C::DMA_PER_WAVE; ++i) {
    gk[i] = dma_src_off<C::LW, D>((w * C::DMA_PER_WAVE + i) * 64 + lane, k_row_bytes);
    gv[i] = dma_src_off<C::LW, D>((w * C::DMA_PER_WAVE + i) * 64 + lane, v_row_bytes);
  }
  auto load_tile = [&](int u) __attribute__((always_inline)) {  // tile t0 + u
    const uint32_t ks = smem_lds + (u % kSt) * C::TILE_BYTES;
    const uint32_t kb = (uint32_t)((t0 + u) * C::BN) * k_row_bytes;
    const uint32_t vb = (uint32_t)((t0 + u) * C::BN) * v_row_bytes;
#pragma unroll
    for (int i = 0; i < C::DMA_PER_WAVE; ++i) {
      const uint32_t lds_off = ks + (w * C::DMA_PER_WAVE + i) * 1024;
      copy16_to_lds(rk, kb + gk[i], lds_off);
      copy16_to_lds(rv, vb + gv[i], lds_off + kVRegion);
    }
  };
  // Tiles 0 .. kSt-2 are issued up front; iteration u waits for its own copies of
  // tile u, passes the barrier and issues tile u + kSt-1 into the stage of tile
  // u-1, which every wave has finished with.
  auto begin_tile = [&](int u) __attribute__((always_inline)) {
    if constexpr (kSt == 4) {
      const int ahead = min(2, nt - 1 - u);
      if (ahead >= 2) wait_vmcnt<4 * C::DMA_PER_WAVE>();
      else if (ahead == 1) wait_vmcnt<2 * C::DMA_PER_WAVE>();
      else wait_vmcnt<0>();
    } else {
      wait_vmcnt<0>();
    }
    barrier_no_fence();
    if (u + kSt - 1 < nt) load_tile(u + kSt - 1);
  };
#pragma unroll
  for (int u = 0; u < kSt - 1; ++u)
    if (u < nt) load_tile(u);

  // This lane's operand reads: K row l32 and V^T rows of the wave's part.
  const int part_off = part * 32 * C::KM * T::ROW_BYTES;
  int k_off[C::NS], v_off[C::NE][2];
#pragma unroll
  for (int s = 0; s < C::NS; ++s) {
    k_off[s] = T::off(l32, 2 * s + hh) + part_off;
    asm volatile("" : "+v"(k_off[s]));
  }
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      v_off[n][x] = kVRegion + part_off +
                    tr_piece_off<C::LW>(4 * hh + 8 * x, 32 * n + 16 * ((lane >> 4) & 1), lane);
      asm volatile("" : "+v"(v_off[n][x]));
    }

  const float c = a.scale * kSpanLog2e;
  const float c1 = CAP ? 2.f * c / a.cap : 0.f, cap2 = CAP ? a.cap * kSpanLog2e : 0.f;
  const bool fixed = CAP && a.cap <= kSpanFixedCap;
  // The exponents' reference.  With a cap that allows it (kSpanFixedCap) it
  // is the largest bias of the row, at its nearest or farthest key; else the
  // running maximum.
  float m_ref = -INFINITY, l_run = 0.f;
  if (fixed) {
    const int near = row < lo ? lo - row : row >= hi ? row - hi + 1 : 0;
    const int far = max(abs(row - lo), abs(row - hi + 1));
    m_ref = BIAS && hi > lo ? fmaxf(-sl * (float)near, -sl * (float)far) : 0.f;
  }
  f32x16 oacc[C::NE];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[n][r] = 0.f;
  };
  clear();

  // One tile.  EDGE: some row sees only some of its keys (or the bias changes its
  // sign in it).  CAREFUL: V holds infinities or NaN somewhere, which must not
  // reach a row through a weight of 0.
  auto tile = [&](int u, auto edge_tag, auto careful_tag) __attribute__((always_inline)) {
    constexpr bool EDGE = decltype(edge_tag)::value, CAREFUL = decltype(careful_tag)::value;
    const int j0 = (t0 + u) * C::BN + 32 * C::KM * part;
    const unsigned char *Ks = smem + (u % kSt) * C::TILE_BYTES;
    keep_apart<EDGE>();
#pragma unroll
    for (int m = 0; m < C::KM; ++m) {
      f32x16 sc;
      wave_priority<1>();
#pragma unroll
      for (int s = 0; s < C::NS; ++s) {
        const bf16x8 x = *reinterpret_cast<const bf16x8 *>(Ks + k_off[s] + m * 32 * T::ROW_BYTES);
        sc = mfma32x32x16(x, qf[s], s == 0 ? f32x16{} : sc);
      }
      wave_priority<0>();
      // sc[r] = (q . k) of key jl + 8(r/4) + r%4 for this lane's row
      const int jl = j0 + 32 * m + 4 * hh;
      float ahead = (float)(row - jl);  // distance to the lane's first key
      int past = jl - lo;
      // (else sums of these and the 16 offsets are kept over the whole loop)
      asm volatile("" : "+v"(ahead), "+v"(past));
      const float slp = j0 + 32 * m > wrow0 ? -sl : sl;  // not EDGE: all keys on one side
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int jo = 8 * (r >> 2) + (r & 3);
        float x = sc[r];
        if constexpr (CAP) x = fmaf(cap_r(x, c1), -2.f * cap2, cap2);
        else x *= c;
        if constexpr (BIAS) {
          if constexpr (EDGE) x = fmaf(-sl, fabsf(ahead - (float)jo), x);
          else x = fmaf(-slp, ahead - (float)jo, x);
        }
        if constexpr (EDGE)
          if ((uint32_t)(past + jo) >= (uint32_t)(hi - lo)) x = -INFINITY;
        sc[r] = x;
      }
      if (!fixed) {
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
      }
      // A row of which no key has come yet: every score is -inf, P = 0.
      const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
      float psum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[r] = fast_exp2(sc[r] - m_use);
        psum += sc[r];
      }
      l_run += psum;
      u32x4 pw[2];
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const int b8 = 8 * s2;
        pw[s2] = u32x4{pack_bf16x2(sc[b8 + 0], sc[b8 + 1]), pack_bf16x2(sc[b8 + 2], sc[b8 + 3]),
                       pack_bf16x2(sc[b8 + 4], sc[b8 + 5]), pack_bf16x2(sc[b8 + 6], sc[b8 + 7])};
      }
#pragma unroll
      for (int n = 0; n < C::NE; ++n) {
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          const int ro = (2 * m + s2) * 16 * T::ROW_BYTES;
          bf16x8 x = tr_operand(Ks, v_off[n][0] + ro, v_off[n][1] + ro);
          if constexpr (CAREFUL) {
            u32x4 v = __builtin_bit_cast(u32x4, x), bad;
#pragma unroll
            for (int y = 0; y < 4; ++y) bad[y] = nonfinite_halves(v[y]);
            if (__builtin_amdgcn_ballot_w64((bad.x | bad.y | bad.z | bad.w) != 0)) {
              // how many such values of its column each row sees: 1 for each
              // in V's place, 1 for each key seen in P's
              u32x4 seen;
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const uint32_t one_hi = bad[y] & 0x80000000u, one_lo = bad[y] & 0x8000u;
                if (one_hi) v[y] &= 0xFFFFu;
                if (one_lo) v[y] &= 0xFFFF0000u;
                bad[y] = (one_hi ? 0x3F800000u : 0u) | (one_lo ? 0x3F80u : 0u);
                const int r = 8 * s2 + 2 * y, j = jl + 8 * (r >> 2) + (r & 3);
                seen[y] = ((uint32_t)(j - lo) < (uint32_t)(hi - lo) ? 0x3F80u : 0u) |
                          ((uint32_t)(j + 1 - lo) < (uint32_t)(hi - lo) ? 0x3F800000u : 0u);
              }
              const f32x16 count = mfma32x32x16(as_bf16x8(bad), as_bf16x8(seen), f32x16{});
#pragma unroll
              for (int r = 0; r < 16; ++r)
                if (count[r] > 0.f) oacc[n][r] = __builtin_nanf("");
              x = as_bf16x8(v);
            }
          }
          oacc[n] = mfma32x32x16(x, as_bf16x8(pw[s2]), oacc[n]);
        }
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
    keep_apart<EDGE>();
  };
  using No = std::false_type;
  using Yes = std::true_type;
  constexpr int kWaveKeys = 32 * C::KM;
  for (int u = 0; u < nt; ++u) {
    begin_tile(u);
    const int j0 = (t0 + u) * C::BN + kWaveKeys * part;
    if (wh.none(j0, kWaveKeys)) continue;  // wave-uniform
    const bool crosses = BIAS && j0 + kWaveKeys - 1 > wrow0 && j0 < wrow0 + 31;
    if (wh.full(j0, kWaveKeys) && !crosses) tile(u, No{}, No{});
    else tile(u, Yes{}, No{});
  }

  // O of no finite value anywhere in the workgroup: infinities or NaN in V, which
  // 0 * V may have carried to rows that do not see them (or an overflow).  All rows
  // again, tile by tile, with such values kept apart.
  {
    float z = 0.f;
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) z = fmaf(0.f, oacc[n][r], z);
    if (__syncthreads_or(!(z == 0.f))) {
      if (!fixed) m_ref = -INFINITY;
      l_run = 0.f;
      clear();
      for (int u = 0; u < nt; ++u) {
        barrier_no_fence();  // every wave is done with the stage
        load_tile(u);
        wait_vmcnt<0>();
        barrier_no_fence();
        if (!wh.none((t0 + u) * C::BN + kWaveKeys * part, kWaveKeys)) tile(u, Yes{}, Yes{});
      }
    }
  }

  // oacc[n][r] = O^T[e = 32n + 8(r/4) + 4hh + r%4][query row] (unnormalised)
  float l_tot = pair_sum(l_run);
  if constexpr (C::P > 1) {
    if (!merge_parts<C>(smem, rg, part, lane, m_ref, l_tot, oacc)) return;
  }
  if (row >= S) return;
  const bool empty = hi <= lo;
  const float inv = empty ? 0.f : 1.f / l_tot;
  uint16_t *ob = o + (((size_t)beta * S + row) * Hl + h) * D;
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
    lse[((size_t)beta * Hl + h) * S + row] =
        empty ? -INFINITY : (m_ref + fast_log2(l_tot)) * kSpanLn2;
}

// Row groups of a workgroup: fewer rows fill the GPU where there are few, more
// let a K or V tile feed more products.
int row_groups(const SpanArgs &a) {
  const long long rows = (long long)a.b * a.Hl * a.S;
  return rows <= 32768 ? 2 : rows <= 65536 ? 4 : 8;
}

}  // namespace

hipError_t launch_span_fwd(const SpanArgs &a, uint16_t *o, float *lse, hipStream_t stream) {
  const int R = row_groups(a);
  const int qtiles = (a.S + 32 * R - 1) / (32 * R);
  const int heads_total = a.b * a.Hl;
  const long long blocks = (long long)qtiles * heads_total;
  auto by_rule = [&](auto dim, auto groups, auto cap, auto bias) {
    constexpr int D = decltype(dim)::value, RG = decltype(groups)::value;
    hipLaunchKernelGGL((span_fwd_kernel<D, RG, decltype(cap)::value, decltype(bias)::value>),
                       dim3((unsigned)blocks), dim3(kThreads), 0, stream, a, o, lse, heads_total,
                       qtiles);
  };
  auto by_groups = [&](auto dim, auto groups) {
    using No = std::false_type;
    using Yes = std::true_type;
    if (a.cap > 0.f) a.slopes ? by_rule(dim, groups, Yes{}, Yes{}) : by_rule(dim, groups, Yes{}, No{});
    else a.slopes ? by_rule(dim, groups, No{}, Yes{}) : by_rule(dim, groups, No{}, No{});
  };
  auto by_dim = [&](auto dim) {
    switch (R) {
      case 2: by_groups(dim, std::integral_constant<int, 2>{}); break;
      case 4: by_groups(dim, std::integral_constant<int, 4>{}); break;
      default: by_groups(dim, std::integral_constant<int, 8>{}); break;
    }
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
