// basp_span_bwd.hip -- backward of attention over spans.
//
// With P recomputed from the LSE and D_i = dO_i . O_i:
//   dU_ij = P_ij (dO_i . v_j - D_i),   dS_ij = dU_ij (1 - tanh^2(s_ij / cap))
//   dV_j = sum_i P_ij dO_i,  dK_j = scale sum_i dS_ij q_i,  dQ_i = scale sum_j dS_ij k_j
// (sums over the keys a row sees, and over the query heads of a kv head).  Bound
// by the matrix cores: five products of 2 d operations a seen pair are needed,
// seven are formed (S and dP in both passes).  On MI355X, 16K tokens, 8 heads on 2 of
// 128: one document with a cap 2035 us, 675 TFLOP/s of the five; documents of some 2K with
// a bias 420 us, 535 TFLOP/s.
//
// Kernels, all deterministic (no atomics):
//   span_pre     per row and head -LSE and -D, of rows padded to 64; per row its span;
//                per 32 rows which keys some and all of them see
//   span_main    each workgroup one unit of either pass:
//     dQ pass    query-stationary: 32 R rows sweep the tiles of their spans
//     key pass   key-stationary: 128 keys sweep those 64-row steps of a row chunk
//                that see any of them (a list built at its start), for all or a
//                part of the query heads; dV and dK in registers
//   span_reduce  sums the chunks' and parts' dK and dV in order
// Both passes skip what nobody sees, take without a mask what everybody sees, and
// mask the rest element by element.
#include <math.h>

#include <type_traits>

#include "basp_span_device.hpp"

namespace basp {
namespace {

constexpr int kPreThreads = 256;
constexpr int kThreads = kSpanThreads;
constexpr int kWaves = kThreads / 64;
constexpr int kKN = kKvKeys;     // keys of a key pass unit: 32 per pair of waves
constexpr int kQM = kSpanStep;   // rows of its step
constexpr int kSchedMfma = 0x008;
constexpr int kSchedDsRead = 0x100;

// Order the LDS operand reads of a run of MFMAs that each take R reads: the
// first A reads up front, then one MFMA per R further reads.
template <int NMFMA, int R, int A>
__device__ __forceinline__ void sched_reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(kSchedDsRead, A, 0);
#pragma unroll
  for (int i = 0; i < NMFMA - A / R; ++i) {
    __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
    __builtin_amdgcn_sched_group_barrier(kSchedDsRead, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kSchedMfma, A / R, 0);
}

static_assert(sizeof(SpanHull) == kSpanHullBytes, "the workspace's");

struct BwdArgs {
  SpanArgs s;
  const uint16_t *d_o;
  const float *lse;
  float *aux;              // [b][Hl][Sp / 64][kPlanes][64]: what span_pre says of 64 rows
  int *rows;               // [b][Sp][kPlanes]: lo and hi
  const SpanHull *hulls;   // [b][Sp / 32]
  int *touched;            // [slot][b][ktiles], or NULL: dk, dv written by the units
  void *dq, *dk, *dv;      // outputs
  float *dk_part, *dv_part;
  size_t part_elems;       // b S Hkl d
  int grad_bf16;
  int Sp, chunk_rows, nchunks, nsplits, ktiles;
  uint32_t dq_blocks, pre_rows_blocks, causal_units, keys_first;
};

// Planes of 64 rows: -LSE, then -D, and with slopes -LSE without the rows' part of the bias
// and an empty one: a step's planes, and its spans, so are copies of a kilobyte (three
// planes were some 5% slower at d = 96 and 64, for scalar registers that the sizes took).
template <bool BIAS>
constexpr int kPlanes = BIAS ? kSpanPlanes : 2;

// Four consecutive gradients, in the output's type.
__device__ __forceinline__ void store4(void *p, size_t elem, f32x4 x, int bf16) {
  if (bf16)
    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(p) + elem) =
        u32x2{pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w)};
  else
    *reinterpret_cast<f32x4 *>(static_cast<float *>(p) + elem) = x;
}

// Sixteen weights of the accumulator as two operands.
__device__ __forceinline__ void pack16(const f32x16 &x, bf16x8 (&out)[2]) {
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
    const int b8 = 8 * s2;
    out[s2] = as_bf16x8(u32x4{pack_bf16x2(x[b8 + 0], x[b8 + 1]), pack_bf16x2(x[b8 + 2], x[b8 + 3]),
                              pack_bf16x2(x[b8 + 4], x[b8 + 5]), pack_bf16x2(x[b8 + 6], x[b8 + 7])});
  }
}

// ---------------------------------------------------------------- span_pre
// Blocks below pre_rows_blocks: a group of lanes per (sequence, row, head) of the
// padded rows, 16-byte loads of O and dO:
//   -(LSE log2(e) + slope' (i % 64)) / c   (not divided with a cap), and -D_i
// c = scale log2(e), slope' = slope log2(e): with the rows' part of the bias in it, the
// key pass adds one number per step and key where all keys lie before the rows.  Elsewhere
// it starts from -LSE / c alone, of which steep slopes would leave nothing.  Rows that
// see nothing, and those past S, have -inf: P = 0.  The other blocks: a wave per 64 rows,
// their spans and two hulls.
template <int D, bool CAP>
__global__ __launch_bounds__(kPreThreads) void span_pre_kernel(const BwdArgs a,
                                                               const uint16_t *__restrict__ o,
                                                               SpanHull *hulls) {
  const int S = a.s.S, Sp = a.Sp, Hl = a.s.Hl;
  if (blockIdx.x >= a.pre_rows_blocks) {  // workgroup-uniform
    const int lane = threadIdx.x & 63;
    const long long step = (long long)(blockIdx.x - a.pre_rows_blocks) * (kPreThreads / 64) +
                           threadIdx.x / 64;
    const int per_seq = Sp / 64;
    if (step >= (long long)a.s.b * per_seq) return;
    const int beta = (int)(step / per_seq), row = (int)(step % per_seq) * 64 + lane;
    int lo = 0, hi = 0;
    if (row < S) span_of(a.s.spans, beta, S, row, lo, hi);
    *reinterpret_cast<u32x2 *>(a.rows + ((size_t)beta * Sp + row) *
                                            (a.s.slopes ? kPlanes<true> : kPlanes<false>)) =
        u32x2{(uint32_t)lo, (uint32_t)hi};
    SpanHull h = hull_of(lo, hi, row < S);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1)
      h = join(h, SpanHull{__shfl_xor(h.any_lo, x), __shfl_xor(h.any_hi, x),
                           __shfl_xor(h.all_lo, x), __shfl_xor(h.all_hi, x)});
    if (lane % 32 == 0) hulls[2 * step + lane / 32] = h;
    return;
  }
  constexpr int LPR = D <= 64 ? 8 : 16;  // lanes per row (a power of two >= D/8)
  const long long gid = (long long)blockIdx.x * kPreThreads + threadIdx.x;
  const long long r = gid / LPR, rows = (long long)a.s.b * Sp * Hl;
  const int sub = (int)(gid % LPR);
  const long long bi = r / Hl;
  const int h = (int)(r - bi * Hl);
  const int beta = (int)(bi / Sp), i = (int)(bi - (long long)beta * Sp);
  float acc = 0.f;
  if (r < rows && i < S && sub < D / 8) {
    const size_t e = (((size_t)beta * S + i) * Hl + h) * D;
    const u32x4 x = reinterpret_cast<const u32x4 *>(o + e)[sub];
    const u32x4 y = reinterpret_cast<const u32x4 *>(a.d_o + e)[sub];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      acc += bf16_bits_to_f32(x[k] & 0xFFFFu) * bf16_bits_to_f32(y[k] & 0xFFFFu);
      acc += bf16_bits_to_f32(x[k] >> 16) * bf16_bits_to_f32(y[k] >> 16);
    }
  }
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) acc += __shfl_xor(acc, off, 64);
  if (r >= rows || sub != 0) return;
  int lo = 0, hi = 0;
  if (i < S) span_of(a.s.spans, beta, S, i, lo, hi);
  const size_t row = (size_t)beta * Hl + h;
  float l = -INFINITY, alone = -INFINITY;
  if (hi > lo) {
    l = alone = -a.lse[row * S + i] * kSpanLog2e;
    if (a.s.slopes) l = fmaf(-a.s.slopes[h] * kSpanLog2e, (float)(i % 64), l);
    if (!CAP) l /= a.s.scale * kSpanLog2e, alone /= a.s.scale * kSpanLog2e;
  }
  float *aux = a.aux + (row * Sp + i / 64 * 64) * (a.s.slopes ? kPlanes<true> : kPlanes<false>) +
               i % 64;
  aux[0] = l;
  aux[64] = i < S ? -acc : 0.f;
  if (a.s.slopes) aux[128] = alone;
}

// ---------------------------------------------------------------- key pass
// An entry of the list of steps is the step's number, and two bits for each of its
// 32-row halves and 32-key blocks (bit 16 + 2 (4 half + block)): 0 nobody sees anything,
// 1 mask, 2 everybody sees everything.
template <int D>
struct KvCfg {
  static constexpr int DC = HeadDim<D>::DC;
  static constexpr int LW = HeadDim<D>::LW;
  static constexpr int TILE_BYTES = kQM * LW * 2;   // a step's Q or dO rows
  static constexpr int KT_BYTES = kKN * LW * 2;     // the workgroup's V rows
  // the planes of the step's rows, and from byte 1024 on their spans
  static constexpr int AUX_BYTES = 2048;
  static constexpr int NS = D / 16;
  static constexpr int NE = DC / 32;
  static constexpr int CPR = LW / 8;
  static constexpr int DMA_PER_WAVE = kQM * CPR / kThreads;     // 1 KB copies per tile
  static constexpr int KV_DMA_PER_WAVE = kKN * CPR / kThreads;  // for the V tile
  static constexpr bool V_REGS = D < 128;  // V of the wave's keys fits in registers
  // LDS: Q tiles of the two ring stages, their dO tiles, their AUX blocks,
  // then (d = 128) the V tile, then the list of steps.  After the last step the same
  // bytes hold the second waves' partial sums.
  static constexpr int DO_REGION = 2 * TILE_BYTES;
  static constexpr int AUX_REGION = 4 * TILE_BYTES;
  static constexpr int KV_REGION = AUX_REGION + 2 * AUX_BYTES;
  static constexpr int PART_BYTES = kWaves / 2 * 2 * NE * 4 * 1024;
  static constexpr int LIST_REGION = KV_REGION + (V_REGS ? 0 : KT_BYTES);
  static constexpr int RING_BYTES = LIST_REGION + span_max_steps(D) * 4;
  static constexpr int LDS_BYTES = RING_BYTES > PART_BYTES ? RING_BYTES : PART_BYTES;
  static_assert(span_max_steps(D) <= 65536 && LDS_BYTES <= 163840 - 1024, "16 bits, 160 KB");
};

template <int D, bool CAP, bool BIAS>
__device__ __forceinline__ void key_unit(const BwdArgs &a, int L, unsigned char *smem,
                                         int *counts) {
  using C = KvCfg<D>;
  using T = LdsTile<C::LW>;
  uint32_t *list = reinterpret_cast<uint32_t *>(smem + C::LIST_REGION);
  constexpr int kDoRegion = C::DO_REGION, kAuxRegion = C::AUX_REGION, kKvRegion = C::KV_REGION;
  const int S = a.s.S, Sp = a.Sp, Hl = a.s.Hl, Hkl = a.s.Hkl, n_rep = Hl / Hkl;
  const int kvheads_total = a.s.b * Hkl;

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = w & 3, h = w >> 2;  // key block, row half
  const int l32 = lane & 31, hh = lane >> 5;
  const int hb = L % kvheads_total, u = L / kvheads_total;
  const int part = u % a.nsplits, pair = u / a.nsplits;
  const int T128 = a.chunk_rows / kKN;
  int kt, ch;
  if (pair < (int)a.causal_units) {
    kv_unit(pair, a.nchunks, T128, kt, ch);
    if (kt >= a.ktiles) return;  // workgroup-uniform
  } else {  // rows before the keys
    kt = (pair - (int)a.causal_units) % a.ktiles;
    ch = (pair - (int)a.causal_units) / a.ktiles;
    if (kt < (ch + 1) * T128) return;
  }
  const int beta = hb / Hkl, kvh = hb % Hkl;
  const int rep0 = part * n_rep / a.nsplits, rep1 = (part + 1) * n_rep / a.nsplits;
  const int k0 = kt * kKN;
  const int r_lo = ch * a.chunk_rows, r_hi = min(S, r_lo + a.chunk_rows);
  const int wk0 = k0 + 32 * kw;
  const int key = wk0 + l32;

  // The steps that see any of the keys, in order.
  int count = 0;
  {
    const int n = (r_hi - r_lo + kQM - 1) / kQM;
    const SpanHull *hulls = a.hulls + ((size_t)beta * Sp + r_lo) / 32;
    for (int s0 = 0; s0 < n; s0 += kThreads) {
      const int s = s0 + tid;
      uint32_t bits = 0;
      if (s < n) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const SpanHull x = hulls[2 * s + half];
          const int row0 = r_lo + s * kQM + 32 * half;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int j0 = k0 + 32 * k;
            uint32_t kind = x.none(j0, 32) ? 0 : x.full(j0, 32) ? 2 : 1;
            // the bias without a mask is for keys at or before the rows
            if (BIAS && kind == 2 && j0 + 31 > row0) kind = 1;
            bits |= kind << (16 + 2 * (4 * half + k));
          }
        }
      }
      const uint64_t mask = __builtin_amdgcn_ballot_w64(bits != 0);
      __syncthreads();  // counts of the turn before are read
      if (lane == 0) counts[w] = __builtin_popcountll(mask);
      __syncthreads();
      int at = count;
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        if (x < w) at += counts[x];
        count += counts[x];
      }
      if (bits != 0)
        list[at + __builtin_popcountll(mask & ((1ull << lane) - 1))] = bits | (uint32_t)s;
    }
    count = __builtin_amdgcn_readfirstlane(count);
    __syncthreads();
  }
  const int slot_index = ch * a.nsplits + part;
  if (a.touched) {
    if (tid == 0)
      a.touched[((size_t)slot_index * kvheads_total + hb) * a.ktiles + kt] = count > 0;
    if (count == 0) return;
  }

  const uint32_t q_row_bytes = a.s.q.row_elems * 2, do_row_bytes = (uint32_t)(Hl * D) * 2;
  const uint32_t k_row_bytes = a.s.k.row_elems * 2, v_row_bytes = a.s.v.row_elems * 2;
  const uint32_t smem_lds = lds_addr_of(smem);
  constexpr bool kVRegs = C::V_REGS;
  bf16x8 kf[C::NS], vf[kVRegs ? C::NS : 1];
  {
    const uint16_t *kp = a.s.k.p + ((size_t)beta * S + k0) * a.s.k.row_elems + (size_t)kvh * D;
    const uint16_t *vp = a.s.v.p + ((size_t)beta * S + k0) * a.s.v.row_elems + (size_t)kvh * D;
    const rsrc_t rk = make_rsrc(kp, (uint32_t)(S - k0) * k_row_bytes);
#pragma unroll
    for (int s = 0; s < C::NS; ++s)
      kf[s] = as_bf16x8(buf_load16(rk, (uint32_t)(key - k0) * k_row_bytes + (2 * s + hh) * 16));
    if constexpr (kVRegs) {
      const rsrc_t rv = make_rsrc(vp, (uint32_t)(S - k0) * v_row_bytes);
#pragma unroll
      for (int s = 0; s < C::NS; ++s)
        vf[s] = as_bf16x8(buf_load16(rv, (uint32_t)(key - k0) * v_row_bytes + (2 * s + hh) * 16));
    }
    wait_vmcnt<0>();  // retire the tracked loads before untracked copies start
    if constexpr (!kVRegs) {
      const u32x4 rv = make_rsrc_words(vp, (uint32_t)(S - k0) * v_row_bytes);
#pragma unroll
      for (int i = 0; i < C::KV_DMA_PER_WAVE; ++i) {
        const int pos = (w * C::KV_DMA_PER_WAVE + i) * 64 + lane;
        copy16_to_lds(rv, dma_src_off<C::LW, D>(pos, v_row_bytes),
                             smem_lds + kKvRegion + (w * C::KV_DMA_PER_WAVE + i) * 1024);
      }
    }
  }

  f32x16 accv[C::NE], acck[C::NE];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        accv[n][r] = 0.f;
        acck[n][r] = 0.f;
      }
  };
  clear();

  const CopySource<C::LW, D, C::DMA_PER_WAVE> src(w, lane);
  // Rows of Q and dO; a row of the V tile lies as far from them as the wave's keys from
  // its half.
  int a_off[C::NS];
#pragma unroll
  for (int s = 0; s < C::NS; ++s) {
    a_off[s] = T::off(32 * h + l32, 2 * s + hh);
    asm volatile("" : "+v"(a_off[s]));
  }
  const int to_v = kKvRegion + 32 * (kw - h) * T::ROW_BYTES;
  // Transposed rows 32h + 4hh (+ 16, and + 8 in the operand's second half) of columns
  // 16((lane/16)%2): 32 n columns on, and 8 rows, the swizzle flips bits of the offset.
  int t_base = tr_piece_off<C::LW>(32 * h + 4 * hh, 16 * ((lane >> 4) & 1), lane);
  asm volatile("" : "+v"(t_base));
  auto transposed = [&](const unsigned char *tile, int n, int s2) __attribute__((always_inline)) {
    const int lo = t_base ^ (64 * n), hi = lo ^ 32, ro = s2 * 16 * T::ROW_BYTES;
    return tr_operand(tile, lo + ro, hi + 8 * T::ROW_BYTES + ro);
  };
  int aux_lane = kAuxRegion + 4 * 32 * h + 16 * hh;
  asm volatile("" : "+v"(aux_lane));

  // Keeps the compiler from holding derived addresses in registers of their own.
  auto launder_offsets = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < C::NS; ++s) {
      asm volatile("" : "+v"(a_off[s]));
    }
    asm volatile("" : "+v"(t_base));
    asm volatile("" : "+v"(aux_lane));
  };

  // Copies of step s of the head whose resources are at hand.  Wave 0 copies the
  // rows' planes, wave 1 their spans.
  constexpr uint32_t kAuxBytes = 256 * kPlanes<BIAS>;
  u32x4 rq, rd, ra;
  float sl = 0.f;
  auto head_resources = [&](int hq) __attribute__((always_inline)) {
    rq = make_rsrc_words(a.s.q.p + ((size_t)beta * S + r_lo) * a.s.q.row_elems + (size_t)hq * D,
                         (uint32_t)(S - r_lo) * q_row_bytes);
    rd = make_rsrc_words(a.d_o + (((size_t)beta * S + r_lo) * Hl + hq) * D,
                         (uint32_t)(S - r_lo) * do_row_bytes);
    if (w == 0)
      ra = make_rsrc_words(a.aux + (((size_t)beta * Hl + hq) * Sp + r_lo) * kPlanes<BIAS>,
                           (uint32_t)(Sp - r_lo) * 4 * kPlanes<BIAS>);
    else
      ra = make_rsrc_words(a.rows + ((size_t)beta * Sp + r_lo) * kPlanes<BIAS>,
                           (uint32_t)(Sp - r_lo) * 4 * kPlanes<BIAS>);
  };
  auto load_step = [&](int st, uint32_t s) __attribute__((always_inline)) {
    const uint32_t sq = (uint32_t)st & 1;
    const uint32_t stage = smem_lds + sq * C::TILE_BYTES;
    const uint32_t qb = s * kQM * q_row_bytes, db = s * kQM * do_row_bytes;
#pragma unroll
    for (int i = 0; i < C::DMA_PER_WAVE; ++i) {
      const uint32_t lds = stage + (w * C::DMA_PER_WAVE + i) * 1024;
      copy16_to_lds(rq, src.off(i, q_row_bytes) + qb, lds);
      copy16_to_lds(rd, src.off(i, do_row_bytes) + db, lds + kDoRegion);
    }
    if (w < 2)
      copy16_to_lds(ra, (16u * lane < kAuxBytes ? 16u * lane : kZeroOffset) + s * kAuxBytes,
                           smem_lds + kAuxRegion + sq * C::AUX_BYTES + 1024 * w);
  };
  auto aux_rows = [&](int stg, int which) __attribute__((always_inline)) {
    const unsigned char *src = smem + aux_lane + stg * C::AUX_BYTES + 256 * which;
    f32x16 v;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(src + 4 * 8 * g);
#pragma unroll
      for (int y = 0; y < 4; ++y) v[4 * g + y] = x[y];
    }
    return v;
  };
  const float c = a.s.scale * kSpanLog2e;
  const float c1 = CAP ? 2.f * c / a.s.cap : 0.f, cap2 = CAP ? a.s.cap * kSpanLog2e : 0.f;

  const float rc = 1.f / c;
  // One step's half for this wave.  What a mask and a bias of both signs take is put
  // into the scores (with a cap: into what their exponents start from) behind one
  // branch, so that everything else, and above all the accumulators, exists once.
  auto step = [&](int stg, int row0, bool edge, auto careful_tag) __attribute__((always_inline)) {
    constexpr bool CAREFUL = decltype(careful_tag)::value;
    const unsigned char *Qs = smem + stg * C::TILE_BYTES, *dOs = Qs + kDoRegion;
    f32x16 sacc, pacc;
    {
      const f32x16 negd = aux_rows(stg, 1);
      f32x16 neglse;
      if constexpr (CAP) neglse = f32x16{};
      else neglse = aux_rows(stg, BIAS && edge ? 2 : 0);
#pragma unroll
      for (int s = 0; s < C::NS; ++s) {
        const bf16x8 aq = *reinterpret_cast<const bf16x8 *>(Qs + a_off[s]);
        const bf16x8 ad = *reinterpret_cast<const bf16x8 *>(dOs + a_off[s]);
        bf16x8 bv;
        if constexpr (kVRegs) bv = vf[s];
        else bv = *reinterpret_cast<const bf16x8 *>(smem + (a_off[s] + to_v));
        sacc = mfma32x32x16(aq, kf[s], s == 0 ? neglse : sacc);
        pacc = mfma32x32x16(ad, bv, s == 0 ? negd : pacc);
      }
    }
    bf16x8 bp[2], bds[2];
    constexpr uint32_t kOnes = 0x3F803F80u;
    u32x4 seen[2] = {{kOnes, kOnes, kOnes, kOnes}, {kOnes, kOnes, kOnes, kOnes}};
    {
      f32x16 neglse;
      if constexpr (CAP) neglse = aux_rows(stg, BIAS && edge ? 2 : 0);
      // row0: first row of the wave's half
      float base = BIAS ? sl * (float)(key - (row0 - 32 * h)) : 0.f;
      if (edge) {  // wave-uniform
        asm volatile("" ::: "memory");
        const float ahead = (float)(row0 + 4 * hh - key);
        constexpr int kRow = 4 * kPlanes<BIAS>;
        const unsigned char *spans = smem + stg * C::AUX_BYTES + kAuxRegion + 1024 + kRow * 32 * h +
                                     kRow * 4 * hh;
        base = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int io = 8 * (r >> 2) + (r & 3);
          const u32x2 span = *reinterpret_cast<const u32x2 *>(spans + kRow * io);
          const bool vis = key - span.x < span.y - span.x;
          const float bias = BIAS ? -fabsf(ahead + (float)io) : 0.f;
          if constexpr (CAP) {
            neglse[r] = vis ? fmaf(sl, bias, neglse[r]) : -INFINITY;
            sacc[r] = vis ? sacc[r] : 0.f;
          } else {
            sacc[r] = vis ? fmaf(sl * rc, bias, sacc[r]) : -INFINITY;
          }
          pacc[r] = vis ? pacc[r] : 0.f;
          if (CAREFUL && !vis) seen[r / 8][r % 8 / 2] &= r % 2 ? 0xFFFFu : 0xFFFF0000u;
        }
        asm volatile("" ::: "memory");
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (CAP) {
          const float rr = cap_r(sacc[r], c1);
          sacc[r] = fast_exp2(fmaf(rr, -2.f * cap2, neglse[r] + (cap2 + base)));
          pacc[r] = sacc[r] * pacc[r] * fmaf(-rr, rr, rr);
        } else {
          sacc[r] = fast_exp2(fmaf(sacc[r], c, base));
          pacc[r] = sacc[r] * pacc[r];
        }
      }
      pack16(sacc, bp);
      pack16(pacc, bds);
    }
    wave_priority<1>();
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        bf16x8 av = transposed(dOs, n, s2);
        if constexpr (CAREFUL) av = finite_operand(av, seen[s2], accv[n]);
        accv[n] = mfma32x32x16(av, bp[s2], accv[n]);
        bf16x8 ak = transposed(Qs, n, s2);
        if constexpr (CAREFUL) ak = finite_operand(ak, seen[s2], acck[n]);
        acck[n] = mfma32x32x16(ak, bds[s2], acck[n]);
      }
    if constexpr (!CAREFUL) sched_reads_ahead<4 * C::NE, 2, 4>();
    __builtin_amdgcn_sched_barrier(0);
    wave_priority<0>();
  };
  using No = std::false_type;
  using Yes = std::true_type;
  auto sweep = [&](auto careful_tag) __attribute__((always_inline)) {
    const int heads = rep1 - rep0;
    const int n = count * heads;
    int ld_i = 0, ld_h = rep0;  // the next step to copy
    auto load_next = [&](int st) __attribute__((always_inline)) {
      if (ld_h >= rep1) return;
      if (ld_i == 0) head_resources(kvh * n_rep + ld_h);
      load_step(st, (uint32_t)__builtin_amdgcn_readfirstlane((int)list[ld_i]) & 0xFFFFu);
      if (++ld_i == count) ld_i = 0, ++ld_h;
    };
    if (n > 0) load_next(0);
    int i = 0, hr = rep0;
    auto turn = [&](int st, auto stage_tag) __attribute__((always_inline)) {
      constexpr int STG = decltype(stage_tag)::value;  // st % 2
      const uint32_t e = (uint32_t)__builtin_amdgcn_readfirstlane((int)list[i]);
      if constexpr (BIAS)
        if (i == 0) sl = a.s.slopes[kvh * n_rep + hr] * kSpanLog2e;
      launder_offsets();
      wait_vmcnt<0>();
      barrier_no_fence();
      load_next(st + 1);
      const int row0 = r_lo + (int)(e & 0xFFFFu) * kQM + 32 * h;
      const uint32_t kind = (e >> (16 + 2 * (4 * h + kw))) & 3u;
      if (kind != 0) step(STG, row0, kind == 1, careful_tag);
      if (++i == count) i = 0, ++hr;
    };
    // Two stages: step st's copies landed, then the barrier, after which the
    // other stage is free.  Every operand address is a lane's offset plus an
    // immediate.
    for (int st = 0; st < n; st += 2) {
      turn(st, std::integral_constant<int, 0>{});
      if (st + 1 < n) turn(st + 1, std::integral_constant<int, 1>{});
    }
  };
  sweep(No{});
  wait_vmcnt<0>();  // without a step nothing has waited for the V tile yet
  // dK or dV of no finite value anywhere in the unit: infinities or NaN in Q or
  // dO, which 0 * them may have carried to keys that their rows do not see.
  {
    float z = 0.f;
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        z = fmaf(0.f, accv[n][r], z);
        z = fmaf(0.f, acck[n][r], z);
      }
    if (__syncthreads_or(!(z == 0.f))) {
      clear();
      sweep(Yes{});
      __syncthreads();
    }
  }

  // The pair's partial sums (waves w and w + 4): the second waves put theirs in
  // LDS, the first add them.
  auto slot = [&](int tensor, int n, int g) __attribute__((always_inline)) {
    return smem + (((kw * 2 + tensor) * C::NE + n) * 4 + g) * 1024 + 16 * lane;
  };
  if (h == 1) {
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        *reinterpret_cast<f32x4 *>(slot(0, n, g)) =
            f32x4{accv[n][4 * g], accv[n][4 * g + 1], accv[n][4 * g + 2], accv[n][4 * g + 3]};
        *reinterpret_cast<f32x4 *>(slot(1, n, g)) =
            f32x4{acck[n][4 * g], acck[n][4 * g + 1], acck[n][4 * g + 2], acck[n][4 * g + 3]};
      }
  }
  __syncthreads();
  if (h == 1 || key >= S) return;
  const float dk_scale = a.s.scale * (CAP ? 4.f : 1.f);
  const size_t e0 = (((size_t)beta * S + key) * Hkl + kvh) * D;
  const bool direct = a.touched == nullptr;
  void *ov = direct ? a.dv : a.dv_part + (size_t)slot_index * a.part_elems;
  void *ok = direct ? a.dk : a.dk_part + (size_t)slot_index * a.part_elems;
  const int bf = direct ? a.grad_bf16 : 0;
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (32 * n + 8 * g >= D) continue;  // padding columns
      const f32x4 pv = *reinterpret_cast<const f32x4 *>(slot(0, n, g));
      const f32x4 pk = *reinterpret_cast<const f32x4 *>(slot(1, n, g));
      const size_t e = e0 + 32 * n + 8 * g + 4 * hh;
      store4(ov, e, f32x4{accv[n][4 * g] + pv[0], accv[n][4 * g + 1] + pv[1],
                          accv[n][4 * g + 2] + pv[2], accv[n][4 * g + 3] + pv[3]}, bf);
      store4(ok, e, f32x4{(acck[n][4 * g] + pk[0]) * dk_scale,
                          (acck[n][4 * g + 1] + pk[1]) * dk_scale,
                          (acck[n][4 * g + 2] + pk[2]) * dk_scale,
                          (acck[n][4 * g + 3] + pk[3]) * dk_scale}, bf);
    }
}

// ------------------------------------------------------------- span_reduce
// dK or dV (grid.z) of a key = the sum of the slots whose unit saw it, in order.  One
// thread per 4 consecutive elements.
__global__ __launch_bounds__(kPreThreads) void span_reduce_kernel(const BwdArgs a,
                                                                  uint32_t row_quads,
                                                                  FastDiv by_row_quads,
                                                                  uint32_t seq_quads, int d4,
                                                                  FastDiv by_d4) {
  const uint32_t i = blockIdx.x * kPreThreads + threadIdx.x;
  if (i >= seq_quads) return;
  const int beta = blockIdx.y;
  const uint32_t key = by_row_quads.div(i), kvh = by_d4.div(i - key * row_quads);
  const size_t e = ((size_t)beta * seq_quads + i) * 4;
  const float *part = (blockIdx.z ? a.dv_part : a.dk_part) + e;
  const int kt = (int)(key / kKN), heads = a.s.b * a.s.Hkl;
  const int *touched = a.touched + (size_t)(beta * a.s.Hkl + (int)kvh) * a.ktiles + kt;
  // causal: chunks of rows before the keys have no unit
  const int first = a.s.spans ? 0 : (int)(key / a.chunk_rows) * a.nsplits;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s = first; s < a.nchunks * a.nsplits; ++s)
    if (touched[(size_t)s * heads * a.ktiles]) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(part + (size_t)s * a.part_elems);
#pragma unroll
      for (int y = 0; y < 4; ++y) acc[y] += x[y];
    }
  store4(blockIdx.z ? a.dv : a.dk, e, acc, a.grad_bf16);
}

// ---------------------------------------------------------------- dQ pass
template <int D, int RG>
struct DqCfg {
  static constexpr int R = RG, P = kWaves / R;
  static constexpr int DC = HeadDim<D>::DC;
  static constexpr int LW = HeadDim<D>::LW;
  static constexpr int BM = 32 * R;                  // query rows per workgroup
  static constexpr int KM = P == 1 ? 2 : 1;          // 32-key blocks per wave and tile
  static constexpr int BN = 32 * KM * P;             // keys per tile
  static constexpr int TILE_BYTES = BN * LW * 2;
  static constexpr int STAGE_BYTES = 2 * TILE_BYTES;  // K, V
  static constexpr int STAGES = STAGE_BYTES > 32768 ? 2 : 4;
  static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
  static constexpr int NS = D / 16;
  static constexpr int NE = DC / 32;
  static constexpr int CPR = LW / 8;
  static constexpr int DMA_PER_WAVE = BN * CPR / kThreads;
  static_assert((P - 1) * R * NE * 4096 <= LDS_BYTES, "the parts' dQ fit the ring");
};

template <int D, int R, bool CAP, bool BIAS>
__device__ __forceinline__ void dq_tile(const BwdArgs &a, int L, unsigned char *smem,
                                        int *scratch) {
  using C = DqCfg<D, R>;
  using T = LdsTile<C::LW>;
  constexpr int kSt = C::STAGES, kVRegion = kSt * C::TILE_BYTES;
  const int S = a.s.S, Hl = a.s.Hl, heads_total = a.s.b * Hl;
  const int qtiles = (S + C::BM - 1) / C::BM;

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hh = lane >> 5;
  const int qt = qtiles - 1 - L / heads_total;
  const int hb = L % heads_total;
  const int beta = hb / Hl, h = hb % Hl, kvh = h / (Hl / a.s.Hkl);
  const int q0 = qt * C::BM;
  const int rg = w % R, part = w / R;  // row group, key part
  const int wrow0 = q0 + 32 * rg;
  const int row = wrow0 + l32;

  const uint32_t q_row_bytes = a.s.q.row_elems * 2, do_row_bytes = (uint32_t)(Hl * D) * 2;
  const uint32_t k_row_bytes = a.s.k.row_elems * 2, v_row_bytes = a.s.v.row_elems * 2;
  const rsrc_t rq = make_rsrc(a.s.q.p + ((size_t)beta * S + q0) * a.s.q.row_elems + (size_t)h * D,
                              (uint32_t)(S - q0) * q_row_bytes);
  const rsrc_t rd = make_rsrc(a.d_o + (((size_t)beta * S + q0) * Hl + h) * D,
                              (uint32_t)(S - q0) * do_row_bytes);
  const u32x4 rk = make_rsrc_words(a.s.k.p + (size_t)beta * S * a.s.k.row_elems + (size_t)kvh * D,
                                   (uint32_t)S * k_row_bytes);
  const u32x4 rv = make_rsrc_words(a.s.v.p + (size_t)beta * S * a.s.v.row_elems + (size_t)kvh * D,
                                   (uint32_t)S * v_row_bytes);
  const uint32_t smem_lds = lds_addr_of(smem);

  bf16x8 qf[C::NS], df[C::NS];
#pragma unroll
  for (int s = 0; s < C::NS; ++s) {
    qf[s] = as_bf16x8(buf_load16(rq, (uint32_t)(row - q0) * q_row_bytes + (2 * s + hh) * 16));
    df[s] = as_bf16x8(buf_load16(rd, (uint32_t)(row - q0) * do_row_bytes + (2 * s + hh) * 16));
  }
  int lo = 0, hi = 0;
  float nlse = -INFINITY, nd = 0.f;  // rows that see nothing, and past S: P = 0
  if (row < S) {
    span_of(a.s.spans, beta, S, row, lo, hi);
    if (hi > lo) nlse = -a.lse[((size_t)beta * Hl + h) * S + row] * kSpanLog2e;
    nd = a.aux[(((size_t)beta * Hl + h) * a.Sp + row / 64 * 64) * kPlanes<BIAS> + 64 +
               row % 64];
  }
  float sl = 0.f;
  if constexpr (BIAS) sl = a.s.slopes[h] * kSpanLog2e;
  // dP^T starts from -D (the accumulator's initial value), so dU = P dP'.
  f32x16 negd;
#pragma unroll
  for (int r = 0; r < 16; ++r) negd[r] = nd;
  const SpanHull wh = wave_hull(hull_of(lo, hi, row < S));
  if (lane == 0) scratch[w] = wh.any_lo, scratch[kWaves + w] = wh.any_hi;
  wait_vmcnt<0>();  // retire the tracked loads before untracked copies start
  __syncthreads();
  int wg_lo = scratch[0], wg_hi = scratch[kWaves];
#pragma unroll
  for (int i = 1; i < R; ++i) {
    wg_lo = min(wg_lo, scratch[i]);
    wg_hi = max(wg_hi, scratch[kWaves + i]);
  }
  wg_lo = __builtin_amdgcn_readfirstlane(wg_lo);
  wg_hi = __builtin_amdgcn_readfirstlane(wg_hi);
  const int t0 = wg_lo < wg_hi ? wg_lo / C::BN : 0;
  const int nt = wg_lo < wg_hi ? (wg_hi + C::BN - 1) / C::BN - t0 : 0;

  uint32_t gk[C::DMA_PER_WAVE], gv[C::DMA_PER_WAVE];
#pragma unroll
  for (int i = 0; i < C::DMA_PER_WAVE; ++i) {
    gk[i] = dma_src_off<C::LW, D>((w * C::DMA_PER_WAVE + i) * 64 + lane, k_row_bytes);
    gv[i] = dma_src_off<C::LW, D>((w * C::DMA_PER_WAVE + i) * 64 + lane, v_row_bytes);
  }
  auto load_tile = [&](int u) __attribute__((always_inline)) {
    const uint32_t ks = smem_lds + (u % kSt) * C::TILE_BYTES;
    const uint32_t kb = (uint32_t)((t0 + u) * C::BN) * k_row_bytes;
    const uint32_t vb = (uint32_t)((t0 + u) * C::BN) * v_row_bytes;
#pragma unroll
    for (int i = 0; i < C::DMA_PER_WAVE; ++i) {
      const uint32_t lds = ks + (w * C::DMA_PER_WAVE + i) * 1024;
      copy16_to_lds(rk, kb + gk[i], lds);
      copy16_to_lds(rv, vb + gv[i], lds + kVRegion);
    }
  };
  const int part_off = part * 32 * C::KM * T::ROW_BYTES;
  int a_off[C::NS], v_off[C::NS];
#pragma unroll
  for (int s = 0; s < C::NS; ++s) {
    a_off[s] = T::off(l32, 2 * s + hh) + part_off;
    asm volatile("" : "+v"(a_off[s]));
    v_off[s] = a_off[s] + kVRegion;
    asm volatile("" : "+v"(v_off[s]));
  }
  int t_off[C::NE][2];
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      t_off[n][x] =
          tr_piece_off<C::LW>(4 * hh + 8 * x, 32 * n + 16 * ((lane >> 4) & 1), lane) + part_off;
      asm volatile("" : "+v"(t_off[n][x]));
    }
  const float c = a.s.scale * kSpanLog2e;
  const float c1 = CAP ? 2.f * c / a.s.cap : 0.f, cap2 = CAP ? a.s.cap * kSpanLog2e : 0.f;

  f32x16 qacc[C::NE];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) qacc[n][r] = 0.f;
  };
  clear();
  const float rc = 1.f / c;
  auto tile = [&](int u, int st, bool edge, auto careful_tag)  // st: u % kSt
                  __attribute__((always_inline)) {
    constexpr bool CAREFUL = decltype(careful_tag)::value;
    const int j0 = (t0 + u) * C::BN + 32 * C::KM * part;
    const unsigned char *Ks = smem + st * C::TILE_BYTES;
#pragma unroll
    for (int m = 0; m < C::KM; ++m) {
      f32x16 sacc, pacc;
#pragma unroll
      for (int s = 0; s < C::NS; ++s) {
        const bf16x8 ak = *reinterpret_cast<const bf16x8 *>(Ks + a_off[s] + m * 32 * T::ROW_BYTES);
        const bf16x8 av = *reinterpret_cast<const bf16x8 *>(Ks + v_off[s] + m * 32 * T::ROW_BYTES);
        sacc = mfma32x32x16(ak, qf[s], s == 0 ? f32x16{} : sacc);
        pacc = mfma32x32x16(av, df[s], s == 0 ? negd : pacc);
      }
      sched_reads_ahead<2 * C::NS, 1, 4>();
      const int jl = j0 + 32 * m + 4 * hh;
      const float ahead = (float)(row - jl);
      // not an edge: all keys on one side of the rows
      float slp = j0 + 32 * m > wrow0 ? -sl : sl;
      float base = BIAS ? fmaf(-slp, ahead, nlse) : nlse;
      constexpr uint32_t kOnes = 0x3F803F80u;
      u32x4 seen[2] = {{kOnes, kOnes, kOnes, kOnes}, {kOnes, kOnes, kOnes, kOnes}};
      f32x16 add;  // with a cap and a bias
      if constexpr (CAP && BIAS) {
#pragma unroll
        for (int r = 0; r < 16; ++r) add[r] = fmaf(slp, (float)(8 * (r >> 2) + (r & 3)), base) + cap2;
      }
      if (edge) {  // wave-uniform; as in the key pass
        asm volatile("" ::: "memory");
        const int past = jl - lo;
        slp = 0.f;
        base = nlse;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int jo = 8 * (r >> 2) + (r & 3);
          const bool vis = (uint32_t)(past + jo) < (uint32_t)(hi - lo);
          const float dist = BIAS ? fabsf(ahead - (float)jo) : 0.f;
          if constexpr (CAP && BIAS) {
            add[r] = vis ? fmaf(-sl, dist, nlse + cap2) : -INFINITY;
            sacc[r] = vis ? sacc[r] : 0.f;
          } else if constexpr (BIAS) {
            sacc[r] = vis ? fmaf(-sl * rc, dist, sacc[r]) : -INFINITY;
          } else {  // with a cap P is at most 1 there: no LSE is below -cap
            sacc[r] = vis ? sacc[r] : -INFINITY;
          }
          pacc[r] = vis ? pacc[r] : 0.f;
          if (CAREFUL && !vis) seen[r / 8][r % 8 / 2] &= r % 2 ? 0xFFFFu : 0xFFFF0000u;
        }
        asm volatile("" ::: "memory");
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (CAP) {
          const float rr = cap_r(sacc[r], c1);
          const float p = fast_exp2(fmaf(rr, -2.f * cap2, BIAS ? add[r] : base + cap2));
          pacc[r] = p * pacc[r] * fmaf(-rr, rr, rr);
        } else {
          const int jo = 8 * (r >> 2) + (r & 3);
          const float b = BIAS ? fmaf(slp, (float)jo, base) : base;
          pacc[r] = fast_exp2(fmaf(sacc[r], c, b)) * pacc[r];
        }
      }
      bf16x8 sb[2];
      pack16(pacc, sb);
      wave_priority<1>();
#pragma unroll
      for (int n = 0; n < C::NE; ++n)
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          const int ro = (2 * m + s2) * 16 * T::ROW_BYTES;
          bf16x8 x = tr_operand(Ks, t_off[n][0] + ro, t_off[n][1] + ro);
          if constexpr (CAREFUL) x = finite_operand(x, seen[s2], qacc[n]);
          qacc[n] = mfma32x32x16(x, sb[s2], qacc[n]);
        }
      if constexpr (!CAREFUL) sched_reads_ahead<2 * C::NE, 2, 4>();
      __builtin_amdgcn_sched_barrier(0);
      wave_priority<0>();
    }
  };
  auto begin_tile = [&](int u) __attribute__((always_inline)) {
    if constexpr (kSt == 4) {
      if (u + 2 < nt) {
        load_tile(u + 2);
        wait_vmcnt<4 * C::DMA_PER_WAVE>();
      } else {
        wait_vmcnt<0>();
      }
      barrier_no_fence();
    } else {
      wait_vmcnt<0>();
      barrier_no_fence();
      if (u + 1 < nt) load_tile(u + 1);
    }
  };
  using No = std::false_type;
  using Yes = std::true_type;
  constexpr int kWaveKeys = 32 * C::KM;
  for (int u = 0; u < kSt / 2 && u < nt; ++u) load_tile(u);
  auto take = [&](int u, int st, auto careful_tag) __attribute__((always_inline)) {
    const int j0 = (t0 + u) * C::BN + kWaveKeys * part;
    if (wh.none(j0, kWaveKeys)) return;  // wave-uniform
    const bool crosses = BIAS && j0 + kWaveKeys - 1 > wrow0 && j0 < wrow0 + 31;
    tile(u, st, !wh.full(j0, kWaveKeys) || crosses, careful_tag);
  };
  for (int u0 = 0; u0 < nt; u0 += kSt)
#pragma unroll
    for (int st = 0; st < kSt; ++st)
      if (u0 + st < nt) {
        begin_tile(u0 + st);
        take(u0 + st, st, No{});
      }
  // As in the key pass: infinities or NaN in K.
  {
    float z = 0.f;
#pragma unroll
    for (int n = 0; n < C::NE; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) z = fmaf(0.f, qacc[n][r], z);
    if (__syncthreads_or(!(z == 0.f))) {
      clear();
      for (int u = 0; u < nt; ++u) {
        barrier_no_fence();
        load_tile(u);
        wait_vmcnt<0>();
        barrier_no_fence();
        take(u, u % kSt, Yes{});
      }
      __syncthreads();
    }
  }

  if constexpr (C::P > 1) {
    // The parts' sums: parts 1 .. P-1 put theirs in LDS, part 0 adds them in order.
    auto slot = [&](int p, int n, int g) __attribute__((always_inline)) {
      return smem + ((((p - 1) * R + rg) * C::NE + n) * 4 + g) * 1024 + 16 * lane;
    };
    if (part > 0) {
#pragma unroll
      for (int n = 0; n < C::NE; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4 *>(slot(part, n, g)) =
              f32x4{qacc[n][4 * g], qacc[n][4 * g + 1], qacc[n][4 * g + 2], qacc[n][4 * g + 3]};
    }
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int p = 1; p < C::P; ++p)
#pragma unroll
      for (int n = 0; n < C::NE; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 x = *reinterpret_cast<const f32x4 *>(slot(p, n, g));
#pragma unroll
          for (int y = 0; y < 4; ++y) qacc[n][4 * g + y] += x[y];
        }
  }
  if (row >= S) return;
  const float scale = a.s.scale * (CAP ? 4.f : 1.f);
  const size_t e0 = (((size_t)beta * S + row) * Hl + h) * D;
#pragma unroll
  for (int n = 0; n < C::NE; ++n)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (32 * n + 8 * g >= D) continue;  // padding columns
      store4(a.dq, e0 + 32 * n + 8 * g + 4 * hh,
             f32x4{qacc[n][4 * g] * scale, qacc[n][4 * g + 1] * scale, qacc[n][4 * g + 2] * scale,
                   qacc[n][4 * g + 3] * scale}, a.grad_bf16);
    }
}

// Both passes in one launch: neither reads what the other writes.
template <int D, int R, bool CAP, bool BIAS>
__global__ __launch_bounds__(kThreads, 1) void span_main_kernel(const BwdArgs a) {
  constexpr int kKvLds = KvCfg<D>::LDS_BYTES, kDqLds = DqCfg<D, R>::LDS_BYTES;
  __shared__ __attribute__((aligned(16))) unsigned char smem[kKvLds > kDqLds ? kKvLds : kDqLds];
  __shared__ int scratch[2 * kWaves];
  const uint32_t kv_blocks = gridDim.x - a.dq_blocks;
  const uint32_t first = a.keys_first ? kv_blocks : a.dq_blocks;
  const uint32_t i = blockIdx.x < first ? blockIdx.x : blockIdx.x - first;
  if ((blockIdx.x < first) == (a.keys_first != 0))  // workgroup-uniform
    key_unit<D, CAP, BIAS>(a, (int)i, smem, scratch);
  else
    dq_tile<D, R, CAP, BIAS>(a, (int)i, smem, scratch);
}

}  // namespace

hipError_t launch_span_bwd(const SpanArgs &s, const uint16_t *o, const float *lse,
                           const uint16_t *d_o, void *dq, void *dk, void *dv, bool grad_bf16,
                           void *workspace, hipStream_t stream) {
  const SpanCut ck = span_cut(s);
  char *ws = static_cast<char *>(workspace);
  BwdArgs a{};
  a.s = s;
  a.d_o = d_o;
  a.lse = lse;
  a.aux = reinterpret_cast<float *>(ws);
  a.rows = reinterpret_cast<int *>(ws + ck.rows);
  SpanHull *hulls = reinterpret_cast<SpanHull *>(ws + ck.hulls);
  a.hulls = hulls;
  a.dq = dq, a.dk = dk, a.dv = dv;
  a.grad_bf16 = grad_bf16;
  a.Sp = ck.Sp, a.chunk_rows = ck.chunk_rows, a.nchunks = ck.nchunks, a.nsplits = ck.nsplits;
  a.ktiles = ck.ktiles;
  a.part_elems = (size_t)s.b * s.S * s.Hkl * s.d;
  const int slots = ck.nchunks * ck.nsplits;
  if (slots > 1) {
    a.touched = reinterpret_cast<int *>(ws + ck.touched);
    a.dk_part = reinterpret_cast<float *>(ws + ck.parts);
    a.dv_part = a.dk_part + slots * a.part_elems;
  }
  const int T128 = ck.chunk_rows / kKN;
  a.causal_units = (uint32_t)kv_units(ck.nchunks, T128);
  const int R = span_row_groups(s);
  a.dq_blocks = (uint32_t)span_dq_blocks(s);
  const uint32_t kv_blocks = (uint32_t)span_key_blocks(s, ck);
  {
    const int n_rep = s.Hl / s.Hkl;
    const long long unit = (long long)(ck.chunk_rows / 64) * ((n_rep + ck.nsplits - 1) / ck.nsplits);
    a.keys_first = unit * 1024 > 3LL * R * s.S;
  }
  const long long rows = (long long)s.b * ck.Sp * s.Hl;
  a.pre_rows_blocks = (uint32_t)((rows * (s.d <= 64 ? 8 : 16) + kPreThreads - 1) / kPreThreads);
  const uint32_t hull_blocks =
      (uint32_t)(((long long)s.b * (ck.Sp / 64) + kPreThreads / 64 - 1) / (kPreThreads / 64));

  auto by_rule = [&](auto dim, auto cap, auto bias) {
    constexpr int D = decltype(dim)::value;
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    hipLaunchKernelGGL((span_pre_kernel<D, CAP>), dim3(a.pre_rows_blocks + hull_blocks),
                       dim3(kPreThreads), 0, stream, a, o, hulls);
    const dim3 grid(a.dq_blocks + kv_blocks);
    switch (R) {
      case 2:
        hipLaunchKernelGGL((span_main_kernel<D, 2, CAP, BIAS>), grid, dim3(kThreads), 0, stream, a);
        break;
      case 4:
        hipLaunchKernelGGL((span_main_kernel<D, 4, CAP, BIAS>), grid, dim3(kThreads), 0, stream, a);
        break;
      default:
        hipLaunchKernelGGL((span_main_kernel<D, 8, CAP, BIAS>), grid, dim3(kThreads), 0, stream, a);
    }
  };
  auto by_dim = [&](auto dim) {
    using No = std::false_type;
    using Yes = std::true_type;
    if (s.cap > 0.f) s.slopes ? by_rule(dim, Yes{}, Yes{}) : by_rule(dim, Yes{}, No{});
    else s.slopes ? by_rule(dim, No{}, Yes{}) : by_rule(dim, No{}, No{});
  };
  switch (s.d) {
    case 64: by_dim(std::integral_constant<int, 64>{}); break;
    case 80: by_dim(std::integral_constant<int, 80>{}); break;
    case 96: by_dim(std::integral_constant<int, 96>{}); break;
    default: by_dim(std::integral_constant<int, 128>{}); break;
  }
  if (slots > 1) {
    const uint32_t row_quads = (uint32_t)(s.Hkl * s.d / 4);
    const uint32_t seq_quads = (uint32_t)s.S * row_quads;
    hipLaunchKernelGGL(span_reduce_kernel,
                       dim3((seq_quads + kPreThreads - 1) / kPreThreads, (unsigned)s.b, 2),
                       dim3(kPreThreads), 0, stream, a, row_quads, FastDiv::make(row_quads),
                       seq_quads, s.d / 4, FastDiv::make((uint32_t)s.d / 4));
  }
  return hipGetLastError();
}

}  // namespace basp
