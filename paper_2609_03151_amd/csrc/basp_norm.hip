// basp_norm.hip -- RMS norm of every query and key head and the position
// rotation in one pass, and its backward.
//
// Row x (d elements of one head of one token at position p), weight w:
//   r = 1/sqrt(mean(x^2) + eps),  n = x r w
//   y_a = n_a c - n_b s,  y_b = n_b c + n_a s     (c, s: cos, sin of pair (a, b) at p)
// and with z the transpose of the rotation applied to dy (z_a = dy_a c + dy_b s,
// z_b = dy_b c - dy_a s) and g = z w:
//   dw = sum over rows of z x r,   dx = r (g - x r^2 mean(g x)).
//
// Both kernels are bound by HBM: every row is read once and written once.  A
// row is held by d/8 of a group of 16 lanes (8 at d = 64), eight elements a
// lane, chosen so that both elements of a pair lie in the same lane: four
// pairs, that is two runs of four elements, rot/2 apart or side by side when
// the pairs are interleaved.  Each run is one 8-byte (bf16) or 16-byte (fp32)
// access, and the 16 lanes of a row cover two contiguous stretches of it; the
// rotation then needs no lane exchange, and a pair's cos and sin are loaded
// once (16 bytes of each per lane).  Sums over a row are four DPP adds.  All
// arithmetic is fp32; the one rounding to bf16 is that of the result.
#include <math.h>

#include "basp_device.hpp"
#include "basp_ops.hpp"

namespace basp {

namespace {

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true);
  return x + __builtin_bit_cast(float, y);
}

// Sum over a group of L = 8 or 16 lanes, in every lane: lanes 1 and 2 away
// (quad_perm), then the mirrored half row and row, whose lanes hold the other
// half's sum by then.
template <int L>
__device__ __forceinline__ float group_sum(float x) {
  x = dpp_add<0xB1>(x);
  x = dpp_add<0x4E>(x);
  x = dpp_add<0x141>(x);
  if (L == 16) x = dpp_add<0x140>(x);
  return x;
}

// Four elements in fp32.  NT: read with the non-temporal hint.
__device__ __forceinline__ f32x4 widen(u32x2 v) {
  return f32x4{__builtin_bit_cast(float, v.x << 16), __builtin_bit_cast(float, v.x & 0xFFFF0000u),
               __builtin_bit_cast(float, v.y << 16), __builtin_bit_cast(float, v.y & 0xFFFF0000u)};
}
__device__ __forceinline__ f32x4 load4(const float *p) {
  return *reinterpret_cast<const f32x4 *>(p);
}
template <bool NT>
__device__ __forceinline__ f32x4 load4(const uint16_t *p) {
  const u32x2 *q = reinterpret_cast<const u32x2 *>(p);
  return widen(NT ? __builtin_nontemporal_load(q) : *q);
}
template <bool NT>
__device__ __forceinline__ f32x4 load4(const float *p) {
  const f32x4 *q = reinterpret_cast<const f32x4 *>(p);
  return NT ? __builtin_nontemporal_load(q) : *q;
}
__device__ __forceinline__ void store4(uint16_t *p, f32x4 v) {
  __builtin_nontemporal_store(u32x2{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)},
                              reinterpret_cast<u32x2 *>(p));
}
__device__ __forceinline__ void store4(float *p, f32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<f32x4 *>(p));
}

// The elements of a row that a lane holds: runs [a, a+4) and [b, b+4), and the
// first of the four pairs (a column of the cos and sin tables), or turns =
// false where they are not rotated.
struct LaneCols {
  int a, b, pair;
  bool turns;
};
template <bool INTER>
__device__ __forceinline__ LaneCols lane_cols(int m, int rot) {
  LaneCols c;
  c.pair = 4 * m;
  c.turns = c.pair < rot / 2;
  if (INTER || !c.turns) {
    // side by side; past the rotated elements both orders are the same
    c.a = 8 * m;
    c.b = 8 * m + 4;
  } else {
    c.a = c.pair;
    c.b = c.pair + rot / 2;
  }
  return c;
}

// (a, b) turned by (c, s); the transpose is the turn by (c, -s).
template <bool INTER>
__device__ __forceinline__ void turn(f32x4 &a, f32x4 &b, f32x4 c, f32x4 s) {
  const f32x4 x = a, y = b;
  if (INTER) {
    a = f32x4{x.x * c.x - x.y * s.x, x.y * c.x + x.x * s.x, x.z * c.y - x.w * s.y,
              x.w * c.y + x.z * s.y};
    b = f32x4{y.x * c.z - y.y * s.z, y.y * c.z + y.x * s.z, y.z * c.w - y.w * s.w,
              y.w * c.w + y.z * s.w};
  } else {
    a = f32x4{x.x * c.x - y.x * s.x, x.y * c.y - y.y * s.y, x.z * c.z - y.z * s.z,
              x.w * c.w - y.w * s.w};
    b = f32x4{y.x * c.x + x.x * s.x, y.y * c.y + x.y * s.y, y.z * c.z + x.z * s.z,
              y.w * c.w + x.w * s.w};
  }
}

__device__ __forceinline__ float dot8(f32x4 a, f32x4 b, f32x4 c, f32x4 d) {
  return a.x * c.x + a.y * c.y + a.z * c.z + a.w * c.w + b.x * d.x + b.y * d.y + b.z * d.z +
         b.w * d.w;
}

// Where row `row` of a side lies, and its position (below zero: padding).
struct RowAt {
  uint32_t token, head;
  int pos;
};
__device__ __forceinline__ RowAt row_at(const NormArgs &a, const NormSide &s, uint32_t row) {
  RowAt r;
  r.token = s.by_n.div(row);
  r.head = row - r.token * s.n;
  r.pos = a.positions ? a.positions[r.token]
                      : a.pos0 + (int)(r.token - a.by_S.div(r.token) * a.S);
  return r;
}

constexpr int kThreads = 256;

template <int D>
constexpr int kLanes = D <= 64 ? 8 : 16;  // lanes per row
template <int D>
constexpr int kGroups = kThreads / kLanes<D>;  // rows a workgroup holds at once

// The other element of each pair, for both runs.
template <bool INTER>
__device__ __forceinline__ void partners(f32x4 a, f32x4 b, f32x4 &oa, f32x4 &ob) {
  oa = INTER ? f32x4{a.y, a.x, a.w, a.z} : b;
  ob = INTER ? f32x4{b.y, b.x, b.w, b.z} : a;
}

// Forward.  A group of lanes takes up to kHeads consecutive heads of one token: its
// indices, position and table values are found once for them, and the weights go
// into the rotation's coefficients once,
//   y_a = r (x_a (w_a c) - x_b (w_b s)),  y_b = r (x_b (w_b c) + x_a (w_a s)),
// which leaves about 70 vector instructions a row: with 150 (all of this per row)
// these took most of the time of a large call, 165 us for 128K tokens of 8 + 1
// heads of 128 in bf16.
constexpr int kHeads = 4;

template <typename T, int D, bool INTER, bool NT>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(const NormArgs a, uint32_t q_blocks) {
  constexpr int L = kLanes<D>, R = kGroups<D>;
  const bool is_k = blockIdx.x >= q_blocks;
  const NormSide &s = a.side[is_k];
  const uint32_t blk = blockIdx.x - (is_k ? q_blocks : 0);
  const int m = threadIdx.x % L;
  const LaneCols lc = lane_cols<INTER>(m, a.rot);
  const uint32_t unit = blk * R + threadIdx.x / L;
  const bool on = 8 * m < D && unit < s.units;
  const uint32_t token = s.by_chunks.div(unit), h0 = (unit - token * s.chunks) * kHeads;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f}, one = {1.f, 1.f, 1.f, 1.f};
  int heads = 0, pos = 0;
  f32x4 xa[kHeads], xb[kHeads];  // zero in lanes past a row's end, which its sum includes
#pragma unroll
  for (int h = 0; h < kHeads; ++h) xa[h] = xb[h] = zero;
  if (on) {
    heads = s.n - h0 < kHeads ? s.n - h0 : kHeads;
    const T *x = static_cast<const T *>(s.x) + (long long)token * s.x_row + (size_t)h0 * D;
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < heads) {
        xa[h] = load4<NT>(x + h * D + lc.a);
        xb[h] = load4<NT>(x + h * D + lc.b);
      }
    pos = a.positions ? a.positions[token] : a.pos0 + (int)(token - a.by_S.div(token) * a.S);
  }
  f32x4 ca = one, cb = one, sa = zero, sb = zero;  // y_a = x_a ca + (its partner) sa
  if (s.w && on) ca = load4(s.w + lc.a), cb = load4(s.w + lc.b);
  const bool turned = a.rot > 0;
  if (lc.turns && on) {
    f32x4 c = one * __builtin_nanf(""), sn = c, wa, wb;
    if (pos >= 0 && pos < a.table_rows) {
      const size_t t = (size_t)pos * (a.rot / 2) + lc.pair;
      c = load4(a.cos + t);
      sn = load4(a.sin + t);
    }
    partners<INTER>(ca, cb, wa, wb);
    if (INTER) {
      sa = wa * f32x4{-sn.x, sn.x, -sn.y, sn.y};
      sb = wb * f32x4{-sn.z, sn.z, -sn.w, sn.w};
      ca *= f32x4{c.x, c.x, c.y, c.y};
      cb *= f32x4{c.z, c.z, c.w, c.w};
    } else {
      sa = wa * -sn;
      sb = wb * sn;
      ca *= c;
      cb *= c;
    }
  } else if (turned && pos >= a.table_rows) {
    ca = cb = one * __builtin_nanf("");
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    f32x4 ya = xa[h] * ca, yb = xb[h] * cb;
    if (turned) {
      f32x4 oa, ob;
      partners<INTER>(xa[h], xb[h], oa, ob);
      if (a.rot < D && !lc.turns) oa = ob = zero;
      ya += oa * sa;
      yb += ob * sb;
    }
    if (s.w) {
      const float r =
          rsqrtf(group_sum<L>(dot8(xa[h], xb[h], xa[h], xb[h])) * (1.f / D) + a.eps);
      ya *= r;
      yb *= r;
    }
    if (h < heads) {
      if (pos < 0) ya = yb = zero;
      T *y = static_cast<T *>(s.y) + (long long)token * s.y_row + (size_t)(h0 + h) * D;
      store4(y + lc.a, ya);
      store4(y + lc.b, yb);
    }
  }
}

// Backward.  A lane's columns are the same in every row it holds, so dw's
// partial sums stay in its eight registers over all rows of its workgroup
// (rows blk*R.., a grid stride apart); the workgroup's groups are then added
// in LDS in a fixed order and written as one row of `partials`.
template <typename TX, typename TG, int D, bool INTER, bool NT>
__global__ __launch_bounds__(kThreads) void norm_rope_bwd_kernel(const NormArgs a,
                                                                 float *partials,
                                                                 uint32_t q_blocks) {
  constexpr int L = kLanes<D>, R = kGroups<D>;
  const bool is_k = blockIdx.x >= q_blocks;
  const NormSide &s = a.side[is_k];
  const uint32_t blk = blockIdx.x - (is_k ? q_blocks : 0);
  const uint32_t blocks = is_k ? gridDim.x - q_blocks : q_blocks;
  const int m = threadIdx.x % L;
  const LaneCols lc = lane_cols<INTER>(m, a.rot);
  const bool on = 8 * m < D;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f}, one = {1.f, 1.f, 1.f, 1.f};
  f32x4 wa = one, wb = one;
  if (s.w && on) wa = load4(s.w + lc.a), wb = load4(s.w + lc.b);
  f32x4 dwa = zero, dwb = zero;
  const uint64_t step = (uint64_t)blocks * R;
  for (uint64_t r0 = (uint64_t)blk * R; r0 < s.rows; r0 += step) {  // workgroup-uniform
    const uint64_t row = r0 + threadIdx.x / L;
    f32x4 xa = zero, xb = zero, za = zero, zb = zero;
    RowAt at;
    at.pos = -1;
    if (row < s.rows && on) {
      at = row_at(a, s, (uint32_t)row);
      if (at.pos >= 0) {
        const TG *dy = static_cast<const TG *>(s.dy) + row * D;
        za = load4<NT>(dy + lc.a);
        zb = load4<NT>(dy + lc.b);
        if (s.w) {
          const TX *x = static_cast<const TX *>(s.x) + (long long)at.token * s.x_row +
                        (size_t)at.head * D;
          xa = load4<NT>(x + lc.a);
          xb = load4<NT>(x + lc.b);
        }
        if (lc.turns && at.pos < a.table_rows) {
          const size_t t = (size_t)at.pos * (a.rot / 2) + lc.pair;
          turn<INTER>(za, zb, load4(a.cos + t), -load4(a.sin + t));
        }
        if (a.rot > 0 && at.pos >= a.table_rows) za = zb = one * __builtin_nanf("");
      }
    }
    if (s.w) {
      const f32x4 ga = za * wa, gb = zb * wb;
      const float ss = group_sum<L>(dot8(xa, xb, xa, xb));
      const float gx = group_sum<L>(dot8(ga, gb, xa, xb));
      const float r = rsqrtf(ss * (1.f / D) + a.eps);
      const float k = r * r * (gx * (1.f / D));
      if (at.pos >= 0) {  // a row of padding adds nothing, also where eps = 0
        dwa += za * (xa * r);
        dwb += zb * (xb * r);
        za = r * (ga - xa * k);
        zb = r * (gb - xb * k);
      }
    }
    if (row < s.rows && on) {
      TG *dx = static_cast<TG *>(s.y) + row * D;
      store4(dx + lc.a, za);
      store4(dx + lc.b, zb);
    }
  }
  if (!s.w) return;
  __shared__ float part[R][D];
  if (on) {
    float *p = part[threadIdx.x / L];
    *reinterpret_cast<f32x4 *>(p + lc.a) = dwa;
    *reinterpret_cast<f32x4 *>(p + lc.b) = dwb;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < D; e += kThreads) {
    float t = 0.f;
#pragma unroll
    for (int g = 0; g < R; ++g) t += part[g][e];
    partials[(size_t)blockIdx.x * D + e] = t;
  }
}

// dw of one side: the sum of its workgroups' partial rows, 16 columns per
// workgroup, four a thread, 64 threads each over every 64th row.
template <int D>
__global__ __launch_bounds__(kThreads) void norm_dw_kernel(const NormArgs a, const float *partials,
                                                           uint32_t q_blocks, uint32_t k_blocks) {
  const bool is_k = blockIdx.y;
  const uint32_t first = is_k ? q_blocks : 0, n = is_k ? k_blocks : q_blocks;
  const int col = blockIdx.x * 16 + threadIdx.x % 4 * 4, row = threadIdx.x / 4;
  f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (uint32_t i = row; i < n; i += 64)
    t += *reinterpret_cast<const f32x4 *>(partials + (size_t)(first + i) * D + col);
  __shared__ float part[64][17];
#pragma unroll
  for (int i = 0; i < 4; ++i) part[row][threadIdx.x % 4 * 4 + i] = t[i];
  __syncthreads();
  // 16 threads a column, four rows each, then the 16 by lane exchange
  const int c = threadIdx.x / 16, r = threadIdx.x % 16;
  float x = part[r][c] + part[r + 16][c] + (part[r + 32][c] + part[r + 48][c]);
  x = group_sum<16>(x);
  if (r == 0) a.side[is_k].dw[blockIdx.x * 16 + c] = x;
}

// Whether a call's inputs are read with the non-temporal hint: where what it
// moves (`bytes`) does not stay in the 256 MB of the last-level cache anyway.  128K
// tokens of 8 + 1 heads of 128 in bf16 (604 MB): 130 -> 120 us, their backward 301 ->
// 269; but 4K tokens of 8 + 2 heads (21 MB, the inputs still cached) 6.6 -> 7.1,
// backward 16.2 -> 17.6.  The other types are alike (8 + 2 heads of 128, without -> with):
// fp32 forward 100 MB 19.1 -> 20.6, 400 MB 73.3 -> 71.3, 1 GB 188 -> 174; backward of
// fp32 with fp32 gradients 23.6 -> 25.5, 83.4 -> 79.5, 213 -> 195, of bf16 with bf16
// gradients 24.9 -> 27.1, 86.3 -> 85.1, 218 -> 200.  Results are stored with the hint always (137 -> 130, 4K
// tokens 7.6 -> 6.6).
bool streams(const NormArgs &a, int d, int bytes_per_element) {
  return ((uint64_t)a.side[0].rows + a.side[1].rows) * d * bytes_per_element > 192ull << 20;
}

template <typename T, int D, bool INTER>
hipError_t fwd_typed(const NormArgs &a, bool nt, hipStream_t stream) {
  const uint64_t per = kGroups<D>;
  const uint64_t qb = (a.side[0].units + per - 1) / per, kb = (a.side[1].units + per - 1) / per;
  const dim3 grid((unsigned)(qb + kb));
  if (nt)
    hipLaunchKernelGGL((norm_rope_kernel<T, D, INTER, true>), grid, dim3(kThreads), 0, stream, a,
                       (uint32_t)qb);
  else
    hipLaunchKernelGGL((norm_rope_kernel<T, D, INTER, false>), grid, dim3(kThreads), 0, stream, a,
                       (uint32_t)qb);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t fwd_order(const NormArgs &a, bool interleaved, bool nt, hipStream_t stream) {
  return interleaved ? fwd_typed<T, D, true>(a, nt, stream) : fwd_typed<T, D, false>(a, nt, stream);
}

template <typename T>
hipError_t fwd_dim(const NormArgs &a, int d, bool interleaved, bool nt, hipStream_t stream) {
  switch (d) {
    case 64: return fwd_order<T, 64>(a, interleaved, nt, stream);
    case 80: return fwd_order<T, 80>(a, interleaved, nt, stream);
    case 96: return fwd_order<T, 96>(a, interleaved, nt, stream);
    default: return fwd_order<T, 128>(a, interleaved, nt, stream);
  }
}

template <typename TX, typename TG, int D, bool INTER>
hipError_t bwd_typed(const NormArgs &a, float *partials, bool nt, hipStream_t stream) {
  const uint32_t qb = norm_bwd_blocks(a.side[0].rows, D), kb = norm_bwd_blocks(a.side[1].rows, D);
  if (nt)
    hipLaunchKernelGGL((norm_rope_bwd_kernel<TX, TG, D, INTER, true>), dim3(qb + kb), dim3(kThreads),
                       0, stream, a, partials, qb);
  else
    hipLaunchKernelGGL((norm_rope_bwd_kernel<TX, TG, D, INTER, false>), dim3(qb + kb),
                       dim3(kThreads), 0, stream, a, partials, qb);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.side[0].w) return e;
  hipLaunchKernelGGL((norm_dw_kernel<D>), dim3(D / 16, 2), dim3(kThreads), 0, stream, a, partials,
                     qb, kb);
  return hipGetLastError();
}

template <typename TX, typename TG, int D>
hipError_t bwd_order(const NormArgs &a, float *partials, bool interleaved, bool nt,
                     hipStream_t stream) {
  return interleaved ? bwd_typed<TX, TG, D, true>(a, partials, nt, stream)
                     : bwd_typed<TX, TG, D, false>(a, partials, nt, stream);
}

template <typename TX, typename TG>
hipError_t bwd_dim(const NormArgs &a, float *partials, int d, bool interleaved, bool nt,
                   hipStream_t stream) {
  switch (d) {
    case 64: return bwd_order<TX, TG, 64>(a, partials, interleaved, nt, stream);
    case 80: return bwd_order<TX, TG, 80>(a, partials, interleaved, nt, stream);
    case 96: return bwd_order<TX, TG, 96>(a, partials, interleaved, nt, stream);
    default: return bwd_order<TX, TG, 128>(a, partials, interleaved, nt, stream);
  }
}

}  // namespace

hipError_t launch_norm_rope(NormArgs a, int d, bool interleaved, bool f32, hipStream_t stream) {
  for (NormSide &s : a.side) {
    s.chunks = (s.n + kHeads - 1) / kHeads;
    s.by_chunks = FastDiv::make(s.chunks);
    s.units = s.rows / s.n * s.chunks;
  }
  const bool nt = streams(a, d, f32 ? 8 : 4);
  return f32 ? fwd_dim<float>(a, d, interleaved, nt, stream)
             : fwd_dim<uint16_t>(a, d, interleaved, nt, stream);
}

int norm_bwd_blocks(uint32_t rows, int d) {
  const uint32_t per = kThreads / (d <= 64 ? 8 : 16);
  const uint64_t blocks = ((uint64_t)rows + per - 1) / per;
  return (int)(blocks < 1024 ? blocks : 1024);
}

hipError_t launch_norm_rope_bwd(const NormArgs &a, float *partials, int d, bool interleaved,
                                bool f32, bool grad_f32, hipStream_t stream) {
  const bool nt = streams(a, d, (f32 ? 4 : 2) + (grad_f32 ? 8 : 4));
  if (f32)
    return grad_f32 ? bwd_dim<float, float>(a, partials, d, interleaved, nt, stream)
                    : bwd_dim<float, uint16_t>(a, partials, d, interleaved, nt, stream);
  return grad_f32 ? bwd_dim<uint16_t, float>(a, partials, d, interleaved, nt, stream)
                  : bwd_dim<uint16_t, uint16_t>(a, partials, d, interleaved, nt, stream);
}

}  // namespace basp
