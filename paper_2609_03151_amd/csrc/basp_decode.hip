// basp_decode.hip -- attention of one new token per sequence over a paged
// key-value cache:
//   O = sum_{j < len} softmax_j(scale q . k_j) v_j,  LSE = log sum_j exp(scale q . k_j).
//
// A sequence is split over its keys, one workgroup per (split, query head),
// each with a running maximum and sum; a second kernel joins the splits:
//   M = max_i m_i,  O = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i
// (scores in log2 units).
#include <math.h>

#include "basp_device.hpp"
#include "basp_ops.hpp"

namespace basp {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true);
  return x + __builtin_bit_cast(float, y);
}

// Partial results of split i of (sequence, query head) r, n splits a row:
// o [rows][n][d] (not divided by l), then (m, l) [rows][n].
struct Partials {
  float *o;
  f32x2 *ml;
};
__host__ __device__ inline Partials partials_at(void *ws, int rows, int n, int d) {
  Partials p;
  p.o = static_cast<float *>(ws);
  p.ml = reinterpret_cast<f32x2 *>(p.o + (size_t)rows * n * d);
  return p;
}

template <int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void decode_split_kernel(const DecodeArgs a, DecodeSplit sp) {
  const int i = blockIdx.x % sp.splits;
  const int r = blockIdx.x / sp.splits, s = r / a.n_q, h = r % a.n_q;
  const int len = a.lens[s];
  const int lo = i * sp.keys;
  if (len > a.max_len || lo >= len) return;
  const int hi = len < lo + sp.keys ? len : lo + sp.keys;
  const int kvh = h / (a.n_q / a.s.n_k);
  const int lane = threadIdx.x % 16, grp = threadIdx.x / 16;
  const bool on = 8 * lane < D;
  float q[8], o[8], m = -INFINITY, l = 0.f;
  const uint16_t *qp = static_cast<const uint16_t *>(a.q) + (long long)s * a.q_row + h * D;
  for (int e = 0; e < 8; ++e) {
    q[e] = on ? bf16_bits_to_f32(qp[8 * lane + e]) : 0.f;
    o[e] = 0.f;
  }
  for (int t = lo + grp; t < hi; t += 16) {
    const int p = t >> a.s.page_log2;
    const int id = p < a.s.max_pages ? a.table[(size_t)s * a.s.max_pages + p] : -1;
    const bool bad = id < 0 || id >= a.s.n_pages;
    const size_t row = (((size_t)(bad ? 0 : id) * a.s.n_k + kvh) << a.s.page_log2) +
                       (t & ((1 << a.s.page_log2) - 1));
    float k[8], v[8], ks = 1.f, vs = 1.f;
    for (int e = 0; e < 8; ++e) {
      const size_t at = row * D + 8 * lane + e;
      if (!on) {
        k[e] = v[e] = 0.f;
      } else if (E4M3) {
        k[e] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t *>(a.k_pages)[at], 0);
        v[e] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t *>(a.v_pages)[at], 0);
      } else {
        k[e] = bf16_bits_to_f32(static_cast<const uint16_t *>(a.k_pages)[at]);
        v[e] = bf16_bits_to_f32(static_cast<const uint16_t *>(a.v_pages)[at]);
      }
    }
    if (E4M3) {
      ks = __builtin_bit_cast(float, (uint32_t)a.k_scales[row] << 23);
      vs = __builtin_bit_cast(float, (uint32_t)a.v_scales[row] << 23);
    }
    float x = 0.f;
    for (int e = 0; e < 8; ++e) x += q[e] * k[e];
    x = dpp_add<0xB1>(x);
    x = dpp_add<0x4E>(x);
    x = dpp_add<0x141>(x);
    x = dpp_add<0x140>(x);
    x *= ks * (a.scale * kLog2e);
    if (bad) x = __builtin_nanf("");
    const float m1 = fmaxf(m, x), ref = m1 == -INFINITY ? 0.f : m1;
    const float c = exp2f(m - ref), w = exp2f(x - ref);
    m = m1;
    l = l * c + w;
    for (int e = 0; e < 8; ++e) o[e] = o[e] * c + w * vs * v[e];
  }
  // the 16 groups of the workgroup
  __shared__ float so[16][D], sm[16], sl[16];
  for (int e = 0; e < 8; ++e)
    if (on) so[grp][8 * lane + e] = o[e];
  if (lane == 0) sm[grp] = m, sl[grp] = l;
  __syncthreads();
  if (threadIdx.x < D) {
    float M = -INFINITY, L = 0.f, O = 0.f;
    for (int g = 0; g < 16; ++g) M = fmaxf(M, sm[g]);
    const float ref = M == -INFINITY ? 0.f : M;
    for (int g = 0; g < 16; ++g) {
      const float c = exp2f(sm[g] - ref);
      L += c * sl[g];
      O += c * so[g][threadIdx.x];
    }
    const int rows = gridDim.x / sp.splits;
    const Partials p = partials_at(a.workspace, rows, sp.splits, D);
    p.o[((size_t)r * sp.splits + i) * D + threadIdx.x] = O;
    if (threadIdx.x == 0) p.ml[(size_t)r * sp.splits + i] = f32x2{M, L};
  }
}

template <int D>
__global__ __launch_bounds__(D) void decode_join_kernel(const DecodeArgs a, DecodeSplit sp) {
  const int r = blockIdx.x, s = r / a.n_q, e = threadIdx.x;
  const int len = a.lens[s];
  uint16_t *o = static_cast<uint16_t *>(a.o) + (size_t)r * D;
  float M = -INFINITY, L = 0.f, O = 0.f;
  if (len > a.max_len) {
    O = L = __builtin_nanf("");
  } else if (len > 0) {
    const Partials p = partials_at(a.workspace, gridDim.x, sp.splits, D);
    const int n = (len + sp.keys - 1) / sp.keys;
    for (int i = 0; i < n; ++i) M = fmaxf(M, p.ml[(size_t)r * sp.splits + i].x);
    const float ref = M == -INFINITY ? 0.f : M;
    for (int i = 0; i < n; ++i) {
      const f32x2 ml = p.ml[(size_t)r * sp.splits + i];
      const float c = exp2f(ml.x - ref);
      L += c * ml.y;
      O += c * p.o[((size_t)r * sp.splits + i) * D + e];
    }
    O /= L;
  }
  o[e] = (uint16_t)(pack_bf16x2(O, 0.f) & 0xFFFFu);
  if (e == 0 && a.lse) a.lse[r] = len > 0 ? (M + log2f(L)) * kLn2 : -INFINITY;
}

template <int D>
hipError_t decode_dim(const DecodeArgs &a, hipStream_t stream) {
  const DecodeSplit sp = decode_split(a.s.b, a.n_q, a.s.n_k, a.max_len);
  const unsigned rows = (unsigned)a.s.b * a.n_q;
  if (a.s.e4m3)
    hipLaunchKernelGGL((decode_split_kernel<D, true>), dim3(rows * sp.splits), dim3(kThreads), 0,
                       stream, a, sp);
  else
    hipLaunchKernelGGL((decode_split_kernel<D, false>), dim3(rows * sp.splits), dim3(kThreads), 0,
                       stream, a, sp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((decode_join_kernel<D>), dim3(rows), dim3(D), 0, stream, a, sp);
  return hipGetLastError();
}

}  // namespace

DecodeSplit decode_split(int b, int n_q, int n_k, int max_len) {
  DecodeSplit sp;
  sp.keys = 1024;
  const long long most = (1ll << 24) / ((long long)b * n_q);
  while (((long long)max_len + sp.keys - 1) / sp.keys > most - 1 && sp.keys < (1 << 30)) sp.keys *= 2;
  sp.splits = (int)(((long long)max_len + sp.keys - 1) / sp.keys);
  return sp;
}

size_t decode_workspace_bytes(int b, int n_q, int n_k, int d, int max_len) {
  const DecodeSplit sp = decode_split(b, n_q, n_k, max_len);
  return (size_t)b * n_q * sp.splits * (d + 2) * sizeof(float);
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
