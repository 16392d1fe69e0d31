// basp_cache.hip -- the rank's keys and values into the pages of a key-value
// cache, and back.
//
// A row (d elements of one head of one token) is a contiguous run in a page,
// [n_pages, n_k, page, d]: the tokens of one head of a page lie side by side,
// which is what attention reads.  In 8 bits a row is v * 2^e with v in e4m3 and
// one scale byte e + 127: e is the least whole number (-110 or more) with
// max finite |x| <= 448 * 2^e.  A power of two costs nothing in precision (an
// e4m3 value keeps its four significant bits at any scale, so a finer scale would only
// move which values fall below the least normal one, 2^-6 * 2^e: with the maximum in
// (224, 448] * 2^e that is 2^-14.8 to 2^-13.8 of it) and makes every step but the rounding of v exact:
// x * 2^-e, v * 2^e in bf16, and the scores and weights that attention multiplies.
//
// Both kernels are bound by HBM: one group of 16 lanes (8 at d = 64) per token
// and head moves its K and its V row, eight elements a lane (16 bytes of bf16).
// Two such pairs of rows per group are slower (a call of 16K rows: 17.2 us
// against 16.1 for write and read), four more so.  What is read back is stored with
// the non-temporal hint (256K tokens of 2 heads in bf16, both calls: 171 us
// without, 149 with), pages are not (157 with: the 8- and 16-byte stores of a row
// come together in the cache).
#include "basp_device.hpp"
#include "basp_ops.hpp"

namespace basp {

namespace {

constexpr int kThreads = 256;

template <int D>
constexpr int kLanes = D <= 64 ? 8 : 16;

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  const uint32_t y =
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
  return x > y ? x : y;
}
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  x = dpp_max<0xB1>(x);   // one lane away
  x = dpp_max<0x4E>(x);   // two
  x = dpp_max<0x141>(x);  // the mirrored half row: the other four
  if (L == 16) x = dpp_max<0x140>(x);
  return x;
}

// Largest finite magnitude of the two bf16 of a word, as bf16 bits.
__device__ __forceinline__ uint32_t mag2(uint32_t w) {
  const uint32_t lo = w & 0x7FFFu, hi = (w >> 16) & 0x7FFFu;
  const uint32_t a = lo < 0x7F80u ? lo : 0u, b = hi < 0x7F80u ? hi : 0u;
  return a > b ? a : b;
}

// Scale byte of a row whose largest finite magnitude is `mag` (bf16 bits):
// with mag = m * 2^k, 1 <= m < 2, e = k - 8 where m <= 1.75 (448 = 1.75 * 2^8),
// else k - 7; 17 (e = -110) for all smaller rows, subnormals among them.
__device__ __forceinline__ uint32_t scale_byte(uint32_t mag) {
  const int byte = (int)(mag >> 7) - 8 + ((mag & 0x7Fu) > 0x60u ? 1 : 0);
  return byte < 17 ? 17u : (uint32_t)byte;
}

__device__ __forceinline__ float pow2_of_byte(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}

// Two bf16 scaled by `f` to two e4m3, round to nearest even; infinities and NaN
// become NaN.
template <bool HI>
__device__ __forceinline__ int pack_e4m3(uint32_t w, float f, int old) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_bit_cast(float, w << 16) * f,
                                         __builtin_bit_cast(float, w & 0xFFFF0000u) * f, old, HI);
}

// Magnitudes that would round to 2^128, which no bf16 holds, down to the next
// smaller value of such a row, 1.875 * 2^127 (off by less than 2^-4 of it).
__device__ __forceinline__ uint32_t below_top(uint32_t w) {
  const uint32_t lo = w & 0x7FFFu, hi = w & 0x7FFF0000u;
  if (lo > 0x7F70u && lo < 0x7F80u) w = (w & 0xFFFF8000u) | 0x7F70u;
  if (hi > 0x7F700000u && hi < 0x7F800000u) w = (w & 0x8000FFFFu) | 0x7F700000u;
  return w;
}

// Page and row of token t of sequence s: false where it is on no valid page.
__device__ __forceinline__ bool find_row(const CacheArgs &a, uint32_t s, long long pos,
                                         uint32_t h, size_t &row) {
  const long long p = pos >> a.s.page_log2;
  if (p >= a.s.max_pages) return false;
  const int id = a.table[(size_t)s * a.s.max_pages + p];
  if (id < 0 || id >= a.s.n_pages) return false;
  row = (((size_t)id * a.s.n_k + h) << a.s.page_log2) + (pos & ((1 << a.s.page_log2) - 1));
  return true;
}

template <int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(const CacheArgs a) {
  constexpr int L = kLanes<D>;
  const int m = threadIdx.x % L;
  const uint32_t i = blockIdx.x * (kThreads / L) + threadIdx.x / L;  // (token, head)
  u32x4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  size_t row = 0;
  bool live = false;
  if (i < a.rows) {
    const uint32_t token = a.by_n.div(i), h = i - token * a.s.n_k;
    const uint32_t s = a.by_T.div(token), t = token - s * a.T;
    const int start = a.start[s];
    if (start >= 0 && (!a.count || (int)t < a.count[s]))
      live = find_row(a, s, (long long)start + t, h, row);
    live = live && 8 * m < D;
    if (live)
#pragma unroll
      for (int w = 0; w < 2; ++w)
        x[w] = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.x[w]) +
                                                (long long)token * a.x_row[w] + (size_t)h * D +
                                                8 * m);
  }
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    u32x4 v = x[w];
    if constexpr (E4M3) {
      uint32_t mag = mag2(v.x);
      mag = mag2(v.y) > mag ? mag2(v.y) : mag;
      mag = mag2(v.z) > mag ? mag2(v.z) : mag;
      mag = mag2(v.w) > mag ? mag2(v.w) : mag;
      const uint32_t byte = scale_byte(group_max<L>(mag));
      if (byte == 247)  // e = 120, the largest
        v = u32x4{below_top(v.x), below_top(v.y), below_top(v.z), below_top(v.w)};
      const float f = pow2_of_byte(254 - byte);  // 2^-e
      const u32x2 q = {(uint32_t)pack_e4m3<true>(v.y, f, pack_e4m3<false>(v.x, f, 0)),
                       (uint32_t)pack_e4m3<true>(v.w, f, pack_e4m3<false>(v.z, f, 0))};
      if (live) {
        *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(a.pages[w]) + row * D + 8 * m) = q;
        if (m == 0) a.scales[w][row] = (uint8_t)byte;
      }
    } else if (live) {
      *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.pages[w]) + row * D + 8 * m) = v;
    }
  }
}

// Two e4m3 (the low or high half of a word) times `f` as two bf16: exact, the
// scale being 2^-110 or more.
template <bool HI>
__device__ __forceinline__ uint32_t unpack_e4m3(uint32_t w, float f) {
  const f32x2 v = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HI);
  return pack_bf16x2(v.x * f, v.y * f);
}

template <int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(const CacheArgs a) {
  constexpr int L = kLanes<D>;
  const int m = threadIdx.x % L;
  const uint32_t i = blockIdx.x * (kThreads / L) + threadIdx.x / L;  // (token, head)
  if (i >= a.rows || 8 * m >= D) return;
  u32x4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  float f[2] = {1.f, 1.f};
  const uint32_t token = a.by_n.div(i), h = i - token * a.s.n_k;
  const uint32_t s = a.by_T.div(token), t = token - s * a.T;
  const int start = a.start ? a.start[s] : 0;
  if (start >= 0 && (!a.count || (int)t < a.count[s])) {
    size_t row;
    if (find_row(a, s, (long long)start + t, h, row)) {
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if constexpr (E4M3) {
          const u32x2 q = *reinterpret_cast<const u32x2 *>(
              static_cast<const uint8_t *>(a.pages[w]) + row * D + 8 * m);
          x[w].x = q.x, x[w].y = q.y;
          f[w] = pow2_of_byte(a.scales[w][row]);
        } else {
          x[w] = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.pages[w]) +
                                                  row * D + 8 * m);
        }
      }
    } else {  // NaN: bf16 0x7FFF, and as e4m3 bytes
      x[0] = x[1] = u32x4{0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu};
    }
  }
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    u32x4 v = x[w];
    if constexpr (E4M3)
      v = u32x4{unpack_e4m3<false>(v.x, f[w]), unpack_e4m3<true>(v.x, f[w]),
                unpack_e4m3<false>(v.y, f[w]), unpack_e4m3<true>(v.y, f[w])};
    __builtin_nontemporal_store(
        v, reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.x[w]) + (size_t)i * D + 8 * m));
  }
}

template <int D>
hipError_t write_dim(const CacheArgs &a, hipStream_t stream) {
  const uint32_t per = kThreads / kLanes<D>;
  const dim3 grid((unsigned)(((uint64_t)a.rows + per - 1) / per));
  if (a.s.e4m3)
    hipLaunchKernelGGL((kv_write_kernel<D, true>), grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((kv_write_kernel<D, false>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

template <int D>
hipError_t read_dim(const CacheArgs &a, hipStream_t stream) {
  const uint32_t per = kThreads / kLanes<D>;
  const dim3 grid((unsigned)(((uint64_t)a.rows + per - 1) / per));
  if (a.s.e4m3)
    hipLaunchKernelGGL((kv_read_kernel<D, true>), grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((kv_read_kernel<D, false>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const CacheArgs &a, hipStream_t stream) {
  switch (a.s.d) {
    case 64: return write_dim<64>(a, stream);
    case 80: return write_dim<80>(a, stream);
    case 96: return write_dim<96>(a, stream);
    default: return write_dim<128>(a, stream);
  }
}

hipError_t launch_kv_read(const CacheArgs &a, hipStream_t stream) {
  switch (a.s.d) {
    case 64: return read_dim<64>(a, stream);
    case 80: return read_dim<80>(a, stream);
    case 96: return read_dim<96>(a, stream);
    default: return read_dim<128>(a, stream);
  }
}

}  // namespace basp
