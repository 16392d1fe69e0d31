// basp_span_device.hpp -- device side of the score rule of attention over spans.
#pragma once

#include "basp_device.hpp"
#include "basp_span.hpp"

namespace basp {

// buf_load16_lds_async with the wait states that a resource may need which was read
// back from a vector register's lanes just before (kernels with more scalar values than
// registers keep some there): five between a vector instruction's write of a scalar
// register and a memory instruction's use of it.  The compiler does not see into the
// asm and adds none.
__device__ __forceinline__ void copy16_to_lds(u32x4 rsrc, uint32_t off, uint32_t lds_addr) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :
               : "v"(off), "s"(rsrc), "{m0}"(lds_addr)
               : "memory");
}

// Where the 16 bytes come from that a lane copies into an LdsTile<LW> of D-element rows
// by the i-th of N copies of its wave (dma_src_off of chunk slot (N wave + i) 64 + lane):
// each copy is 64 / (LW / 8) rows further on, where the swizzle flips one bit of the
// chunk's number.  Formed anew for each copy from two registers: offsets kept for
// both tensors take up to 16, and one register too many sends a loop's values to
// scratch memory, whose loads wait for every copy in flight.
template <int LW, int D, int N>
struct CopySource {
  static constexpr int CPR = LW / 8, ROWS = 64 / CPR, FLIP = LW == 128 ? 1 : 2;
  static_assert(N <= (LW == 128 ? 4 : 2), "the flips are those of the swizzle");
  uint32_t row, col;
  __device__ __forceinline__ CopySource(int wave, int lane) {
    const int pos = wave * N * 64 + lane;
    row = pos / CPR;
    col = ((pos % CPR) ^ LdsTile<LW>::swz(pos / CPR)) << 4;
  }
  __device__ __forceinline__ uint32_t off(int i, uint32_t row_bytes) const {
    uint32_t r = row, c = col;
    asm volatile("" : "+v"(r), "+v"(c));  // not kept over the loop
    c ^= (uint32_t)(FLIP * i) << 4;
    const uint32_t x = __umul24(r + ROWS * i, row_bytes) + c;
    return D < LW && c >= D * 2 ? kZeroOffset : x;
  }
};

// lo and hi of a row, inside [0, S]; empty spans as lo = hi = 0.
__device__ __forceinline__ void span_of(const int *spans, size_t beta, int S, int row, int &lo,
                                        int &hi) {
  lo = 0;
  hi = row + 1;
  if (spans) {
    const u32x2 x = *reinterpret_cast<const u32x2 *>(spans + (beta * S + row) * 2);
    lo = max((int)x.x, 0);
    hi = min((int)x.y, S);
    if (hi <= lo) lo = hi = 0;
  }
}

// Which keys some and all rows of a group see: keys outside [any_lo, any_hi)
// no row, keys of [all_lo, all_hi) every row.
struct SpanHull {
  int any_lo, any_hi, all_lo, all_hi;
  __device__ __forceinline__ bool none(int j0, int n) const {
    return j0 >= any_hi || j0 + n <= any_lo;
  }
  __device__ __forceinline__ bool full(int j0, int n) const {
    return j0 >= all_lo && j0 + n <= all_hi;
  }
};

// A row's own hull; rows past S stand back.
__device__ __forceinline__ SpanHull hull_of(int lo, int hi, bool row_exists) {
  if (!row_exists) return SpanHull{0x7fffffff, 0, 0, 0x7fffffff};
  if (hi <= lo) return SpanHull{0x7fffffff, 0, 0x7fffffff, 0};
  return SpanHull{lo, hi, lo, hi};
}
__device__ __forceinline__ SpanHull join(const SpanHull &x, const SpanHull &y) {
  return SpanHull{min(x.any_lo, y.any_lo), max(x.any_hi, y.any_hi), max(x.all_lo, y.all_lo),
                  min(x.all_hi, y.all_hi)};
}
// Over the 32 lanes l % 32, in scalar registers (lanes l and l + 32 hold the
// same row).
__device__ __forceinline__ SpanHull wave_hull(SpanHull h) {
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) {
    const SpanHull y{__shfl_xor(h.any_lo, x), __shfl_xor(h.any_hi, x), __shfl_xor(h.all_lo, x),
                     __shfl_xor(h.all_hi, x)};
    h = join(h, y);
  }
  return SpanHull{__builtin_amdgcn_readfirstlane(h.any_lo),
                  __builtin_amdgcn_readfirstlane(h.any_hi),
                  __builtin_amdgcn_readfirstlane(h.all_lo),
                  __builtin_amdgcn_readfirstlane(h.all_hi)};
}

// Words of two bf16: the bits 15 and 31 are set where a half is infinite or NaN.
__device__ __forceinline__ uint32_t nonfinite_halves(uint32_t w) {
  return ((w & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u;
}

// An operand of eight bf16 whose infinities and NaN must not meet weights of
// 0: they become 0, and where a key (or row) that `seen` marks has one, the element of
// acc becomes NaN.  seen: 1 (0x3F80) in the halves of slots that count.
__device__ __forceinline__ bf16x8 finite_operand(bf16x8 x, u32x4 seen, f32x16 &acc) {
  u32x4 v = __builtin_bit_cast(u32x4, x), bad;
#pragma unroll
  for (int y = 0; y < 4; ++y) bad[y] = nonfinite_halves(v[y]);
  if (__builtin_amdgcn_ballot_w64((bad.x | bad.y | bad.z | bad.w) != 0)) {
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const uint32_t hi = bad[y] & 0x80000000u, lo = bad[y] & 0x8000u;
      if (hi) v[y] &= 0xFFFFu;
      if (lo) v[y] &= 0xFFFF0000u;
      bad[y] = (hi ? 0x3F800000u : 0u) | (lo ? 0x3F80u : 0u);
    }
    const f32x16 count = mfma32x32x16(as_bf16x8(bad), as_bf16x8(seen), f32x16{});
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (count[r] > 0.f) acc[r] = __builtin_nanf("");
  }
  return as_bf16x8(v);
}

}  // namespace basp
