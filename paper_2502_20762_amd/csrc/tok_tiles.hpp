// Tiles of 16-bit rows in LDS as MFMA operands, and fp32 values as sums of 16-bit
// operands: shared by the attentions.
#pragma once
#include "tokens.hpp"

namespace nc {

// Slot of 16-byte unit u of a row of W elements: 16 consecutive rows of one
// unit, and four consecutive rows of four units (a transposed read), each
// touch every LDS bank once.
template <int W>
__device__ __forceinline__ int unit_slot(int row, int u) {
  if (W == 128) return u ^ (((row & 3) << 2) | ((row >> 2) & 3));
  if (W == 64) return u ^ ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
  return u ^ ((row >> 2) & 3);
}

// Byte offset, in an LDS tile of W wide rows, of unit h of row l32; unit
// 2 x + h of row l32 + 32 t lies at (this ^ 32 x) + 64 W t.
template <int W>
__device__ __forceinline__ int row_offset(int lane) {
  return (lane & 31) * (2 * W) + 16 * unit_slot<W>(lane & 31, lane >> 5);
}

// Transposed read of four rows x 16 columns per 16 lanes: lane i of the 16
// passes the address of element (i / 4, 4 (i % 4)) and receives column i of the
// four rows.
__device__ __forceinline__ half4 read_tr(const char* p, F16) {
  typedef __fp16 H4 __attribute__((vector_size(8)));
  typedef H4 __attribute__((address_space(3))) L;
  return __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((L*)p));
}
__device__ __forceinline__ bhalf4 read_tr(const char* p, BF16) {
  typedef bhalf4 __attribute__((address_space(3))) L;
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((L*)p);
}
// MFMA fragment of 32 columns of an LDS tile as rows, contraction over the
// tile's rows ("tokens") in the order of an accumulator: lane half h, element e
// holds token 16 s + 8 (e / 4) + 4 h + e % 4.  Two transposed reads, p = 0 and 1,
// at col_offset(p); columns 32 d.. lie at (that ^ 64 d), tokens 16 s.. at that +
// 32 W s.  With PI the columns of each 16 are taken as 0-3, 8-11, 4-7, 12-15, so
// that a lane of the resulting accumulator holds eight consecutive columns in
// eight registers.
template <int W, bool PI>
__device__ __forceinline__ int col_offset(int lane, int p) {
  const int h = lane >> 5, c = (lane >> 4) & 1, i = lane & 15, k = i & 3;
  const int col = 16 * c + 4 * (PI ? ((k & 1) << 1 | k >> 1) : k), row = 8 * p + 4 * h + (i >> 2);
  return row * (2 * W) + 16 * unit_slot<W>(row, col >> 3) + 2 * (col & 7);
}
template <class E>
__device__ __forceinline__ typename E::V8 read_cols(const char* p0, const char* p1) {
  const auto x = read_tr(p0, E{}), y = read_tr(p1, E{});
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

// fp32 values in the unit u, a power of two, as two 16-bit terms, the second the rest of
// the first: 22 bits in fp16; in bf16 16, or 17 where the first may be rounded to the nearest (NEAR).
template <class E, bool NEAR = false>
__device__ __forceinline__ void two_terms(const float (&x)[8], float u, typename E::V8& hi, typename E::V8& lo) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float a = x[i] * u, b = x[i + 1] * u;  // u a power of two: exact, however often it is formed
    typename E::V2 h;
    if (NEAR || __is_same(E, F16))
      h = {(typename E::T)a, (typename E::T)b};
    else  // bf16 has no unit: the upper halves, which no value close to the end of fp32 rounds up to infinity
      h = __builtin_bit_cast(typename E::V2, __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u));
    asm("" : "+v"(h));  // or each half would be formed anew for its rest
    const typename E::V2 l = {(typename E::T)(a - (float)h.x), (typename E::T)(b - (float)h.y)};
    hi[i] = h.x;
    hi[i + 1] = h.y;
    lo[i] = l.x;
    lo[i + 1] = l.y;
  }
}

}  // namespace nc
