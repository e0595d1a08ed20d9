// Device code of caches in 4 bits (the row of include/commitkv.h): where a row's
// parts lie and how codes become values.
#pragma once

#include "ckv_device.h"

namespace ckv {

namespace {

template <int D>
struct PackedRow {
  static constexpr int kBytes = 5 * D / 4;
  static constexpr int kValue = D / 2;               // codes of the value
  static constexpr int kParams = D;                  // scales and bases of the key
  static constexpr int kValueParams = D + D / 8;     // and of the value
  static constexpr int CH = kBytes / 16;             // 16-byte chunks
};

typedef _Float16 h2 __attribute__((ext_vector_type(2)));

template <int N>
struct Int {
  static constexpr int value = N;
};

// scale and base of a group, in both halves of a word each
struct Scale {
  h2 s, b;
};
__device__ __forceinline__ Scale scale_of(uint32_t params) {
  const h2 p = __builtin_bit_cast(h2, params);
  return {h2{p[0], p[0]}, h2{p[1], p[1]}};
}
// the same of two tokens, one in each half
__device__ __forceinline__ Scale scale_of(uint32_t p0, uint32_t p1) {
  return {__builtin_bit_cast(h2, __builtin_amdgcn_perm(p1, p0, 0x05040100u)),
          __builtin_bit_cast(h2, __builtin_amdgcn_perm(p1, p0, 0x07060302u))};
}

// Codes p of both halves of w as values, in fp16.  In the upper 4 of its 10
// bits, behind the exponent of 16, a code n is the number 16 + n, exactly: a shift,
// one instruction that masks and joins, and a fused product and sum make two
// values.  (With a code at the low end of the mantissa, 1024 + n, the base would
// be 64 times as far from the values, and its rounding with it.)
template <int P>
__device__ __forceinline__ uint32_t two_values(uint32_t w, const Scale& c) {
  constexpr int up = 6 - 4 * P;
  const uint32_t at = up > 0 ? w << (up > 0 ? up : 0) : w >> (up < 0 ? -up : 0);
  uint32_t n;      // (at & mask) | exponents: with both as literals the compiler takes two instructions
  asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(n) : "v"(at), "s"(0x03C003C0u), "v"(0x4C004C00u));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(h2, n), c.s, c.b));
}
// the eight widths of a word, in their order
__device__ __forceinline__ u32x4 eight_values(uint32_t w, const Scale& c) {
  return u32x4{two_values<0>(w, c), two_values<1>(w, c), two_values<2>(w, c), two_values<3>(w, c)};
}

// Widths 8j to 8j+7 of a key (or value) of a row in memory.
template <int D>
__device__ __forceinline__ u32x4 row_values(const char* row, bool value, int j) {
  const uint32_t word = ldg_i32(row + (value ? PackedRow<D>::kValue : 0) + 4 * j);
  return eight_values(word, scale_of(ldg_i32(row + (value ? PackedRow<D>::kValueParams : PackedRow<D>::kParams) + j / 4 * 4)));
}
// the fp16 number in one half of a word
__device__ __forceinline__ float half_of(uint32_t w, int h) { return (float)__builtin_bit_cast(h2, w)[h]; }

// A row's 8 KS elements of the lane as fp16 times a power of two that brings the
// row's largest to [2^14, 2^15); returns the inverse.  max_row: over the lanes of a row.
template <int KS, class Max>
__device__ __forceinline__ float queries_to_f16(u32x4 (&qf)[KS], Max max_row) {
  float m = 0.f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(bf16_bits_to_float(chunk_elem(qf[ks], e))));
  const uint32_t ex = max(__float_as_uint(max_row(m)) >> 23, 15u);
  const float mul = __uint_as_float((268u - ex) << 23);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const h2 v = {(_Float16)(bf16_bits_to_float(qf[ks][r] & 0xFFFFu) * mul), (_Float16)(__uint_as_float(qf[ks][r] & 0xFFFF0000u) * mul)};
      qf[ks][r] = __builtin_bit_cast(uint32_t, v);
    }
  return __uint_as_float((ex - 14u) << 23);
}

}  // namespace

}  // namespace ckv
