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

// Codes p of both halves of w, shifted into the upper 4 of the 10 bits of an fp16 mantissa.
template <int P>
__device__ __forceinline__ uint32_t two_codes(uint32_t w) {
  constexpr int up = 6 - 4 * P;
  return up > 0 ? w << (up > 0 ? up : 0) : w >> (up < 0 ? -up : 0);
}

// Four such pairs as the values they stand for, in fp16.  Behind the exponent of 16 a
// code n in those bits is the number 16 + n, exactly: one instruction that masks and
// joins, and a fused product and sum make two values.  (With a code at the low end of
// the mantissa, 1024 + n, the base would be 64 times as far from the values, and its
// rounding with it.  In assembly, because the compiler takes two instructions where mask and
// exponents are literals, and keeps them where the many-rows kernel has no registers if they are not; four
// together, because it waits a cycle behind assembly.)
__device__ __forceinline__ u32x4 values_of(uint32_t n0, uint32_t n1, uint32_t n2, uint32_t n3, const Scale& c0, const Scale& c1,
                                           const Scale& c2, const Scale& c3) {
  asm("v_and_or_b32 %0, %0, %4, %5\n\tv_and_or_b32 %1, %1, %4, %5\n\tv_and_or_b32 %2, %2, %4, %5\n\tv_and_or_b32 %3, %3, %4, %5"
      : "+v"(n0), "+v"(n1), "+v"(n2), "+v"(n3)
      : "s"(0x03C003C0u), "v"(0x4C004C00u));
  const auto value = [](uint32_t n, const Scale& c) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(h2, n), c.s, c.b));
  };
  return u32x4{value(n0, c0), value(n1, c1), value(n2, c2), value(n3, c3)};
}
// the eight widths of a word, in their order
__device__ __forceinline__ u32x4 eight_values(uint32_t w, const Scale& c) {
  return values_of(two_codes<0>(w), two_codes<1>(w), two_codes<2>(w), two_codes<3>(w), c, c, c, c);
}

// Widths 8j to 8j+7 of a key (or value) of a row in memory.
template <int D>
__device__ __forceinline__ u32x4 row_values(const char* row, bool value, int j) {
  const uint32_t word = ldg_i32(row + (value ? PackedRow<D>::kValue : 0) + 4 * j);
  return eight_values(word, scale_of(ldg_i32(row + (value ? PackedRow<D>::kValueParams : PackedRow<D>::kParams) + j / 4 * 4)));
}
// the fp16 number in one half of a word
__device__ __forceinline__ float half_of(uint32_t w, int h) { return (float)__builtin_bit_cast(h2, w)[h]; }

// bf16 queries as fp16 times a power of two that brings the largest finite element to [2^14, 2^15).
__device__ __forceinline__ float largest_finite(u32x4 x, float m) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = fabsf(bf16_bits_to_float(chunk_elem(x, e)));
    m = fmaxf(m, y < INFINITY ? y : 0.f);
  }
  return m;
}
struct PowerOfTwo {
  float mul, back;      // the factor and its inverse
};
__device__ __forceinline__ PowerOfTwo factor_of(float largest) {
  const uint32_t ex = max(__float_as_uint(largest) >> 23, 15u);
  return {__uint_as_float((268u - ex) << 23), __uint_as_float((ex - 14u) << 23)};
}
__device__ __forceinline__ u32x4 to_f16(u32x4 x, float mul) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const h2 v = {(_Float16)(bf16_bits_to_float(x[r] & 0xFFFFu) * mul), (_Float16)(__uint_as_float(x[r] & 0xFFFF0000u) * mul)};
    x[r] = __builtin_bit_cast(uint32_t, v);
  }
  return x;
}

}  // namespace

}  // namespace ckv
