// Caches in 4 bits: tokens quantised as they are written, and read back.
#include "packed_device.h"
#include "ckv_kernels.h"

#include <algorithm>

namespace ckv {

namespace {

constexpr int kNT = 256;
constexpr float kMostElem = 16384.f;   // b reaches -3.2 times this: inside fp16's range

// within each four lanes
__device__ __forceinline__ float quad_swap1(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xB1, 0xF, 0xF, true));   // 1, 0, 3, 2
}
__device__ __forceinline__ float quad_swap2(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x4E, 0xF, 0xF, true));   // 2, 3, 0, 1
}

__device__ __forceinline__ float nan_min(float x, float y) { return __builtin_elementwise_minimum(x, y); }
__device__ __forceinline__ float nan_max(float x, float y) { return __builtin_elementwise_maximum(x, y); }

template <bool F16>
__device__ __forceinline__ float as_float(uint32_t bits) {
  if constexpr (F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
  else return bf16_bits_to_float(bits);
}

// ---------------------------------------------------------------------------
// A thread quantises 8 widths of a token's key or value; the four threads of a
// group find its smallest and largest element between them (NaN stays NaN).
//
// The code is the largest n with t >= (n + 15.5) s.  t / s is formed with a
// reciprocal, off by less than 2^-17 below 32, and rounded after 2^-12 is taken
// from it: that is n or n - 1, and one exact comparison (n + 15.5 has 6 bits, s has
// 11) tells which, so the codes are those of the exact quotient.
//
// Bound: HBM (4 D bytes in and 1.25 D out a token and head).
// ---------------------------------------------------------------------------
template <int D, bool F16>
__global__ __launch_bounds__(kNT) void pack_kernel(PackArgs a) {
  using R = PackedRow<D>;
  constexpr int LPT = D / 4, TPB = kNT / LPT;      // threads of a token, tokens of a workgroup
  const int in = threadIdx.x % LPT, w8 = in % (D / 8);
  const bool value = in >= D / 8;
  const int live = a.n_live ? min(max(*a.n_live, 0), a.n_rows) : a.n_rows;
  const int64_t n_items = (int64_t)((live + TPB - 1) / TPB) * a.Hkv;
  for (int64_t item = blockIdx.x; item < n_items; item += gridDim.x) {
    const int g = (int)(item % a.Hkv), t = (int)(item / a.Hkv) * TPB + threadIdx.x / LPT;
    if (t >= live) continue;
    const int row = a.row[t];
    if ((uint32_t)row >= (uint32_t)a.pool_rows) continue;
    const u32x4 x16 = ldg_u4((value ? a.v : a.k) + t * a.tok_stride + g * a.head_stride + 8 * w8);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = as_float<F16>(chunk_elem(x16, e));
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      lo = nan_min(lo, x[e]);
      hi = nan_max(hi, x[e]);
    }
    lo = nan_min(lo, quad_swap1(lo));
    hi = nan_max(hi, quad_swap1(hi));
    lo = nan_min(lo, quad_swap2(lo));
    hi = nan_max(hi, quad_swap2(hi));
    const bool whole = __builtin_isfinite(lo) && __builtin_isfinite(hi);
    lo = fminf(fmaxf(lo, -kMostElem), kMostElem);
    hi = fminf(fmaxf(hi, -kMostElem), kMostElem);
    _Float16 s = (_Float16)((hi - lo) / 15.f);
    const float sf = (float)s;
    _Float16 b = (_Float16)(lo - 16.f * sf + 0.f);           // (a zero is +0, whatever signs the group's have)
    const float bf = (float)b, inv = sf > 0.f ? __builtin_amdgcn_rcpf(sf) : 0.f;
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t0 = x[e] - bf;
      const float m = floorf(__builtin_fmaf(t0, inv, 0.5f - 0x1p-12f));
      const float n = m + (t0 >= (m + 0.5f) * sf ? -15.f : -16.f);
      word |= (uint32_t)fminf(fmaxf(n, 0.f), 15.f) << (4 * (e / 2) + 16 * (e % 2));
    }
    if (!whole) {
      word = 0;
      s = (_Float16)0.f;
      b = (_Float16)__builtin_nanf("");
    }
    char* to = a.pool + g * a.pool_head + row * a.pool_row;
    *reinterpret_cast<uint32_t*>(to + (value ? R::kValue : 0) + 4 * w8) = word;
    if (w8 % 4 == 0)
      *reinterpret_cast<uint32_t*>(to + (value ? R::kValueParams : R::kParams) + w8) = __builtin_bit_cast(uint32_t, h2{s, b});
  }
}

// ---------------------------------------------------------------------------
// A thread reads 8 widths of a token's key or value back.
//
// Bound: HBM (1.25 D bytes in and 4 D out a token and head).
// ---------------------------------------------------------------------------
template <int D, bool F16>
__global__ __launch_bounds__(kNT) void unpack_kernel(PackArgs a) {
  using R = PackedRow<D>;
  constexpr int LPT = D / 4, TPB = kNT / LPT;
  const int in = threadIdx.x % LPT, w8 = in % (D / 8);
  const bool value = in >= D / 8;
  const int64_t tiles = (a.max_tokens + TPB - 1) / TPB, n_items = tiles * a.Hkv * a.n_seq;
  for (int64_t item = blockIdx.x; item < n_items; item += gridDim.x) {
    const int g = (int)(item / tiles % a.Hkv), s = (int)(item / tiles / a.Hkv);
    const int t = (int)(item % tiles) * TPB + threadIdx.x / LPT;
    if (t >= min(max(a.n_tokens[s], 0), a.max_tokens)) continue;
    const int row = a.slot ? (int)min((uint32_t)a.slot[s * a.slot_stride + t], (uint32_t)a.pool_last) : t;
    const char* from = a.pool + (a.slot ? 0 : s * a.pool_seq) + g * a.pool_head + row * a.pool_row;
    const uint32_t word = ldg_i32(from + (value ? R::kValue : 0) + 4 * w8);
    u32x4 y = eight_values(word, scale_of(ldg_i32(from + (value ? R::kValueParams : R::kParams) + w8 / 4 * 4)));
    if constexpr (!F16) {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        y[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector(__builtin_convertvector(__builtin_bit_cast(h2, (uint32_t)y[p]), f32x2), b2));
      }
    }
    *reinterpret_cast<u32x4*>((value ? a.v : a.k) + s * a.seq_stride + g * a.head_stride + t * a.tok_stride + 8 * w8) = y;
  }
}

constexpr int64_t kGroups = 256 * 16;     // workgroups of a launch at most; each takes every so many items

}  // namespace

#define CKV_PACKED(KERNEL, GRID) \
  if (a.D == 64) { \
    if (a.f16) KERNEL<64, true><<<GRID, kNT, 0, s>>>(a); \
    else KERNEL<64, false><<<GRID, kNT, 0, s>>>(a); \
  } else { \
    if (a.f16) KERNEL<128, true><<<GRID, kNT, 0, s>>>(a); \
    else KERNEL<128, false><<<GRID, kNT, 0, s>>>(a); \
  }

hipError_t launch_pack(const PackArgs& a, hipStream_t s) {
  const int tpb = kNT / (a.D / 4);
  const dim3 grid((unsigned)std::min<int64_t>(kGroups, ((int64_t)a.n_rows + tpb - 1) / tpb * a.Hkv));
  CKV_PACKED(pack_kernel, grid)
  return hipGetLastError();
}

hipError_t launch_unpack(const PackArgs& a, hipStream_t s) {
  const int tpb = kNT / (a.D / 4);
  const int64_t tiles = ((int64_t)a.max_tokens + tpb - 1) / tpb;
  const dim3 grid((unsigned)std::min<int64_t>(kGroups, tiles * a.Hkv * a.n_seq));
  CKV_PACKED(unpack_kernel, grid)
  return hipGetLastError();
}

#undef CKV_PACKED

}  // namespace ckv
