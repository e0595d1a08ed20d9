// Caches in 4 bits: tokens quantised as they are written, and read back.
#include "packed_device.h"
#include "ckv_kernels.h"

#include <algorithm>

namespace ckv {

namespace {

constexpr int kNT = 256;
constexpr int kMany = 4;                  // tokens of a thread that reads back, whose loads leave together, where a
constexpr int kFew = 4096;                // launch has more than so many workgroups of one each (16 a compute unit)
// Workgroups of a launch at most, each of which takes every so many items: calls whose
// tables have far more room than tokens launch few that find nothing (4096 cost
// one cache of 131072 tokens 10%).
constexpr int64_t kGroups = 1 << 15;
constexpr float kMostElem = 16384.f;   // b reaches -3.2 times this: inside fp16's range

// of the lane beside it (lanes 2i and 2i + 1)
__device__ __forceinline__ float pair_swap(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xB1, 0xF, 0xF, true));
}

__device__ __forceinline__ float nan_min(float x, float y) { return __builtin_elementwise_minimum(x, y); }
__device__ __forceinline__ float nan_max(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// 16 bytes that are read once
__device__ __forceinline__ u32x4 ldg_once(const void* p) {
  typedef const __attribute__((address_space(1))) u32x4* gptr;
  return __builtin_nontemporal_load((gptr)p);
}

template <bool F16>
__device__ __forceinline__ float as_float(uint32_t bits) {
  if constexpr (F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
  else return bf16_bits_to_float(bits);
}

// ---------------------------------------------------------------------------
// A thread quantises 16 widths of a token's key or value; the two threads of a
// group find its smallest and largest element between them (NaN stays NaN).
//
// The code is the largest n of 1..15 with t >= (n + 15.5) s, or 0.  t - 16 s is exact
// (t lies between 8 s and 32 s wherever it decides).  (t - 16 s) / s is formed with a
// reciprocal, off by less than 2^-18 there, and rounded after 2^-12 is taken from it:
// that is n or n - 1, which stays below 15, and one exact comparison of what is left
// with s / 2 tells which.  So the codes are those of the exact quotient.
// (M - m) / 15 is rounded as a division: a product with the rounded 1/15, corrected
// once by its exact remainder.
//
// Bound: HBM (4 D bytes in and 1.25 D out a token and head), vector issue close
// behind (75% busy: about 13 instructions an element and 40 a thread).  A workgroup takes tokens of
// one head, whose rows often follow one another: 65536 tokens of 8 heads of width
// 128 take 80 us (4.4 TB/s; 8 widths a thread, with 21 instructions an element in all,
// 94 us; two tokens a thread no less).
// ---------------------------------------------------------------------------
template <int D, bool F16>
__global__ __launch_bounds__(kNT) void pack_kernel(PackArgs a) {
  using R = PackedRow<D>;
  constexpr int LPT = D / 8, TPB = kNT / LPT;      // threads of a token, tokens of a workgroup at a time
  const int in = threadIdx.x % LPT, w16 = in % (D / 16);
  const bool value = in >= D / 16;
  const int live = a.n_live ? min(max(*a.n_live, 0), a.n_rows) : a.n_rows;
  const int64_t n_items = (int64_t)((live + TPB - 1) / TPB) * a.Hkv;
  for (int64_t item = blockIdx.x; item < n_items; item += gridDim.x) {
    const int g = (int)(item % a.Hkv), t = (int)(item / a.Hkv) * TPB + threadIdx.x / LPT;
    if (t >= live) continue;
    const int row = a.row[t];
    const uint16_t* from = (value ? a.v : a.k) + t * a.tok_stride + g * a.head_stride + 16 * w16;
    const u32x4 x16[2] = {ldg_once(from), ldg_once(from + 8)};
    if ((uint32_t)row >= (uint32_t)a.pool_rows) continue;
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = as_float<F16>(chunk_elem(x16[e / 8], e % 8));
    float lo = nan_min(x[0], x[1]), hi = nan_max(x[0], x[1]);
#pragma unroll
    for (int e = 2; e < 16; e += 2) {
      lo = nan_min(nan_min(lo, x[e]), x[e + 1]);
      hi = nan_max(nan_max(hi, x[e]), x[e + 1]);
    }
    lo = nan_min(lo, pair_swap(lo));
    hi = nan_max(hi, pair_swap(hi));
    const bool whole = __builtin_isfinite(lo) && __builtin_isfinite(hi);
    lo = fminf(fmaxf(lo, -kMostElem), kMostElem);
    hi = fminf(fmaxf(hi, -kMostElem), kMostElem);
    constexpr float k15 = 1.f / 15.f;
    const float range = hi - lo, q = range * k15;
    // (both are rounded to float32 first, and not by one instruction to fp16)
    float step = __builtin_fmaf(__builtin_fmaf(-15.f, q, range), k15, q);
    asm("" : "+v"(step));
    _Float16 s = (_Float16)step;
    const float sf = (float)s;
    float base = __builtin_fmaf(-16.f, sf, lo);
    asm("" : "+v"(base));
    _Float16 b = (_Float16)base + (_Float16)0.f;       // (a zero is +0, whatever its sign was before or behind the rounding)
    const float bf = (float)b, s16 = 16.f * sf;
    const float inv = sf > 0.f ? __builtin_amdgcn_rcpf(sf) : 0.f, border = sf > 0.f ? 0.5f * sf : INFINITY;
    uint32_t word[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float y = (__builtin_amdgcn_fmed3f(x[e], -kMostElem, kMostElem) - bf) - s16;     // (there b is rounded by up to 8, a narrow group's steps)
      const float m = __builtin_amdgcn_fmed3f(floorf(__builtin_fmaf(y, inv, 0.5f - 0x1p-12f)), 0.f, 14.f);
      const uint32_t n = (uint32_t)m + (__builtin_fmaf(-m, sf, y) >= border ? 1u : 0u);
      word[e / 8] |= n << (4 * (e % 8 / 2) + 16 * (e % 2));
    }
    if (!whole) {
      word[0] = word[1] = 0;
      s = (_Float16)0.f;
      b = (_Float16)__builtin_nanf("");
    }
    char* to = a.pool + g * a.pool_head + row * a.pool_row;
    *reinterpret_cast<uint2*>(to + (value ? R::kValue : 0) + 8 * w16) = make_uint2(word[0], word[1]);
    if (w16 % 2 == 0)
      *reinterpret_cast<uint32_t*>(to + (value ? R::kValueParams : R::kParams) + 2 * w16) = __builtin_bit_cast(uint32_t, h2{s, b});
  }
}

// ---------------------------------------------------------------------------
// A thread reads 8 widths of a token's key or value back.
//
// Bound: HBM (1.25 D bytes in and 4 D out a token and head).  Half of a workgroup takes
// keys, the other values, so that a wave stores 1 KB that lies together; four tokens a
// thread, stores past the caches: one cache of 131072 tokens and 8 heads of width 128 125 us
// (5.6 TB/s; one token a thread, a token's key and value side by side, 216).
// ---------------------------------------------------------------------------
template <int D, bool F16, int U>
__global__ __launch_bounds__(kNT) void unpack_kernel(PackArgs a) {
  using R = PackedRow<D>;
  constexpr int LPT = D / 8, TPB = kNT / 2 / LPT;      // threads of a key or value, tokens of a workgroup at a time
  const bool value = threadIdx.x >= kNT / 2;           // a wave's stores lie together
  const int w8 = threadIdx.x % LPT, tok = threadIdx.x % (kNT / 2) / LPT;
  // workgroup `group` of `groups` of a sequence and head, or of every so many of these
  const int64_t pairs = (int64_t)a.Hkv * a.n_seq;
  const int groups = (int)max((int64_t)gridDim.x / pairs, (int64_t)1), group = (int)(blockIdx.x % groups);
  for (int64_t pair = blockIdx.x / groups; pair < pairs; pair += gridDim.x / groups) {
    const int g = (int)(pair % a.Hkv), s = (int)(pair / a.Hkv);
    const int n = min(max(a.n_tokens[s], 0), a.max_tokens);
    const char* from = a.pool + (a.slot ? 0 : s * a.pool_seq) + g * a.pool_head;
    for (int64_t first = (int64_t)group * (TPB * U); first < n; first += (int64_t)groups * (TPB * U)) {
      const int t0 = (int)first + tok;
      int row[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = min(t0 + u * TPB, n - 1);
        row[u] = a.slot ? (int)min((uint32_t)a.slot[s * a.slot_stride + t], (uint32_t)a.pool_last) : t;
      }
      uint32_t word[U], par[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        word[u] = ldg_i32(from + row[u] * a.pool_row + (value ? R::kValue : 0) + 4 * w8);
        par[u] = ldg_i32(from + row[u] * a.pool_row + (value ? R::kValueParams : R::kParams) + w8 / 4 * 4);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = t0 + u * TPB;
        if (t >= n) break;
        u32x4 y = eight_values(word[u], scale_of(par[u]));
        if constexpr (!F16) {
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            typedef __bf16 b2 __attribute__((ext_vector_type(2)));
            y[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector(__builtin_convertvector(__builtin_bit_cast(h2, (uint32_t)y[p]), f32x2), b2));
          }
        }
        __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>((value ? a.v : a.k) + s * a.seq_stride + g * a.head_stride + t * a.tok_stride + 8 * w8));
      }
    }
  }
}

}  // namespace

#define CKV_PACKED(KERNEL, ...) \
  if (a.D == 64) { \
    if (a.f16) KERNEL<64, true __VA_ARGS__><<<grid, kNT, 0, s>>>(a); \
    else KERNEL<64, false __VA_ARGS__><<<grid, kNT, 0, s>>>(a); \
  } else { \
    if (a.f16) KERNEL<128, true __VA_ARGS__><<<grid, kNT, 0, s>>>(a); \
    else KERNEL<128, false __VA_ARGS__><<<grid, kNT, 0, s>>>(a); \
  }
#define CKV_AND ,

hipError_t launch_pack(const PackArgs& a, hipStream_t s) {
  const int tpb = kNT / (a.D / 8);
  const dim3 grid((unsigned)std::min<int64_t>(kGroups, ((int64_t)a.n_rows + tpb - 1) / tpb * a.Hkv));
  CKV_PACKED(pack_kernel)
  return hipGetLastError();
}

hipError_t launch_unpack(const PackArgs& a, hipStream_t s) {
  const int tpb = kNT / (a.D / 4);
  const int64_t pairs = (int64_t)a.Hkv * a.n_seq;
  auto tiles = [&](int step) { return ((int64_t)a.max_tokens + step - 1) / step; };
  const bool many = tiles(tpb) * pairs > kFew;
  // whole groups of workgroups for each sequence and head, or one for several of them
  const dim3 grid((unsigned)std::min(kGroups, pairs * std::min(tiles(many ? kMany * tpb : tpb), std::max<int64_t>(kGroups / pairs, 1))));
  if (many) {
    CKV_PACKED(unpack_kernel, CKV_AND kMany)
  } else {
    CKV_PACKED(unpack_kernel, CKV_AND 1)
  }
  return hipGetLastError();
}

#undef CKV_AND
#undef CKV_PACKED

}  // namespace ckv
