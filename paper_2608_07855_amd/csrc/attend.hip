// Attention of a ragged batch over its resident caches: sliding window with
// first tokens that stay visible, and prefixes that a whole batch shares.
//
// Row r (position p) of sequence s and query head h:
//   x_t = scale q.k_t over the tokens with p_t <= p and (no window, or
//   p - p_t < window, or p_t < n_sink);  lse = log sum e^x;  o = sum e^(x - lse) v.
// Logits are carried in log2 units (scale * log2(e)).
#include "ckv_device.h"
#include "ckv_kernels.h"

#include <algorithm>
#include <climits>

namespace ckv {

namespace {

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

__device__ __forceinline__ int seq_tokens(const SeqCaches& c, int s) { return clampi(c.n_tokens[s], 0, c.max_tokens); }

__device__ __forceinline__ int row_start(const AttendArgs& a, int s) { return clampi(a.cu_rows[s], 0, a.n_rows); }

// the sequence that owns row r, or -1: the last s with cu_rows[s] <= r
__device__ __forceinline__ int row_seq(const AttendArgs& a, int r) {
  int lo = 0, hi = a.own.n_seq;            // cu_rows[lo] <= r < cu_rows[hi], once both are checked
  if (row_start(a, 0) > r || row_start(a, hi) <= r) return -1;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (row_start(a, m) <= r) lo = m;
    else hi = m;
  }
  return lo;
}

__device__ __forceinline__ bool sees(int p, int qp, int window, int n_sink) {
  return p <= qp && (window == 0 || (uint32_t)qp - (uint32_t)p < (uint32_t)window || p < n_sink);
}

template <bool F16>
__device__ __forceinline__ float elem(uint32_t bits) {
  if constexpr (F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
  else return bf16_bits_to_float(bits);
}

// round to nearest even, NaN stays NaN
template <bool F16>
__device__ __forceinline__ uint16_t to_elem(float x) {
  if constexpr (F16) return __builtin_bit_cast(uint16_t, (_Float16)x);
  else return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// One wave per (row, query head): 64 tokens at a time, one per lane; then
// every lane adds their weighted values into its own widths.
template <int D, bool F16>
__global__ __launch_bounds__(256) void attend_rows_kernel(AttendArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int r = (int)(item / a.Hq), h = (int)(item % a.Hq);
  if (r >= a.n_rows) return;
  const int s = row_seq(a, r);
  if (s < 0) return;
  const int g = h / a.group;
  const int n = seq_tokens(a.own, s), base = a.has_pre ? seq_tokens(a.pre, 0) : 0;
  int qp;
  if (a.qpos) {
    qp = a.qpos[r];
  } else {
    const int t = n - (row_start(a, s + 1) - r);
    if (!a.own.pos) qp = base + t;
    else qp = t >= 0 ? a.own.pos[s * a.own.pos_stride + t] : INT_MIN;
  }
  const uint16_t* q = a.q + r * a.q_row_stride + h * a.q_head_stride;
  constexpr int PW = D / 64;
  float m = -INFINITY, l = 0.f, acc[PW] = {};
  for (int part = a.has_pre ? 0 : 1; part < 2; ++part) {
    const SeqCaches& c = part ? a.own : a.pre;
    const int sq = part ? s : 0, nt = part ? n : base, b = part ? base : 0;
    const int64_t head = g * c.head_stride + (c.slot ? 0 : sq * c.seq_stride);
    for (int t0 = 0; t0 < nt; t0 += 64) {
      const int t = t0 + lane;
      bool vis = t < nt;
      int64_t at = 0;
      float x = -INFINITY;
      if (vis) vis = sees(c.pos ? c.pos[sq * c.pos_stride + t] : b + t, qp, a.window, a.n_sink);
      if (vis) {
        const int row = c.slot ? (int)min((uint32_t)c.slot[sq * c.slot_stride + t], (uint32_t)c.pool_last) : t;
        at = head + row * c.tok_stride;
        x = 0.f;
        for (int e = 0; e < D; e += 8) {
          const u32x4 kk = ldg_u4(c.k + at + e), qq = ldg_u4(q + e);
          for (int j = 0; j < 8; ++j) x = fmaf(elem<F16>(chunk_elem(kk, j)), elem<F16>(chunk_elem(qq, j)), x);
        }
        x *= a.sl2;
      }
      unsigned long long todo = __ballot(vis);
      if (!todo) continue;
      float mx = x;
      for (int off = 32; off; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, 64));
      mx = fmaxf(mx, m);
      const float ref = mx == -INFINITY ? 0.f : mx;
      const float al = exp2f(m - ref);
      const float p = vis ? exp2f(x - ref) : 0.f;
      m = mx;
      float sum = p;
      for (int off = 32; off; off >>= 1) sum += __shfl_xor(sum, off, 64);
      l = l * al + sum;
      for (int w = 0; w < PW; ++w) acc[w] *= al;
      while (todo) {
        const int j = __ffsll((long long)todo) - 1;
        todo &= todo - 1;
        const float pj = __shfl(p, j, 64);
        const int64_t aj = __shfl((long long)at, j, 64);
        for (int w = 0; w < PW; ++w) acc[w] = fmaf(pj, elem<F16>(c.v[aj + w * 64 + lane]), acc[w]);
      }
    }
  }
  const int64_t out = (int64_t)r * a.Hq + h;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bool bad = false;
  for (int w = 0; w < PW; ++w) {
    const float y = l == 0.f ? 0.f : acc[w] * inv;
    bad |= !__builtin_isfinite(y);
    a.o[out * D + w * 64 + lane] = to_elem<F16>(y);
  }
  const float lse = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  bad |= l != 0.f && !__builtin_isfinite(lse);
  if (a.lse && lane == 0) a.lse[out] = lse;
  if (bad) latch_nonfinite(a.nonfinite);
}

}  // namespace

hipError_t launch_attend_rows(const AttendArgs& a, hipStream_t s) {
  const int64_t items = (int64_t)a.n_rows * a.Hq;
  const dim3 grid((unsigned)((items + 3) / 4));
  if (a.D == 64) {
    if (a.f16) attend_rows_kernel<64, true><<<grid, 256, 0, s>>>(a);
    else attend_rows_kernel<64, false><<<grid, 256, 0, s>>>(a);
  } else {
    if (a.f16) attend_rows_kernel<128, true><<<grid, 256, 0, s>>>(a);
    else attend_rows_kernel<128, false><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace ckv
