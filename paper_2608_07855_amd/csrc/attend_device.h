// Device code shared by the attention kernels of ragged batches: work items,
// the tokens that rows see, direct loads into LDS, and how splits are joined.
#pragma once

#include "ckv_device.h"
#include "ckv_kernels.h"

#include <climits>

namespace ckv {

namespace {

// the same in every lane
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x) {
  return (long long)((unsigned long long)(unsigned)uniform((int)x) | (unsigned long long)(unsigned)uniform((int)(x >> 32)) << 32);
}

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

__device__ __forceinline__ int seq_tokens(const SeqCaches& c, int s) { return clampi(c.n_tokens[s], 0, c.max_tokens); }

__device__ __forceinline__ int row_start(const AttendArgs& a, int s) { return clampi(a.cu_rows[s], 0, a.n_rows); }

// the sequence that owns row r, or -1: the last s with cu_rows[s] <= r
__device__ __forceinline__ int row_seq(const AttendArgs& a, int r) {
  if (a.n_rows == a.own.n_seq && row_start(a, r) == r && row_start(a, r + 1) == r + 1) return r;   // one row each
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

// A product that is rounded before anything is taken from it.
__device__ __forceinline__ float product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}

// Weights are exp2(fma(x, sl2, -ref)), with ref the rounded product of the row's
// largest x: the fused difference keeps what ref was rounded by, which for a ref of
// 2^30 is up to 2^6 (weights of 2^64, or a sum of 0).  From this size on (a quarter
// of a log2 unit) the products are rounded first, so that the largest is ref itself.
constexpr float kLargeRef = 1 << 22;
__device__ __forceinline__ bool any_large(float ref) {
  return __ballot(ref != -INFINITY && fabsf(ref) >= kLargeRef) != 0ull;
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

// ---------------------------------------------------------------------------
// Work items.  A sequence's query rows of one KV head (position by position,
// the head's group of query heads innermost) are cut into blocks, and the
// tokens that a block sees into splits of about `chunk` tokens, so that few
// rows behind a long cache still fill the device.  Lengths are known on the
// device only: every workgroup forms the batch's sums itself (two loads and a
// reduction for up to a workgroup's threads of sequences) instead of waiting
// for a planning launch, and the grid is the host's bound of their number.
// ---------------------------------------------------------------------------
struct Item {
  int s;            // sequence, -1: no such item
  int rb;           // row block
  int split, n_split;
  int64_t e;        // number of the item among those of its KV head
};

// tokens that a block of rows of sequence s sees, as far as the lengths tell:
// decides how many splits it gets, not what they hold
__device__ __forceinline__ int seen_estimate(const AttendArgs& a, int n, int block_rows) {
  if (a.window == 0) return n;
  const long long w = (long long)a.window + a.n_sink + block_rows / a.group + 1;
  return (int)min((long long)n, w);
}

template <int NT>
__device__ __forceinline__ long long block_sum(long long v, long long* sh) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off, 64);
  __syncthreads();
  if ((tid & 63) == 0) sh[tid >> 6] = v;
  __syncthreads();
  long long t = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) t += sh[w];
  return t;
}

struct ItemShared {
  long long wave[16];
  int found[4];
};

__device__ __forceinline__ long long wave_scan(long long v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long long u = __shfl_up(v, off, 64);
    if (lane >= off) v += u;
  }
  return v;
}

// Item e of a KV head: blocks of RB rows, about `target` items over all heads,
// at least min_chunk tokens each.  one_round: `target` at most (up to 64
// sequences), as many as run at the same time.
template <int NT, int RB>
__device__ __forceinline__ Item find_item(const AttendArgs& a, int64_t e, int target, int min_chunk, bool one_round, ItemShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_seq = a.own.n_seq;
  auto load = [&](int s, int& nrb, int& est) {
    nrb = est = 0;
    if (s < n_seq) {
      const int r0 = row_start(a, s), R = max(row_start(a, s + 1) - r0, 0);
      nrb = (int)(((int64_t)R * a.group + RB - 1) / RB);
      est = seen_estimate(a, seq_tokens(a.own, s), min(RB, R * a.group));
    }
  };
  auto splits = [&](int est, int64_t chunk) { return est > 0 ? (int)((est + chunk - 1) / chunk) : 1; };
  auto chunk_of = [&](long long work) {
    return min_chunk == INT_MAX ? (int64_t)INT_MAX : max((int64_t)min_chunk, (work * a.Hkv + target - 1) / target);
  };
  Item it;
  it.e = e;
  if (n_seq <= 64) {
    // every wave for itself, a sequence per lane
    int nrb, est;
    load(lane, nrb, est);
    long long work = (long long)nrb * est;
    if (min_chunk != INT_MAX)
#pragma unroll
      for (int off = 32; off; off >>= 1) work += __shfl_xor(work, off, 64);
    int n_split = splits(est, chunk_of(work));
    long long mine = (long long)nrb * n_split, upto = wave_scan(mine);
    if (one_round && min_chunk != INT_MAX && __shfl(upto, 63, 64) * a.Hkv > target) {
      // rounded up, the splits are too many: at most one a block more than this chunk gives
      int blocks = nrb;
#pragma unroll
      for (int off = 32; off; off >>= 1) blocks += __shfl_xor(blocks, off, 64);
      const int left = max(target / a.Hkv - blocks, 1);
      n_split = splits(est, max((int64_t)min_chunk, (int64_t)((work + left - 1) / left)));
      mine = (long long)nrb * n_split;
      upto = wave_scan(mine);
    }
    const long long at = e - (upto - mine);
    const unsigned long long who = __ballot(at >= 0 && at < mine);
    const int s = who ? __ffsll(who) - 1 : 0;
    it.s = who ? s : -1;
    it.n_split = __builtin_amdgcn_readlane(n_split, s);
    const int place = __builtin_amdgcn_readlane((int)at, s);
    it.rb = place / it.n_split;
    it.split = place % it.n_split;
    return it;
  }
  int nrb, est;
  load(tid, nrb, est);
  long long work = (long long)nrb * est;
  for (int s = tid + NT; s < n_seq; s += NT) {
    int b, t;
    load(s, b, t);
    work += (long long)b * t;
  }
  const int64_t chunk = chunk_of(block_sum<NT>(work, sh.wave));
  if (tid == 0) sh.found[0] = -1;
  int64_t before = 0;
  for (int s0 = 0; s0 < n_seq; s0 += NT) {
    if (s0) load(s0 + tid, nrb, est);
    const int n_split = splits(est, chunk);
    const long long mine = (long long)nrb * n_split;
    long long v = wave_scan(mine);
    __syncthreads();
    if (lane == 63) sh.wave[wave] = v;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) v += sh.wave[w];
      total += sh.wave[w];
    }
    const int64_t at = e - before - (v - mine);
    if (at >= 0 && at < mine) {
      sh.found[0] = s0 + tid;
      sh.found[1] = (int)(at / n_split);
      sh.found[2] = (int)(at % n_split);
      sh.found[3] = n_split;
    }
    before += total;
    if (before > e) break;
  }
  __syncthreads();
  it.s = __builtin_amdgcn_readfirstlane(sh.found[0]);
  it.rb = __builtin_amdgcn_readfirstlane(sh.found[1]);
  it.split = __builtin_amdgcn_readfirstlane(sh.found[2]);
  it.n_split = __builtin_amdgcn_readfirstlane(sh.found[3]);
  return it;
}

// First t of [lo, lo + len) with pos[t] > key (its end if none), pos ascending:
// a wave tries 64 places at once, so 4096 places take two dependent loads.
struct Search {
  const int32_t* pos;
  int lo, len;
  long long key;
  int step, t;
  __device__ __forceinline__ int probe() {      // the position to load
    step = (len + 63) / 64;
    t = lo + min((int)(threadIdx.x & 63) * step + step - 1, len - 1);   // last place of the lane's part
    return len > 0 ? pos[t] : 0;
  }
  __device__ __forceinline__ void take(int value) {
    if (len <= 0) return;
    const bool le = value <= key && (int)(threadIdx.x & 63) * step < len;
    const int skip = min(__popcll(__ballot(le)) * step, len);   // parts that lie at or below the key
    lo += skip;
    len = min(step - 1, len - skip);
  }
};

// The tokens that rows at positions qmin..qmax see between them (tail_rows: of
// these rows, one position is that of the sequence's last token), as one range
// of indexes u < cnt: first tokens t = u < ns, then t = u + shift.
struct Range {
  int ns, shift, cnt;
  int lo, hi, n_first;   // by token: from which on, and up to which, they may be seen; first tokens (before n_sink)
  __device__ __forceinline__ int token(int u) const { return u < ns ? u : u + shift; }
};

__device__ __forceinline__ Range seen_range(const SeqCaches& c, int sq, int n, int base, int qmin, int qmax, int window,
                                            int n_sink, bool tail_rows = false) {
  int hi, lo = 0, ns = 0;
  if (c.pos) {
    // Positions are distinct, so at most `window` tokens before the last seen
    // one lie inside a window, and at most n_sink are first ones.  The three
    // searches load together.
    const int32_t* p = c.pos + sq * c.pos_stride;
    const bool last = tail_rows && qmax == qmin;        // the row of the last token sees all of them
    Search h = {p, 0, last ? 0 : n, (long long)qmax, 0, 0};
    const int most = (int)min((long long)n, (long long)window + max((long long)qmax - qmin, 0ll));
    Search w = {p, last ? n - most : 0, window ? (last ? most : n) : 0, (long long)qmin - window, 0, 0};
    Search k = {p, 0, window ? min(n, n_sink) : 0, (long long)n_sink - 1, 0, 0};
    while (max(max(h.len, w.len), k.len) > 0) {
      const int a = h.probe(), b = w.probe(), d = k.probe();
      h.take(a);
      w.take(b);
      k.take(d);
    }
    hi = last ? n : h.lo;
    lo = window ? w.lo : 0;
    ns = window ? k.lo : 0;
  } else {
    auto in = [&](long long t) { return (int)min(max(t, 0ll), (long long)n); };
    hi = in((long long)qmax + 1 - base);
    if (window) {
      lo = in((long long)qmin - window + 1 - base);
      ns = in((long long)n_sink - base);
    }
  }
  lo = min(lo, hi);
  ns = min(ns, hi);
  Range r;
  r.lo = lo;
  r.hi = hi;
  r.n_first = ns;
  if (lo <= ns) {
    r.ns = 0;
    r.shift = 0;
    r.cnt = hi;
  } else {
    r.ns = ns;
    r.shift = lo - ns;
    r.cnt = ns + hi - lo;
  }
  return r;
}

// Position of row p of the R rows of sequence s, whose first row is r0.
__device__ __forceinline__ int row_position(const AttendArgs& a, int s, int r0, int R, int p, int n, int base) {
  if (a.qpos) return a.qpos[r0 + p];
  const int t = n - R + p;
  if (!a.own.pos) return base + t;
  return t >= 0 && t < n ? a.own.pos[s * a.own.pos_stride + t] : INT_MIN;
}

// ---------------------------------------------------------------------------
// Loads from global memory straight into LDS: lane l's 16 (or 4) bytes land at
// base + 16 l (4 l), with the base the same for the whole wave.  No register
// waits for them; the wave counts them itself (vmcnt, in order).
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
__device__ __forceinline__ void load_lds16(const void* g, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(g) : "m0", "memory");
}
// the same at a 32-bit offset from an address that the wave shares
__device__ __forceinline__ void load_lds16_near(const void* g, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)),
               "v"(offset), "s"(uniform((long long)(uintptr_t)g)) : "m0", "memory");
}
__device__ __forceinline__ void load_lds4(const void* g, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(g) : "m0", "memory");
}
// until at most N of the wave's own global loads and stores are under way
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// until the wave's LDS reads have returned (before their place is loaded again)
__device__ __forceinline__ void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
// 64 bits of each lane, transposed inside each 16 lanes: lane i gets element
// i % 4 of lanes 4e + i / 4, e = 0..3
__device__ __forceinline__ s16x4 lds_read_tr(uint32_t at, int plus = 0) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)((const lds_char*)(uintptr_t)at + plus));
}
__device__ __forceinline__ u32x4 lds_read16(uint32_t at, int plus = 0) {
  return *(const __attribute__((address_space(3))) u32x4*)((const lds_char*)(uintptr_t)at + plus);
}

// largest of three in one instruction (v_maximum3_f32; NaN if one of them is)
__device__ __forceinline__ float max3(float x, float y, float z) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z);
}

// Words that cross workgroups (split partials): agent-scope accesses, which
// pass the per-XCD L2 caches by.
__device__ __forceinline__ void put_word(float* p, float v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float get_word(const float* p) {
  return __hip_atomic_load(const_cast<float*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Four widths of a finished row (rr: row of sequence start r0 and KV head g,
// position by position), weighted values `acc` against the largest logit m
// (log2 units) with sum l.
template <int D, bool F16>
__device__ __forceinline__ void store_row(const AttendArgs& a, int r0, int rr, int g, int w4, f32x4 acc, float m, float l) {
  const int64_t out = (int64_t)(r0 + rr / a.group) * a.Hq + g * a.group + rr % a.group;
  const float inv = 1.f / l;
  uint2 w;
  bool bad = false;
  uint16_t y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float v = l == 0.f ? 0.f : acc[e] * inv;
    bad |= !__builtin_isfinite(v);
    y[e] = to_elem<F16>(v);
  }
  w.x = y[0] | (uint32_t)y[1] << 16;
  w.y = y[2] | (uint32_t)y[3] << 16;
  *reinterpret_cast<uint2*>(a.o + out * D + w4) = w;
  if (w4 == 0) {
    const float lse = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    bad |= l != 0.f && !__builtin_isfinite(lse);
    if (a.lse) a.lse[out] = lse;
  }
  if (bad) latch_nonfinite(a.nonfinite);
}

// Weighted values of one row, joined split by split.
struct Joined {
  float m, l;
  f32x4 acc;
  __device__ __forceinline__ void add(float pm, float pl, f32x4 po) {
    const float nm = fmaxf(m, pm), ref = nm == -INFINITY ? 0.f : nm;
    const float f0 = __builtin_amdgcn_exp2f(m - ref), f1 = __builtin_amdgcn_exp2f(pm - ref);
    l = l * f0 + pl * f1;
    acc = acc * f0 + po * f1;
    m = nm;
  }
  // n partial sums, in their order; the loads of N leave together
  template <int N, class Load>
  __device__ __forceinline__ void add_all(int n, Load load) {
    for (int k0 = 0; k0 < n; k0 += N) {
      float pm[N], pl[N];
      f32x4 po[N];
#pragma unroll
      for (int i = 0; i < N; ++i) load(min(k0 + i, n - 1), pm[i], pl[i], po[i]);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (k0 + i < n) add(pm[i], pl[i], po[i]);
    }
  }
};

__device__ __forceinline__ void add_prefix(const AttendArgs& a, const PrefixParts& pp, int D, int packed, int g, int w4, Joined& j) {
  const int64_t at0 = ((int64_t)(packed / pp.block_rows) * pp.n_split * a.Hkv + g) * pp.block_rows + packed % pp.block_rows;
  const int64_t stride = (int64_t)a.Hkv * pp.block_rows;
  j.add_all<16>(pp.n_split, [&](int k, float& m, float& l, f32x4& o) {
    const int64_t at = at0 + k * stride;
    const float2 ml = *reinterpret_cast<const float2*>(pp.ml + at * 2);
    m = ml.x;
    l = ml.y;
    o = *reinterpret_cast<const f32x4*>(pp.o + at * D + w4);
  });
}

}  // namespace

}  // namespace ckv
