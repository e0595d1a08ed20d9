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

// Item e of a KV head: blocks of RB rows, about `target` items over all heads, at least min_chunk tokens each.
template <int NT, int RB>
__device__ Item find_item(const AttendArgs& a, int64_t e, int target, int min_chunk, ItemShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_seq = a.own.n_seq;
  auto load = [&](int s, int& nrb, int& est) {
    nrb = est = 0;
    if (s < n_seq) {
      const int r0 = row_start(a, s), R = max(row_start(a, s + 1) - r0, 0);
      nrb = (int)(((int64_t)R * a.group + RB - 1) / RB);
      est = seen_estimate(a, seq_tokens(a.own, s), min(RB, R * a.group));
    }
  };
  int nrb, est;
  load(tid, nrb, est);
  long long work = (long long)nrb * est;
  for (int s = tid + NT; s < n_seq; s += NT) {
    int b, t;
    load(s, b, t);
    work += (long long)b * t;
  }
  work = block_sum<NT>(work, sh.wave) * a.Hkv;
  const int64_t chunk = max((int64_t)min_chunk, (work + target - 1) / target);
  if (tid == 0) sh.found[0] = -1;
  int64_t before = 0;
  for (int s0 = 0; s0 < n_seq; s0 += NT) {
    if (s0) load(s0 + tid, nrb, est);
    const int n_split = est > 0 ? (int)((est + chunk - 1) / chunk) : 1;
    const long long mine = (long long)nrb * n_split;
    long long v = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const long long u = __shfl_up(v, off, 64);
      if (lane >= off) v += u;
    }
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
  Item it;
  it.s = __builtin_amdgcn_readfirstlane(sh.found[0]);
  it.rb = __builtin_amdgcn_readfirstlane(sh.found[1]);
  it.split = __builtin_amdgcn_readfirstlane(sh.found[2]);
  it.n_split = __builtin_amdgcn_readfirstlane(sh.found[3]);
  it.e = e;
  return it;
}

// First t of [0, n) with pos[t] > key (n if none), pos ascending: a wave
// tries 64 places at once, so 131072 positions take three dependent loads.
__device__ __forceinline__ int upper_bound(const int32_t* pos, int n, long long key) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 0) {
    const int step = (len + 63) / 64;
    const int t = lo + min(lane * step + step - 1, len - 1);     // last place of the lane's part
    const bool le = pos[t] <= key && lane * step < len;
    const int parts = __popcll(__ballot(le));                    // parts that lie at or below the key
    const int skip = min(parts * step, len);
    lo += skip;
    len = min(step - 1, len - skip);
  }
  return lo;
}

// The tokens that rows at positions qmin..qmax see between them, as one range
// of indexes u < cnt: first tokens t = u < ns, then t = u + shift.
struct Range {
  int ns, shift, cnt;
  __device__ __forceinline__ int token(int u) const { return u < ns ? u : u + shift; }
};

__device__ __forceinline__ Range seen_range(const SeqCaches& c, int sq, int n, int base, int qmin, int qmax, int window,
                                            int n_sink) {
  int hi, lo = 0, ns = 0;
  if (c.pos) {
    const int32_t* p = c.pos + sq * c.pos_stride;
    hi = upper_bound(p, n, qmax);
    if (window) {
      lo = upper_bound(p, n, (long long)qmin - window);
      if (n_sink) ns = upper_bound(p, n, (long long)n_sink - 1);
    }
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
  return t >= 0 ? a.own.pos[s * a.own.pos_stride + t] : INT_MIN;
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
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(g) : "memory");
}
__device__ __forceinline__ void load_lds4(const void* g, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(g) : "memory");
}
// until at most N of the wave's own global loads and stores are under way
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// until the wave's LDS reads have returned (before their place is loaded again)
__device__ __forceinline__ void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
// 64 bits of each lane, transposed inside each 16 lanes: lane i gets element
// i % 4 of lanes 4e + i / 4, e = 0..3
__device__ __forceinline__ s16x4 lds_read_tr(uint32_t at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)at);
}
__device__ __forceinline__ u32x4 lds_read16(uint32_t at) {
  return *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)at;
}

template <bool F16>
__device__ __forceinline__ f32x4 mfma16(u32x4 x, u32x4 y, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}

// over the four 16-lane rows of a wave: lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float max_rows16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max32(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_rows16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return sum32(__uint_as_float(r[0]) + __uint_as_float(r[1]));
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

// ---------------------------------------------------------------------------
// Few rows: a wave takes 16 query rows and its own tokens, 32 at a time.
//
// S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_16x16x32: a score block has its
// row on lane column c = l % 16 and tokens 4 q + r (q = l / 16, register r), and
// two blocks of 16 tokens are, register by register, the operand of the second
// product for the token order {4q .. 4q+3, 16+4q .. 16+4q+3}; V^T is read in that
// order by transposing LDS reads, so nothing moves between lanes.
//
// Bound: HBM (2 D 2 bytes a token and KV head against 16 x 32 x D x 4 FLOP a
// tile on the matrix units), so what counts is loads under way: every wave has
// its own two buffers of 32 tokens of K and V, filled by direct loads, without
// any barrier between waves; slots and positions of the tile after the next
// travel the same way (one load of 32 words each).
//
// LDS: token r of a tile is row 4 (r % 8) + r / 8, so that a lane of load i
// (rows i, 8 + i, 16 + i, 24 + i) finds its slots in consecutive words.  The
// 16-byte chunks of a row are exchanged by XOR with the token (K: r, read 8
// tokens at a time; V: 2 (r % 8), read 4 tokens x 32 bytes at a time) against
// bank conflicts.
//
// Softmax weights are split into two values of the type (rounded weight and
// rounded rest), both multiplied: the matrix units have time for it, and the
// output keeps the precision of its own rounding.
// ---------------------------------------------------------------------------
template <int D>
struct Narrow {
  static constexpr int NW = 256 / D;                // waves: 64 KB of tiles a workgroup, two workgroups a compute unit
  static constexpr int NT = 64 * NW;
  static constexpr int kRows = 16, kTok = 32;
  static constexpr int CH = D / 8;                  // 16-byte chunks of a row
  static constexpr int LANES = 64 / CH;             // tokens of one load
  static constexpr int LOADS = kTok / LANES;        // loads of a tile of K (or V)
  static constexpr int kRowB = 2 * D;               // bytes of a row
  static constexpr int kTileB = kTok * kRowB;
  static constexpr int kWaveB = 4 * kTileB + 4 * 256;   // two buffers of K and V, four of slots and positions
  // LDS row of token r: lane group x of load i has token LOADS * x + i
  __device__ static constexpr int row(int r) { return LANES * (r % LOADS) + r / LOADS; }
};

struct SplitSpace {
  float* o;        // [items][rows of a block][D], weighted values against m
  float* ml;       // [items][rows of a block][2]: largest logit (log2 units), sum
  int* arrive;     // [items], zero between calls
};

template <int D, bool F16, bool TAB>
__global__ __launch_bounds__(Narrow<D>::NT) void attend_narrow_kernel(AttendArgs a, SplitSpace sp, int target, int min_chunk) {
  using L = Narrow<D>;
  constexpr int NT = L::NT, NW = L::NW;
  __shared__ __align__(16) char tiles[NW * L::kWaveB];
  __shared__ ItemShared ish;
  __shared__ float sm[NW][16], sl[NW][16];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q = lane >> 4;
  const int g = blockIdx.x % a.Hkv;
  const Item it = find_item<NT, L::kRows>(a, blockIdx.x / a.Hkv, target, min_chunk, ish);
  if (it.s < 0) return;
  const int s = it.s, n = seq_tokens(a.own, s), base = a.has_pre ? seq_tokens(a.pre, 0) : 0;
  const int r0 = row_start(a, s), R = row_start(a, s + 1) - r0;
  const int n_rows = min(L::kRows, R * a.group - it.rb * L::kRows);      // rows of this block
  const int p_first = it.rb * L::kRows / a.group, p_last = (it.rb * L::kRows + n_rows - 1) / a.group;

  // this lane's row
  const int rr = it.rb * L::kRows + min(c, n_rows - 1);
  const int p = rr / a.group, h = g * a.group + rr % a.group;
  int qp = row_position(a, s, r0, R, p, n, base);
  u32x4 qf[D / 32];
  {
    const uint16_t* qr = a.q + (int64_t)(r0 + p) * a.q_row_stride + (int64_t)h * a.q_head_stride;
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) qf[ks] = ldg_u4(qr + 32 * ks + 8 * q);
  }
  const bool one = p_first == p_last;        // one position: what is loaded is what is seen
  int qmin = qp, qmax = qp;
  if (!one) {
#pragma unroll
    for (int off = 8; off; off >>= 1) {
      qmin = min(qmin, __shfl_xor(qmin, off, 64));
      qmax = max(qmax, __shfl_xor(qmax, off, 64));
    }
  }
  Range rg = seen_range(a.own, s, n, base, qmin, qmax, a.window, a.n_sink);
  rg.ns = __builtin_amdgcn_readfirstlane(rg.ns);
  rg.shift = __builtin_amdgcn_readfirstlane(rg.shift);
  rg.cnt = __builtin_amdgcn_readfirstlane(rg.cnt);
  // the split's tokens, and the wave's among them (whole tiles)
  const int n_tiles = (rg.cnt + L::kTok - 1) / L::kTok;
  const int per_split = (n_tiles + it.n_split - 1) / it.n_split;
  const int t_begin = min(it.split * per_split, n_tiles), t_end = min(t_begin + per_split, n_tiles);
  const int per_wave = (t_end - t_begin + NW - 1) / NW;
  const int tile0 = min(t_begin + wave * per_wave, t_end), tile1 = min(tile0 + per_wave, t_end);

  const uint32_t my = lds_at(tiles) + wave * L::kWaveB, tab = my + 4 * L::kTileB;
  const int grp = lane / L::CH, ch = lane % L::CH;
  const char* kh = reinterpret_cast<const char*>(a.own.k + g * a.own.head_stride + (a.own.slot ? 0 : s * a.own.seq_stride));
  const char* vh = reinterpret_cast<const char*>(a.own.v + g * a.own.head_stride + (a.own.slot ? 0 : s * a.own.seq_stride));
  const int32_t* slots = a.own.slot ? a.own.slot + s * a.own.slot_stride : nullptr;
  const int32_t* poss = a.own.pos ? a.own.pos + s * a.own.pos_stride : nullptr;
  const int64_t row_bytes = a.own.tok_stride * 2;

  auto token = [&](int tile, int r) { return rg.token(min(tile * L::kTok + r, rg.cnt - 1)); };
  // slots (lanes 0-31) and positions (lanes 32-63) of a tile; without one of the tables its lanes read the other
  auto load_tables = [&](int tile) {
    if constexpr (TAB) {
      const int32_t* from = lane < 32 ? (slots ? slots : poss) : (poss ? poss : slots);
      load_lds4(from + token(tile, lane & 31), tab + (tile & 3) * 256);
    }
  };
  auto load_tile = [&](int tile) {
    const uint32_t kb = my + (tile & 1) * 2 * L::kTileB, vb = kb + L::kTileB;
    int rows[L::LOADS];
    if (TAB && slots) {
      const auto* w = (const __attribute__((address_space(3))) int*)(uintptr_t)(tab + (tile & 3) * 256 + grp * L::LOADS * 4);
#pragma unroll
      for (int i = 0; i < L::LOADS; ++i) rows[i] = (int)min((uint32_t)w[i], (uint32_t)a.own.pool_last);
    } else {
#pragma unroll
      for (int i = 0; i < L::LOADS; ++i) rows[i] = token(tile, grp * L::LOADS + i);
    }
    wait_lds_reads();
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) {
      const int r = grp * L::LOADS + i;
      const int64_t at = rows[i] * row_bytes;
      load_lds16(kh + at + ((ch ^ (r & (L::CH - 1))) << 4), kb + i * 1024);
      load_lds16(vh + at + ((ch ^ (2 * r & (L::CH - 1))) << 4), vb + i * 1024);
    }
  };

  f32x4 o[D / 16];
#pragma unroll
  for (int db = 0; db < D / 16; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  auto compute = [&](int tile) {
    const uint32_t kb = my + (tile & 1) * 2 * L::kTileB, vb = kb + L::kTileB;
    f32x4 x[2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      x[tb] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int r = 16 * tb + c;
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks)
        x[tb] = mfma16<F16>(lds_read16(kb + L::row(r) * L::kRowB + (((4 * ks + q) ^ (r & (L::CH - 1))) << 4)), qf[ks], x[tb]);
    }
    float mx = -INFINITY;
    const int u0 = tile * L::kTok + 4 * q;
    if (one && (tile + 1) * L::kTok <= rg.cnt) {
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[tb][r]);
    } else {
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int u = u0 + 16 * tb + r;
          bool vis = u < rg.cnt;
          if (!one) {
            int pt;
            if (TAB && poss)
              pt = *(const __attribute__((address_space(3))) int*)(uintptr_t)(tab + (tile & 3) * 256 + 128 + (16 * tb + 4 * q + r) * 4);
            else
              pt = base + rg.token(min(u, rg.cnt - 1));
            vis = vis && sees(pt, qp, a.window, a.n_sink);
          }
          x[tb][r] = vis ? x[tb][r] : -INFINITY;
          mx = fmaxf(mx, x[tb][r]);
        }
    }
    mx = max_rows16(mx) * a.sl2;
    if (__ballot(mx > m) != 0ull) {
      const float nm = fmaxf(mx, m);
      const float al = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - nm);
      l *= al;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) o[db] *= al;
      m = nm;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    u32x4 ph, pl;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tb][r], a.sl2, -ref));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tb][r + 1], a.sl2, -ref));
        l += p0 + p1;
        const uint16_t h0 = to_elem<F16>(p0), h1 = to_elem<F16>(p1);
        ph[2 * tb + r / 2] = h0 | (uint32_t)h1 << 16;
        pl[2 * tb + r / 2] = to_elem<F16>(p0 - elem<F16>(h0)) | (uint32_t)to_elem<F16>(p1 - elem<F16>(h1)) << 16;
      }
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      u32x4 vf;
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        const int r = 16 * tb + 4 * q + (c >> 2);
        const s16x4 t = lds_read_tr(vb + L::row(r) * L::kRowB + (((2 * db + ((c & 3) >> 1)) ^ (2 * r & (L::CH - 1))) << 4) + 8 * (c & 1));
        const uint2 w = __builtin_bit_cast(uint2, t);
        vf[2 * tb] = w.x;
        vf[2 * tb + 1] = w.y;
      }
      o[db] = mfma16<F16>(vf, ph, o[db]);
      o[db] = mfma16<F16>(vf, pl, o[db]);
    }
  };

  // loads of tile t + 1 and tables of tiles t + 2, t + 3 are under way during tile t
  constexpr int KV = 2 * L::LOADS, T = TAB ? 1 : 0;
  if (tile0 < tile1) {
    const int end = tile1 - 1;               // tiles past the wave's last load that one again
    // From here on the wave counts its loads itself: what the compiler loaded
    // has to have arrived, or its own waits inside the loop would drain them.
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) asm volatile("" : "+v"(qf[ks]));
    asm volatile("" : "+v"(qp));
    wait_loads<0>();
    load_tables(tile0);
    load_tables(min(tile0 + 1, end));
    wait_loads<T>();
    load_tile(tile0);
    for (int t = tile0; t < tile1; ++t) {
      // Under way, oldest first: tables(t + 1), tile(t).
      if (t + 1 < tile1) {
        if (t + 2 < tile1) {
          load_tables(t + 2);
          wait_loads<KV + T>();
        } else {
          wait_loads<KV>();
        }
        load_tile(t + 1);
        if (t + 2 < tile1) wait_loads<KV + T>();
        else wait_loads<KV>();
      } else {
        wait_loads<0>();
      }
      compute(t);
    }
  }
  wait_loads<0>();
  wait_lds_reads();

  // A token that only some rows of the block see has weight 0 in the others,
  // and 0 times a value that is not finite is NaN: then the wave's tokens are
  // taken again one by one, each by the rows that see it.
  if (!one) {
    bool bad = !__builtin_isfinite(l);
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) bad |= !__builtin_isfinite(o[db][r]);
    if (__ballot(bad) != 0ull) {
#pragma unroll
      for (int db = 0; db < D / 16; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
      m = -INFINITY;
      l = 0.f;
      for (int u = tile0 * L::kTok; u < min(tile1 * L::kTok, rg.cnt); ++u) {
        const int t = rg.token(u);
        const int64_t at = (slots ? (int)min((uint32_t)slots[t], (uint32_t)a.own.pool_last) : t) * row_bytes;
        float x = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) {
          const u32x4 kk = ldg_u4(kh + at + (32 * ks + 8 * q) * 2);
#pragma unroll
          for (int e = 0; e < 8; ++e) x = fmaf(elem<F16>(chunk_elem(kk, e)), elem<F16>(chunk_elem(qf[ks], e)), x);
        }
        x = sum_rows16(x) * a.sl2;
        if (!sees(poss ? poss[t] : base + t, qp, a.window, a.n_sink)) continue;
        const float nm = fmaxf(m, x), ref = nm == -INFINITY ? 0.f : nm;
        const float al = __builtin_amdgcn_exp2f(m - ref), w = __builtin_amdgcn_exp2f(x - ref);
        m = nm;
        l = l * al + (q == 0 ? w : 0.f);
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            o[db][r] = fmaf(w, elem<F16>(reinterpret_cast<const uint16_t*>(vh + at)[16 * db + 4 * q + r]), o[db][r] * al);
      }
    }
  }

  // a row's sums over the wave's tokens; then over the waves, through LDS
  l = sum_rows16(l);
  float* wo = reinterpret_cast<float*>(tiles + wave * L::kWaveB);          // [16][D + 4]
  constexpr int OP = D + 4;
#pragma unroll
  for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4*>(wo + c * OP + 16 * db + 4 * q) = o[db];
  if (q == 0) {
    sm[wave][c] = m;
    sl[wave][c] = l;
  }
  __syncthreads();
  constexpr int TPR = D / 4;                 // threads of a row, four widths each
  const int64_t item = blockIdx.x;
  for (int i = tid; i < n_rows * TPR; i += NT) {
    const int row = i / TPR, w4 = (i % TPR) * 4;
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) mm = fmaxf(mm, sm[w][row]);
    const float ref = mm == -INFINITY ? 0.f : mm;
    float ll = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm[w][row] - ref);
      ll += f * sl[w][row];
      acc += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(tiles + w * L::kWaveB) + row * OP + w4) * f;
    }
    if (it.n_split == 1) {
      store_row<D, F16>(a, r0, it.rb * L::kRows + row, g, w4, acc, mm, ll);
    } else {
      float* po = sp.o + (item * L::kRows + row) * D + w4;
#pragma unroll
      for (int e = 0; e < 4; ++e) put_word(po + e, acc[e]);
      if (w4 == 0) {
        put_word(sp.ml + (item * L::kRows + row) * 2, mm);
        put_word(sp.ml + (item * L::kRows + row) * 2 + 1, ll);
      }
    }
  }
  if (it.n_split == 1) return;
  // the split that finishes last joins them all, in their order
  const int64_t first = item - (int64_t)it.split * a.Hkv;
  wait_own_stores();
  __syncthreads();
  if (tid == 0) {
    const int before = __hip_atomic_fetch_add(sp.arrive + first, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = before == it.n_split - 1;
    if (last) __hip_atomic_store(sp.arrive + first, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return;
  for (int i = tid; i < n_rows * TPR; i += NT) {
    const int row = i / TPR, w4 = (i % TPR) * 4;
    float mm = -INFINITY, ll = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < it.n_split; ++j) {
      const int64_t at = (first + (int64_t)j * a.Hkv) * L::kRows + row;
      const float pm = get_word(sp.ml + at * 2), pl = get_word(sp.ml + at * 2 + 1);
      f32x4 po;
#pragma unroll
      for (int e = 0; e < 4; ++e) po[e] = get_word(sp.o + at * D + w4 + e);
      const float nm = fmaxf(mm, pm), ref = nm == -INFINITY ? 0.f : nm;
      const float f0 = __builtin_amdgcn_exp2f(mm - ref), f1 = __builtin_amdgcn_exp2f(pm - ref);
      ll = ll * f0 + pl * f1;
      acc = acc * f0 + po * f1;
      mm = nm;
    }
    store_row<D, F16>(a, r0, it.rb * L::kRows + row, g, w4, acc, mm, ll);
  }
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

NarrowPlan plan_narrow(const AttendArgs& a, int64_t max_tokens, bool room) {
  NarrowPlan p;
  const int64_t n_seq = std::min(a.own.n_seq, a.n_rows);
  const int64_t blocks = (int64_t)a.n_rows * a.group / 16 + n_seq;      // row blocks of a KV head, at most
  const int64_t slots = 2 * 256;                                        // workgroups that run at once
  p.target = (int)(2 * slots);
  p.min_chunk = 256;
  int64_t e = p.target / a.Hkv + blocks + 1;
  if (!room || max_tokens <= p.min_chunk || blocks * a.Hkv >= 4 * p.target) {
    p.min_chunk = INT_MAX;                                              // no splits
    e = blocks;
  }
  p.items = e * a.Hkv;
  p.split = p.min_chunk != INT_MAX;
  return p;
}

hipError_t launch_attend_narrow(const AttendArgs& a, const NarrowPlan& p, float* part, int* arrive, hipStream_t s) {
  SplitSpace sp;
  sp.o = part;
  sp.ml = part + p.items * 16 * a.D;
  sp.arrive = arrive;
  const dim3 grid((unsigned)p.items);
  const bool tab = a.own.slot || a.own.pos;
#define CKV_NARROW(D, F16, TAB) attend_narrow_kernel<D, F16, TAB><<<grid, Narrow<D>::NT, 0, s>>>(a, sp, p.target, p.min_chunk)
#define CKV_NARROW2(D, F16) \
  if (tab) CKV_NARROW(D, F16, true); \
  else CKV_NARROW(D, F16, false)
  if (a.D == 64) {
    if (a.f16) { CKV_NARROW2(64, true); } else { CKV_NARROW2(64, false); }
  } else {
    if (a.f16) { CKV_NARROW2(128, true); } else { CKV_NARROW2(128, false); }
  }
#undef CKV_NARROW2
#undef CKV_NARROW
  return hipGetLastError();
}

}  // namespace ckv
