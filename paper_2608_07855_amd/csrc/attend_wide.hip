// Attention of ragged batches, many rows at a time: prompts, chunks, and the
// rows of a whole batch over the tokens that it shares.
#include "attend_device.h"

#include <algorithm>

namespace ckv {

namespace {

// ---------------------------------------------------------------------------
// A workgroup of 8 waves takes blocks of 256 query rows (a sequence's rows of
// one KV head, position by position, the head's group of query heads
// innermost) and streams tiles of 64 tokens through LDS; a wave keeps 32 rows'
// queries and outputs in registers.
//
// S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16 (a row on lane column
// c = l % 32, tokens 8 (r / 4) + 4 h + r % 4 with h = l / 32 and register r):
// registers 8u .. 8u+7 of a score block are the operand of the second product
// for tokens {16u + 4h ..+3, 16u + 8 + 4h ..+3}, and transposing LDS reads give
// V^T in that order.
//
// The reference of the softmax weights follows a row's largest logit only
// when that passes it by 2^kLag, so that the output is rarely rescaled (sums are
// float32).  In bf16 a weight of any size has 8 bits.  fp16 has 11 from 2^-14 to
// 2^16 and none below 2^-25, and behind a dominant token many smaller weights make
// up the output: so they are formed 2^kWeightLog times as large, up to 2^15, and
// those down to 2^-27 of the largest keep their bits (a smaller one is off by
// 2^-38 of it at most).  A lag of 8 would leave 2^-21 and saves 1% at best (16
// fp16 chunks behind a 16K prefix 760, with a lag of 4 763, of 2 769 us).
//
// Weights are rounded once to the type before they multiply the values (float32
// in the sums).  o's error against 64 bits then grows from its own rounding's
// 0.0017 of o to 0.0019 (prompts, a 64K prefix) or 0.0022 (the largest drawn) in bf16,
// and from 0.00021 to 0.00022 in fp16.  A second product for the rest of each
// weight, as few rows have it, takes that away and 22% (a prompt of 4096 tokens 256
// -> 313 us) to 32% longer (the 64K prefix's call 632 -> 836), and spills.
//
// Bound: matrix and vector issue.  A step is 32 products (1024 cycles) and about
// 150 vector instructions a wave; both waves of a SIMD pass the same barrier a
// tile, so each interleaves the two for itself (see step()): 256 rows of 64
// heads on 65536 shared tokens take 540 us, 1.0 PFLOP/s (588 from an idle device),
// the matrix units busy 46% and the vector units 45% of the cycles, 16 fp16 chunks
// behind a 16K prefix 765 us, 0.77 (37% and 40%; an 8192^3 product reaches 1.2).
// (64 rows a wave and one wave a SIMD read LDS half as often, but spill.)
//
// Work is cut evenly: workgroup e of a KV head takes the same share of the
// head's tokens-to-see as every other, wherever that begins and ends; a block
// that falls into several shares leaves partial sums, which the join kernel
// adds.  (Blocks as items of their own left the device idle at the end: 8
// ragged chunks 323 us, in shares 312, and 290 since nothing spills.)
// ---------------------------------------------------------------------------
template <bool F16>
constexpr int kLag = F16 ? 2 : 8;                      // log2 units
template <bool F16>
constexpr int kWeightLog = F16 ? 15 - kLag<F16> : 0;
constexpr int kAhead = 4;     // operands read from LDS ahead of their products
constexpr int kNW = 8, kNT = 64 * kNW, kRB = 256, kTok = 64;

template <int D>
struct Wide {
  static constexpr int CH = D / 8, LANES = 64 / CH;    // 16-byte chunks of a row, rows of a load
  static constexpr int LOADS = kTok / LANES / kNW;     // loads of a wave for a tile of K (or V)
  static constexpr int kOwn = LOADS * LANES;           // tokens of a tile that a wave loads
  static constexpr int kRowB = 2 * D, kTileB = kTok * kRowB;
  static constexpr int kLds = 6 * kTileB + kNW * 4 * 256;   // three tiles of K, three of V, four tables a wave
};

template <bool F16>
__device__ __forceinline__ f32x16 mfma32(u32x4 x, u32x4 y, f32x16 c) {
  if constexpr (F16) return mfma_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c);
  else return mfma_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c);
}

// two values rounded to the type, packed
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 v = {x, y};
  if constexpr (F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2));
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
  }
}

__device__ __forceinline__ void tile_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---------------------------------------------------------------- shares

// What the blocks of a sequence see, as far as the lengths tell, in tokens:
// block rb sees shared + min(first + rb * step, cap).  It decides how blocks are
// cut, not what they hold.
struct BlockWork {
  int shared, first, cap;
  int step, n_blocks, n_below;   // n_below: blocks that see less than cap
  // of the first k blocks
  __device__ __forceinline__ long long sum(int k) const {
    const int m = min(k, n_below);
    return (long long)k * ((long long)shared + cap) + (long long)m * (first - cap) + (long long)m * (m - 1) / 2 * step;
  }
};

__device__ __forceinline__ BlockWork block_work(const AttendArgs& a, int s, int shared) {
  const int r0 = row_start(a, s), R = max(row_start(a, s + 1) - r0, 0), n = seq_tokens(a.own, s);
  BlockWork w;
  w.n_blocks = (int)(((int64_t)R * a.group + kRB - 1) / kRB);
  w.step = max(kRB / a.group, 1);
  w.shared = shared;
  w.cap = max(a.window ? (int)min((long long)n, (long long)a.window + a.n_sink + w.step) : n, 1);
  // rows at given positions may see all; else the last row of block 0 sees what lies before it
  w.first = a.qpos ? w.cap : min(max(n - R + min(R, w.step), 1), w.cap);
  w.n_below = (int)(((unsigned)(w.cap - w.first) + (unsigned)w.step - 1) / (unsigned)w.step);
  return w;
}
// of a sequence that is the same in every lane
__device__ __forceinline__ BlockWork uniform_work(const AttendArgs& a, int s, int shared) {
  BlockWork w = block_work(a, s, shared);
  w.first = uniform(w.first);
  w.cap = uniform(w.cap);
  w.n_below = uniform(w.n_below);
  w.n_blocks = uniform(w.n_blocks);
  return w;
}

// A share of a KV head's work: from place x of block rb of sequence s on.
struct Share {
  int s, rb;
  long long x;      // inside the block
  long long left;   // of the share
  bool whole;       // blocks are not cut: workgroup e has block e (s, rb, x, left unset)
};

struct ShareShared {
  ItemShared item;
  int s;
  long long at;
};

// Share e of W (fewer where that leaves less than four tiles each).  s < 0: none.
// Cutting blocks costs about six tiles a share (partial sums written and
// joined): where whole blocks end hardly later than that, they stay whole, and
// blocks that run at the same time are neighbours (they share tiles in L2).
template <int NT>
__device__ __forceinline__ Share find_share(const AttendArgs& a, int e, int W, int shared, bool whole, ShareShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_seq = a.own.n_seq;
  auto work = [&](int s, long long& blocks, long long& most) {
    if (s >= n_seq) return 0ll;
    const BlockWork w = block_work(a, s, shared);
    blocks += w.n_blocks;
    if (w.n_blocks) most = max(most, (long long)w.shared + w.cap);
    return w.sum(w.n_blocks);
  };
  Share r = {-1, 0, 0, 0, whole};
  if (whole) return r;
  long long blocks = 0, most = 0, total = 0, mine = 0, upto = 0;
  if (n_seq <= 64) {
    mine = work(lane, blocks, most);
    upto = wave_scan(mine);
    total = __shfl(upto, 63, 64);
#pragma unroll
    for (int off = 32; off; off >>= 1) {
      blocks += __shfl_xor(blocks, off, 64);
      most = max(most, (long long)__shfl_xor(most, off, 64));
    }
  } else {
    for (int s = tid; s < n_seq; s += NT) total += work(s, blocks, most);
    total = block_sum<NT>(total, sh.item.wave);
    blocks = block_sum<NT>(blocks, sh.item.wave);
    __syncthreads();
#pragma unroll
    for (int off = 32; off; off >>= 1) most = max(most, (long long)__shfl_xor(most, off, 64));
    if (lane == 0) sh.item.wave[wave] = most;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) most = max(most, sh.item.wave[w]);
  }
  r.whole = (blocks + W - 1) / W * most <= total / W + 6 * kTok;
  r.whole = uniform(r.whole);
  if (r.whole || total == 0) return r;
  const long long n = max(min((long long)W, total / (4 * kTok)), 1ll);
  if (e >= n) return r;
  const long long lo = (long long)((double)total * e / n), hi = e + 1 < n ? (long long)((double)total * (e + 1) / n) : total;
  if (n_seq <= 64) {
    const unsigned long long who = __ballot(lo >= upto - mine && lo < upto);
    if (!who) return r;
    r.s = __ffsll(who) - 1;
    r.x = lo - __shfl(upto - mine, r.s, 64);
  } else {
    if (tid == 0) sh.s = -1;
    long long before = 0;
    for (int s0 = 0; s0 < n_seq; s0 += NT) {
      mine = work(s0 + tid, blocks, most);
      long long v = wave_scan(mine);
      __syncthreads();
      if (lane == 63) sh.item.wave[wave] = v;
      __syncthreads();
      long long all = 0;
      for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) v += sh.item.wave[w];
        all += sh.item.wave[w];
      }
      const long long at = lo - before - (v - mine);
      if (at >= 0 && at < mine) {
        sh.s = s0 + tid;
        sh.at = at;
      }
      before += all;
      if (before > lo) break;
    }
    __syncthreads();
    if (sh.s < 0) return r;
    r.s = sh.s;
    r.x = sh.at;
  }
  r.s = uniform(r.s);
  r.x = uniform(r.x);
  r.left = uniform(hi - lo);
  // the block
  const BlockWork w = uniform_work(a, r.s, shared);
  int k0 = 0, k1 = w.n_blocks;
  while (k1 - k0 > 1) {
    const int k = (k0 + k1) >> 1;
    if (w.sum(k) <= r.x) k0 = k;
    else k1 = k;
  }
  r.rb = uniform(k0);
  r.x = uniform(r.x - w.sum(k0));
  return r;
}

// first tile of place x of a part of `work` tokens that has n tiles
__device__ __forceinline__ int tile_at(long long x, long long work, int n) {
  if (x <= 0) return 0;
  if (x >= work) return n;
  return (int)min((long long)n, (x * n + work - 1) / work);
}

// The cache (or the shared tokens) that a block reads: its tokens and the
// share's tiles of them.
struct Part {
  Range rg;
  int n, base, sq, tile0, tile1;
  int full_lo, full_hi;   // tokens that every row of the wave sees: [full_lo, full_hi), and first ones before full_hi
  int row_lo, row_hi;   // tokens that the lane's row sees: [row_lo, row_hi), and first ones before row_hi
};

// The kernel's first argument, read from memory where it is used next.
__device__ __forceinline__ const AttendArgs& fresh_args(const AttendArgs&) {
  typedef const __attribute__((address_space(4))) AttendArgs* Ptr;
  Ptr p = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const AttendArgs*)p;
}

enum Kept { kS, kRb, kR0, kRows, kX0, kX1 = kX0 + 2, kWork = kX1 + 2, kQmin = kWork + 2, kQmax, kBmin, kBmax, kNextS, kNextRb,
            kNextX, kLeft = kNextX + 2, kOpening = kLeft + 2, kRecord };

// PRE: the rows of all sequences over the shared tokens, in n_split splits, as
// partial sums.  Otherwise a share of the blocks (W shares a KV head), in each
// the shared tokens first; n_split 1: whole blocks only.
template <int D, bool F16, bool TAB, bool PRE>
__global__ __launch_bounds__(kNT, 2) void attend_wide_kernel(AttendArgs args, SplitSpace sp, int W, int n_split) {
  using L = Wide<D>;
  constexpr int KS = D / 16, DB = D / 32;
  __shared__ __align__(256) char tiles[L::kLds];
  __shared__ ShareShared ssh;
  __shared__ int qlim[2][kNW];
  // What a block needs again behind its tiles waits in LDS (a copy a wave), and
  // the arguments are read anew: kept in scalar registers through the tiles they
  // spill, and a spilled register's reload inside the loop drains the loads.
  __shared__ volatile int kept[kNW][32];
  // (One block, and no second part, leave registers enough: PRE keeps both.)
  auto fresh = [&]() -> const AttendArgs& {
    if constexpr (PRE) return args;
    else return fresh_args(args);
  };
  const AttendArgs& a = fresh();
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), c = lane & 31, hf = lane >> 5;
  const int g = blockIdx.x % a.Hkv, e = blockIdx.x / a.Hkv;
  const int pre_n = a.has_pre ? uniform(seq_tokens(a.pre, 0)) : 0;
  const uint32_t lds = lds_at(tiles), tab = lds + 6 * L::kTileB + wave * 4 * 256;
  const int grp = lane / L::CH, ch = lane % L::CH;
  // where in its row the lane's chunk comes from (row r of a tile: chunk ch ^ r, for V ch ^ 2 r)
  const uint32_t kc = (ch ^ ((wave * L::kOwn + grp) & (L::CH - 1))) << 4;
  const uint32_t vc = (ch ^ (2 * (wave * L::kOwn + grp) & (L::CH - 1))) << 4;

  // Per-lane places of the operands inside a tile; the rest is a constant.
  // K: row 32 tb + c, chunk 2 ks + h.  V: token 16 st + 8 part + 4 h + l % 16 / 4,
  // chunk 4 db + 2 (l / 16 % 2) + l % 4 / 2, half a chunk l % 2.  (The chunks of
  // a row are exchanged by XOR with the token against bank conflicts.)
  // Chunk 2 ks + h of token c lies at ((2 ks + h) ^ c) = (h ^ c) ^ 2 ks, so that
  // one register an operand and a XOR give all of them.
  const uint32_t ka = lds + c * L::kRowB + ((hf ^ (c & (L::CH - 1))) << 4);
  uint32_t va;
  {
    const int r = 4 * hf + ((lane & 15) >> 2), chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    va = lds + 3 * L::kTileB + r * L::kRowB + ((chunk ^ (2 * r & (L::CH - 1))) << 4) + 8 * (lane & 1);
  }

  Share me;
  bool whole = false;
  if constexpr (PRE) {
    me = {0, e / n_split, 0, 1, false};
  } else {
    me = find_share<kNT>(a, e, W, pre_n, n_split != 0, ssh);
    whole = me.whole;
    if (sp.share && e < W && tid == 0 && (whole || me.s < 0)) sp.share[blockIdx.x] = make_int4(0, 0, 0, 0);
    if (whole) {
      const Item it = find_item<kNT, kRB>(a, e, 1, INT_MAX, false, ssh.item);
      me = {it.s, it.rb, 0, 1, true};
    }
    if (me.s < 0) return;
  }
  auto keep = [&](int i, int v) {
    if (lane == 0) kept[wave][i] = v;
  };
  auto keep64 = [&](int i, long long v) {
    keep(i, (int)v);
    keep(i + 1, (int)(v >> 32));
  };
  auto get = [&](int i) { return uniform(kept[wave][i]); };
  auto get64 = [&](int i) { return (long long)((unsigned long long)(unsigned)get(i) | (unsigned long long)(unsigned)get(i + 1) << 32); };
  int4 record = make_int4(0, 0, 0, 0);
  for (bool opening = true; me.left > 0; opening = false) {
    if (!opening) tile_barrier();          // the block before is done with LDS
    const AttendArgs& a = fresh();
    // the share's part of this block
    const int s = me.s, rb = me.rb;
    const int r0 = uniform(row_start(a, PRE ? 0 : s)), R = uniform(row_start(a, PRE ? a.own.n_seq : s + 1)) - r0;
    if (PRE && (int64_t)rb * kRB >= (int64_t)R * a.group) return;
    const int n_rows = min(kRB, R * a.group - rb * kRB);
    long long x0 = 0, x1 = 0, work = 0;
    if constexpr (!PRE) {
      const BlockWork w = uniform_work(a, s, pre_n);
      work = w.sum(rb + 1) - w.sum(rb);
      x0 = me.x;
      x1 = whole ? work : min(work, x0 + me.left);
      me.left -= x1 - x0;
      me.x = 0;
      if (++me.rb >= w.n_blocks && me.left > 0) {
        me.rb = 0;
        do ++me.s;
        while (me.s < a.own.n_seq && uniform(row_start(a, me.s)) >= uniform(row_start(a, me.s + 1)));
        if (me.s >= a.own.n_seq) me.left = 0;
      }
    } else {
      me.left = 0;
    }

    // the lane's row: its position and query
    int qp;
    u32x4 qf[KS];
    const bool wave_on = wave * 32 < n_rows;
    const int i = min(wave * 32 + c, n_rows - 1);
    const int rr = rb * kRB + i, p = rr / a.group, h = g * a.group + rr % a.group;
    if constexpr (PRE) {
      const int row = r0 + p, rs = max(row_seq(a, row), 0), f = row_start(a, rs);
      qp = row_position(a, rs, f, row_start(a, rs + 1) - f, row - f, seq_tokens(a.own, rs), pre_n);
    } else {
      qp = row_position(a, s, r0, R, p, seq_tokens(a.own, s), pre_n);
    }
    const uint16_t* qr = a.q + (int64_t)(r0 + p) * a.q_row_stride + (int64_t)h * a.q_head_stride;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = ldg_u4(qr + 16 * ks + 8 * hf);
    int qmin = qp, qmax = qp;
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      qmin = min(qmin, __shfl_xor(qmin, off, 64));
      qmax = max(qmax, __shfl_xor(qmax, off, 64));
    }
    if (lane == 0) {
      qlim[0][wave] = qmin;
      qlim[1][wave] = qmax;
    }
    __syncthreads();
    int bmin = qmin, bmax = qmax;
#pragma unroll
    for (int w = 0; w < kNW; ++w) {
      bmin = min(bmin, qlim[0][w]);
      bmax = max(bmax, qlim[1][w]);
    }
    if constexpr (!PRE) {
      keep(kS, s);
      keep(kRb, rb);
      keep(kR0, r0);
      keep(kRows, n_rows);
      keep64(kX0, x0);
      keep64(kX1, x1);
      keep64(kWork, work);
      keep(kQmin, qmin);
      keep(kQmax, qmax);
      keep(kBmin, bmin);
      keep(kBmax, bmax);
      keep(kNextS, me.s);
      keep(kNextRb, me.rb);
      keep64(kNextX, me.x);
      keep64(kLeft, me.left);
      keep(kOpening, opening);
      keep(kRecord, record.x);
      keep(kRecord + 1, record.y);
      keep(kRecord + 2, record.z);
      keep(kRecord + 3, record.w);
    }

    f32x16 o[DB];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = zero16();
    bool large = false;           // a row's m is: see kLargeRef
    bool hidden = false;          // some tile held tokens that not all rows see

    auto open = [&](int k) {
      const AttendArgs& a = fresh();
      const SeqCaches& kv = k ? a.own : a.pre;
      int w0 = qmin, w1 = qmax, b0 = bmin, b1 = bmax, sq = 0;
      if constexpr (!PRE) {
        sq = get(kS);
        w0 = get(kQmin);
        w1 = get(kQmax);
        b0 = get(kBmin);
        b1 = get(kBmax);
      }
      Part t;
      t.sq = k ? sq : 0;
      t.n = uniform(seq_tokens(kv, t.sq));
      t.base = k ? pre_n : 0;
      t.rg = seen_range(kv, t.sq, t.n, t.base, b0, b1, a.window, a.n_sink);
      t.rg.ns = uniform(t.rg.ns);
      t.rg.shift = uniform(t.rg.shift);
      t.rg.cnt = uniform(t.rg.cnt);
      t.rg.lo = uniform(t.rg.lo);
      t.rg.hi = uniform(t.rg.hi);
      t.rg.n_first = uniform(t.rg.n_first);
      const Range all = seen_range(kv, t.sq, t.n, t.base, w1, w0, a.window, a.n_sink);   // window of the last, end of the first
      t.full_hi = uniform(all.hi);
      t.full_lo = uniform(all.lo);
      if (kv.pos) {
        // between the wave's first row and the block's last one (lane by lane)
        const int32_t* pos = kv.pos + t.sq * kv.pos_stride;
        auto find = [&](int lo, int hi, long long key) {      // first token with a position past key
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (pos[mid] <= key) lo = mid + 1;
            else hi = mid;
          }
          return lo;
        };
        t.row_hi = find(t.full_hi, t.rg.hi, qp);
        t.row_lo = a.window ? find(t.rg.lo, t.rg.hi, (long long)qp - a.window) : 0;
      } else {
        auto in = [&](long long x) { return (int)min(max(x, 0ll), (long long)t.n); };
        t.row_hi = in((long long)qp + 1 - t.base);
        t.row_lo = a.window ? in((long long)qp - a.window + 1 - t.base) : 0;
      }
      const int n_tiles = (t.rg.cnt + kTok - 1) / kTok;
      if constexpr (PRE) {
        const int split = e % n_split, per = (n_tiles + n_split - 1) / n_split;
        t.tile0 = min(split * per, n_tiles);
        t.tile1 = min(t.tile0 + per, n_tiles);
      } else {
        const long long from = k ? pre_n : 0, len = k ? get64(kWork) - pre_n : pre_n;
        t.tile0 = uniform(tile_at(get64(kX0) - from, len, n_tiles));
        t.tile1 = uniform(tile_at(get64(kX1) - from, len, n_tiles));
      }
      return t;
    };

    const bool has_pre = a.has_pre;
    for (int k = has_pre ? 0 : 1; k < (PRE ? 1 : 2); ++k) {
      const AttendArgs& a = fresh();
      const SeqCaches& kv = k ? a.own : a.pre;
      const Part pt = open(k);
      const float sl2 = a.sl2;
      const Range rg = pt.rg;
      const int tile0 = pt.tile0, tile1 = pt.tile1;
      const int64_t head = g * kv.head_stride + (kv.slot ? 0 : pt.sq * kv.seq_stride);
      const char* kh = reinterpret_cast<const char*>(kv.k + head);
      const char* vh = reinterpret_cast<const char*>(kv.v + head);
      const int32_t* slots = kv.slot ? kv.slot + pt.sq * kv.slot_stride : nullptr;
      const uint32_t row_bytes = (uint32_t)kv.tok_stride * 2;
      // rows that 32-bit offsets reach (24-bit products) take one instruction each
      const int last_row = slots ? kv.pool_last : max(pt.n - 1, 0);
      const bool near = (uint64_t)last_row * row_bytes + row_bytes < (1ull << 32) && last_row < (1 << 24) && row_bytes < (1u << 24);
      auto token = [&](int tile, int r) { return rg.token(min(tile * kTok + r, rg.cnt - 1)); };
      // (where only the other part has a table, any word keeps the count of loads)
      auto load_tables = [&](int tile) {
        if constexpr (TAB)
          load_lds4(slots ? slots + token(tile, wave * L::kOwn + lane % L::kOwn) : a.cu_rows, tab + (tile & 3) * 256);
      };
      auto find_rows = [&](int tile, uint32_t (&rows)[L::LOADS]) {
#pragma unroll
        for (int j = 0; j < L::LOADS; ++j) {
          if (TAB && slots) {
            const auto* w = (const __attribute__((address_space(3))) int*)(uintptr_t)(tab + (tile & 3) * 256);
            rows[j] = min((uint32_t)w[j * L::LANES + grp], (uint32_t)kv.pool_last);
          } else {
            rows[j] = token(tile, wave * L::kOwn + j * L::LANES + grp);
          }
        }
      };
      // K (at lane constant kc) or V of a tile; load j's rows are LANES j further
      auto load_rows = [&](const uint32_t (&rows)[L::LOADS], const char* from, uint32_t lane_c, uint32_t step_c, uint32_t to) {
        wait_lds_reads();
        // (opaque, or the compiler keeps a 64-bit sum for every load in registers)
        asm volatile("" : "+v"(lane_c));
        if (near) {
#pragma unroll
          for (int j = 0; j < L::LOADS; ++j)
            load_lds16_near(from, __umul24(rows[j], row_bytes) + (lane_c ^ (j * step_c)), to + (wave * L::LOADS + j) * 1024);
        } else {
#pragma unroll
          for (int j = 0; j < L::LOADS; ++j)
            load_lds16(from + ((uint64_t)rows[j] * row_bytes + (lane_c ^ (j * step_c))), to + (wave * L::LOADS + j) * 1024);
        }
      };
      auto load_k = [&](int tile, const uint32_t (&rows)[L::LOADS]) {
        load_rows(rows, kh, kc, (L::LANES & (L::CH - 1)) << 4, lds + (tile % 3) * L::kTileB);
      };
      auto load_v = [&](int tile, const uint32_t (&rows)[L::LOADS]) {
        load_rows(rows, vh, vc, (2 * L::LANES & (L::CH - 1)) << 4, lds + (3 + tile % 3) * L::kTileB);
      };

      // scores of a tile (raw products)
      auto score = [&](int tile, f32x16 (&x)[2]) {
        const uint32_t off = (tile % 3) * L::kTileB;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
          x[tb] = zero16();
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const u32x4 kf = lds_read16((ka + off) ^ (32 * ks), tb * 32 * L::kRowB);
            x[tb] = mfma32<F16>(kf, qf[ks], x[tb]);
          }
        }
      };
      // hides what a row does not see
      auto mask = [&](int tile, f32x16 (&x)[2]) {
        const int u0 = tile * kTok, u1 = u0 + kTok - 1, ta = rg.token(u0), te = rg.token(u1);
        if (te < pt.full_hi && (ta >= pt.full_lo || te < rg.n_first)) return;
        hidden = true;
        if (ta >= rg.n_first && u0 >= rg.ns) {
          const uint32_t len = max(pt.row_hi - pt.row_lo, 0), d = ta + 4 * hf - pt.row_lo;
#pragma unroll
          for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              x[tb][r] = d + (uint32_t)(32 * tb + 8 * (r / 4) + r % 4) < len ? x[tb][r] : -INFINITY;
          return;
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int t = rg.token(u0 + 32 * tb + 8 * (r / 4) + 4 * hf + r % 4);
            x[tb][r] = t < pt.row_hi && (t >= pt.row_lo || t < rg.n_first) ? x[tb][r] : -INFINITY;
          }
      };

      // One step: the weights of tile t from its scores x (largest one of a lane
      // mx), beside the scores of tile t + 1 (into y); then tile t's values beside
      // the largest of y.  A wave issues in order, so the vector work is written
      // between the products, and operands are read from LDS kAhead products
      // early; the fences keep the compiler from gathering either.
      auto step = [&](int t, f32x16 (&x)[2], float& mx, f32x16 (&y)[2], float& my) {
        const float top = max32(mx) * sl2;
        if (__ballot(top > m + kLag<F16> || (m == -INFINITY && top > m)) != 0ull) {
          const float nm = top > m ? top : m;
          const float al = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - nm);
          l *= al;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[db] *= al;
          m = nm;
          large = any_large(m);
        }
        float ref = m == -INFINITY ? 0.f : m, mul = sl2;
        if (__builtin_expect(large, 0)) {
#pragma unroll
          for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int r = 0; r < 16; ++r) x[tb][r] = product(x[tb][r], sl2) - ref;
          ref = 0.f;
          mul = 1.f;
        }
        ref -= kWeightLog<F16>;
        u32x4 ph[4];
        float lt = 0.f;       // the tile's sum: small weights add up before they meet a large l
        {
          // past the last tile: what an older tile left, used by nobody
          const uint32_t off = ((t + 1) % 3) * L::kTileB;
          u32x4 kf[kAhead];
          auto read = [&](int j) { return lds_read16((ka + off) ^ (32 * (j / 2)), (j % 2) * 32 * L::kRowB); };
#pragma unroll
          for (int j = 0; j < kAhead; ++j) kf[j] = read(j);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < 2 * KS; ++j) {
            y[j % 2] = mfma32<F16>(kf[j % kAhead], qf[j / 2], j < 2 ? zero16() : y[j % 2]);
            if (j + kAhead < 2 * KS) kf[j % kAhead] = read(j + kAhead);
            // the tile's 16 pairs of scores, over the 2 KS products
#pragma unroll
            for (int q = j * 16 / (2 * KS); q < (j + 1) * 16 / (2 * KS); ++q) {
              const int tb = q / 8, r = 2 * (q % 8);
              const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tb][r], mul, -ref));
              const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tb][r + 1], mul, -ref));
              lt = q ? lt + (p0 + p1) : p0 + p1;
              ph[q / 4][q % 4] = pack2<F16>(p0, p1);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          l += lt;
          // keeps the weights here, beside the products
#pragma unroll
          for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(ph[j]));
          asm volatile("" : "+v"(l));
        }
        if (t + 1 < tile1) mask(t + 1, y);
        {
          const uint32_t off = (t % 3) * L::kTileB;
          u32x4 vf[kAhead];
          auto read = [&](int j) {                   // tokens 16 (j / DB) .., widths 32 (j % DB) ..
            const uint2 u = __builtin_bit_cast(uint2, lds_read_tr((va + off) ^ (64 * (j % DB)), 16 * (j / DB) * L::kRowB));
            const uint2 v = __builtin_bit_cast(uint2, lds_read_tr((va + off) ^ (64 * (j % DB)), (16 * (j / DB) + 8) * L::kRowB));
            return u32x4{u.x, u.y, v.x, v.y};
          };
#pragma unroll
          for (int j = 0; j < kAhead; ++j) vf[j] = read(j);
          my = -INFINITY;
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < 4 * DB; ++j) {
            o[j % DB] = mfma32<F16>(vf[j % kAhead], ph[j / DB], o[j % DB]);
            if (j + kAhead < 4 * DB) vf[j % kAhead] = read(j + kAhead);
#pragma unroll
            for (int q = j * 16 / (4 * DB); q < (j + 1) * 16 / (4 * DB); ++q)
              my = max3(my, y[q / 8][2 * (q % 8)], y[q / 8][2 * (q % 8) + 1]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      };

      // A load step j brings V of tile j and K of tile j + 1 (whose rows the next
      // step's V has, too); two steps are under way.
      constexpr int KV = 2 * L::LOADS, T = TAB ? 1 : 0;
      if (tile0 < tile1) {
        if (k == 1 && has_pre) tile_barrier();     // the shared tokens' tiles have been read
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (tile0 + j < tile1) load_tables(tile0 + j);
        if (TAB) wait_loads<0>();
        uint32_t rows[L::LOADS], ahead[L::LOADS];
        find_rows(tile0, rows);
        load_k(tile0, rows);
        if (tile0 + 1 < tile1) {
          find_rows(tile0 + 1, ahead);
          load_k(tile0 + 1, ahead);
        }
        load_v(tile0, rows);
        if (tile0 + 3 < tile1) load_tables(tile0 + 3);
        if (tile0 + 1 < tile1) {
          if (tile0 + 2 < tile1) {
            find_rows(tile0 + 2, rows);
            load_k(tile0 + 2, rows);
          }
          load_v(tile0 + 1, ahead);
        }
        // What the compiler loaded has to have arrived before the loop, or its own
        // waits inside would drain the tiles under way.
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
        asm volatile("" : "+v"(qp));
        f32x16 xa[2], xb[2];
        float ma, mb;
        // under way, oldest first: step t, tables(t + 3), step t + 1; rows: of tile t + 2
        auto turn = [&](int t, bool first, f32x16 (&x)[2], float& mx, f32x16 (&y)[2], float& my) {
          if (t + 3 < tile1) wait_loads<T + KV>();
          else if (t + 2 < tile1) wait_loads<KV>();
          else if (t + 1 < tile1) wait_loads<L::LOADS>();
          else wait_loads<0>();
          tile_barrier();             // step t is there, and no wave reads step t - 1 any more
          if (first && wave_on) {
            score(t, x);
            mask(t, x);
            mx = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = max3(mx, x[0][r], x[1][r]);
          }
          if (first) tile_barrier();  // K of the first tile has been read
          if (t + 2 < tile1) {
            if (t + 4 < tile1) {
              load_tables(t + 4);
              wait_loads<KV + T>();
            } else if (t + 3 < tile1) {
              wait_loads<KV>();
            }
            if (t + 3 < tile1) {
              find_rows(t + 3, ahead);
              load_k(t + 3, ahead);
            }
            load_v(t + 2, rows);
#pragma unroll
            for (int j = 0; j < L::LOADS; ++j) rows[j] = ahead[j];
          }
          if (wave_on) step(t, x, mx, y, my);
        };
        turn(tile0, true, xa, ma, xb, mb);
        for (int t = tile0 + 1; t < tile1; t += 2) {
          turn(t, false, xb, mb, xa, ma);
          if (t + 1 < tile1) turn(t + 1, false, xa, ma, xb, mb);
        }
      }
    }
    wait_loads<0>();

    // What follows the tiles finds its lane, row and query again: kept through
    // the tiles, they would not fit the registers.
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int c2 = ln & 31, hf2 = ln >> 5;
    const AttendArgs& b = fresh();
    int s2 = s, rb2 = rb, r2 = r0, rows2 = n_rows;
    bool begun = true, ends = true, first = true;
    if constexpr (!PRE) {
      s2 = get(kS);
      rb2 = get(kRb);
      r2 = get(kR0);
      rows2 = get(kRows);
      begun = get64(kX0) > 0;
      ends = get64(kX1) >= get64(kWork);
      first = get(kOpening);
      me = {get(kNextS), get(kNextRb), get64(kNextX), get64(kLeft), false};
      record = make_int4(get(kRecord), get(kRecord + 1), get(kRecord + 2), get(kRecord + 3));
    }
    l = sum32(l);
    if constexpr (kWeightLog<F16> > 0) {
      constexpr float back = 1.f / (1 << kWeightLog<F16>);
      l *= back;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= back;
    }
    // A token that only some rows of the block see has weight 0 in the others,
    // and 0 times a value that is not finite is NaN: then the share's tokens
    // are taken again one by one, each by the rows that see it.
    bool lost = !__builtin_isfinite(l);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) lost |= !__builtin_isfinite(o[db][r]);
    if (hidden && __ballot(lost) != 0ull) {
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = zero16();
      m = -INFINITY;
      l = 0.f;
      for (int k = has_pre ? 0 : 1; k < (PRE ? 1 : 2); ++k) {
        const SeqCaches& kv = k ? b.own : b.pre;
        const Part pt = open(k);
        const int64_t head = g * kv.head_stride + (kv.slot ? 0 : pt.sq * kv.seq_stride);
        for (int u = pt.tile0 * kTok; u < min(pt.tile1 * kTok, pt.rg.cnt); ++u) {
          const int t = pt.rg.token(u);
          const int row = kv.slot ? (int)min((uint32_t)kv.slot[pt.sq * kv.slot_stride + t], (uint32_t)kv.pool_last) : t;
          const int64_t at = head + row * kv.tok_stride;
          float x = 0.f;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const u32x4 kk = ldg_u4(kv.k + at + 16 * ks + 8 * hf2);
#pragma unroll
            for (int j = 0; j < 8; ++j) x = fmaf(elem<F16>(chunk_elem(kk, j)), elem<F16>(chunk_elem(qf[ks], j)), x);
          }
          x = product(sum32(x), b.sl2);
          if (!(t < pt.row_hi && (t >= pt.row_lo || t < pt.rg.n_first))) continue;
          const float nm = fmaxf(m, x), ref = nm == -INFINITY ? 0.f : nm;
          const float al = __builtin_amdgcn_exp2f(m - ref), p = __builtin_amdgcn_exp2f(x - ref);
          m = nm;
          l = l * al + p;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              o[db][r] = fmaf(p, elem<F16>(kv.v[at + 32 * db + 8 * (r / 4) + 4 * hf2 + r % 4]), o[db][r] * al);
        }
      }
    }

    if (PRE || begun || !ends) {
      // partial sums: an opening share continues a block that another began
      const bool goes_on = !PRE && first && begun;
      const int64_t item = PRE ? (int64_t)blockIdx.x : 2 * (int64_t)blockIdx.x + (goes_on ? 0 : 1);
      if (goes_on) record.w = ends ? 2 : 1;
      else record = make_int4(s2, rb2, 1, record.w);
      const int row = wave * 32 + c2;
      if (row < rows2) {
        const int64_t at = item * kRB + row;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<f32x4*>(sp.o + at * D + 32 * db + 2 * r + 4 * hf2) =
                f32x4{o[db][r], o[db][r + 1], o[db][r + 2], o[db][r + 3]};
        if (hf2 == 0) *reinterpret_cast<float2*>(sp.ml + at * 2) = make_float2(m, l);
      }
      continue;
    }
    // A wave's rows go through LDS (its own part of the tiles), so that a store
    // covers whole rows.
    constexpr int kPitch = 2 * D + 16;
    static_assert(kRB * kPitch <= 6 * L::kTileB);
    tile_barrier();                                  // no wave reads tiles any more
    const int row0 = wave * 32, row = row0 + c2;
    if (row0 >= rows2) continue;
    char* mine = tiles + row0 * kPitch;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float lse = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    bool bad = l != 0.f && !__builtin_isfinite(lse);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[j] = l == 0.f ? 0.f : o[db][r + j] * inv;
          bad |= !__builtin_isfinite(y[j]);
        }
        *reinterpret_cast<uint2*>(mine + c2 * kPitch + (32 * db + 2 * r + 4 * hf2) * 2) =
            make_uint2(pack2<F16>(y[0], y[1]), pack2<F16>(y[2], y[3]));
      }
    if (bad && row < rows2) latch_nonfinite(b.nonfinite);
    if (b.lse && hf2 == 0 && row < rows2) {
      const int q = rb2 * kRB + row;
      b.lse[(int64_t)(r2 + q / b.group) * b.Hq + g * b.group + q % b.group] = lse;
    }
    wait_lds_reads();                              // the wave's own writes, too
#pragma unroll
    for (int j = 0; j < 32 / L::LANES; ++j) {
      const int r = j * L::LANES + ln / L::CH, ch2 = ln % L::CH, gr = row0 + r;
      if (gr < rows2) {
        const int q = rb2 * kRB + gr;
        const int64_t out = (int64_t)(r2 + q / b.group) * b.Hq + g * b.group + q % b.group;
        *reinterpret_cast<u32x4*>(b.o + out * D + ch2 * 8) = *reinterpret_cast<const u32x4*>(mine + r * kPitch + ch2 * 16);
      }
    }
  }
  if (!PRE && !whole && sp.share && tid == 0) sp.share[blockIdx.x] = record;
}

// Blocks that fell into several shares: the one that share e began and left (its
// record: s, rb, 1), with what the shares after it added (w: 1 and on, 2 done).
template <int D, bool F16>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, SplitSpace sp, int W) {
  const int g = blockIdx.x % a.Hkv, e = blockIdx.x / a.Hkv;
  const int4 began = sp.share[blockIdx.x];
  if (!began.z) return;
  int n = 1;
  for (int w = 1; w == 1 && e + n < W; ++n) w = sp.share[(int64_t)(e + n) * a.Hkv + g].w;
  const int r0 = row_start(a, began.x), R = row_start(a, began.x + 1) - r0;
  const int n_rows = min(kRB, R * a.group - began.y * kRB);
  constexpr int TPR = D / 4;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < n_rows * TPR; i += gridDim.y * 256) {
    const int row = i / TPR, w4 = (i % TPR) * 4;
    Joined j = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    j.template add_all<4>(n, [&](int k, float& m, float& l, f32x4& o) {
      const int64_t item = 2 * ((int64_t)(e + k) * a.Hkv + g) + (k ? 0 : 1), at = item * kRB + row;
      const float2 ml = *reinterpret_cast<const float2*>(sp.ml + at * 2);
      m = ml.x;
      l = ml.y;
      o = *reinterpret_cast<const f32x4*>(sp.o + at * D + w4);
    });
    store_row<D, F16>(a, r0, began.y * kRB + row, g, w4, j.acc, j.m, j.l);
  }
}

}  // namespace

AttendPlan plan_wide(const AttendArgs& a, bool room) {
  AttendPlan p;
  p.rows = kRB;
  p.alone = false;
  p.min_chunk = 0;
  p.target = std::max(1, 256 / a.Hkv);             // a workgroup a compute unit
  const int64_t blocks = (int64_t)a.n_rows * a.group / kRB + std::min(a.own.n_seq, a.n_rows);   // of a head, at most
  p.grid = std::max<int64_t>(p.target, blocks) * a.Hkv;
  p.items = 2 * (int64_t)p.target * a.Hkv;
  p.split = room && p.target > 1;
  return p;
}

PrefixPlan plan_prefix(const AttendArgs& a) {
  PrefixPlan p;
  p.rows = kRB;
  p.blocks = ((int64_t)a.n_rows * a.group + kRB - 1) / kRB;
  // 128 tokens a split at least (8 answers to a 2K prompt 16.9 us; 64: 17.6, 256: 19.2)
  const int64_t tiles = std::max<int64_t>(1, (a.pre.max_tokens + 127) / 128);
  const int64_t wgs = p.blocks * a.Hkv;
  // as many splits as fill the device, then the count that leaves it least idle
  int64_t best = std::max<int64_t>(1, 256 / wgs);
  if (wgs * 2 > 256 && wgs < 2048) {
    double least = 1e30;
    for (int64_t k = 1; k <= 6; ++k) {
      const double t = (double)((wgs * k + 255) / 256) / k * (1 + 0.01 * k);
      if (t < least) {
        least = t;
        best = k;
      }
    }
  }
  p.n_split = (int)std::min(best, tiles);
  return p;
}

#define CKV_WIDE(D, F16, TAB, PRE, GRID, W, K) attend_wide_kernel<D, F16, TAB, PRE><<<GRID, kNT, 0, s>>>(a, sp, W, K)
#define CKV_WIDE3(D, F16, PRE, GRID, W, K) \
  if (tab) CKV_WIDE(D, F16, true, PRE, GRID, W, K); \
  else CKV_WIDE(D, F16, false, PRE, GRID, W, K)
#define CKV_WIDE2(PRE, GRID, W, K) \
  if (a.D == 64) { \
    if (a.f16) { CKV_WIDE3(64, true, PRE, GRID, W, K); } else { CKV_WIDE3(64, false, PRE, GRID, W, K); } \
  } else { \
    if (a.f16) { CKV_WIDE3(128, true, PRE, GRID, W, K); } else { CKV_WIDE3(128, false, PRE, GRID, W, K); } \
  }

hipError_t launch_attend_wide(const AttendArgs& a, const AttendPlan& p, const SplitSpace& sp, hipStream_t s) {
  const dim3 grid((unsigned)p.grid);
  const bool tab = a.own.slot || (a.has_pre && a.pre.slot);
  CKV_WIDE2(false, grid, p.target, p.split ? 0 : 1)
  return hipGetLastError();
}

hipError_t launch_attend_prefix(const AttendArgs& a, const PrefixPlan& p, const SplitSpace& sp, hipStream_t s) {
  const dim3 grid((unsigned)(p.blocks * p.n_split * a.Hkv));
  const bool tab = a.pre.slot != nullptr;
  CKV_WIDE2(true, grid, 0, p.n_split)
  return hipGetLastError();
}

hipError_t launch_attend_join(const AttendArgs& a, const AttendPlan& p, const SplitSpace& sp, hipStream_t s) {
  const dim3 grid((unsigned)(p.target * a.Hkv), 8);
#define CKV_JOIN(D, F16) attend_join_kernel<D, F16><<<grid, 256, 0, s>>>(a, sp, p.target)
  if (a.D == 64) {
    if (a.f16) CKV_JOIN(64, true);
    else CKV_JOIN(64, false);
  } else {
    if (a.f16) CKV_JOIN(128, true);
    else CKV_JOIN(128, false);
  }
#undef CKV_JOIN
  return hipGetLastError();
}

}  // namespace ckv
