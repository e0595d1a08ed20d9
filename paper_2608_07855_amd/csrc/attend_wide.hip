// Attention of ragged batches, many rows at a time: prompts, chunks, and the
// rows of a whole batch over the tokens that it shares.
#include "attend_device.h"

#include <algorithm>

namespace ckv {

namespace {

// ---------------------------------------------------------------------------
// Many rows: a workgroup takes NW x 32 RW query rows and streams tiles of 64
// tokens through LDS; a wave keeps its rows' queries and outputs in registers.
//
// S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16 (a row on lane column
// c = l % 32, tokens 8 (r / 4) + 4 h + r % 4 with h = l / 32 and register r):
// registers 8u .. 8u+7 of a score block are the operand of the second product
// for tokens {16u + 4h ..+3, 16u + 8 + 4h ..+3}, and transposing LDS reads give
// V^T in that order.
//
// The reference of the softmax weights follows a row's largest logit only
// when that passes it by 2^8 (weights up to 256 keep their relative precision
// in either type, sums are float32), so that the output is rarely rescaled.
// ---------------------------------------------------------------------------
constexpr float kLag = 8.f;   // log2 units

template <int D, int RW, int NW>
struct Wide {
  static constexpr int NT = 64 * NW, kRows = 32 * RW * NW, kTok = 64;
  static constexpr int CH = D / 8, LANES = 64 / CH;
  static constexpr int LOADS = kTok / LANES / NW;      // loads of a wave for a tile of K (or V)
  static constexpr int kRowB = 2 * D, kTileB = kTok * kRowB;
  static constexpr int NBUF = 3;
  static constexpr int kLds = NBUF * 2 * kTileB + NW * 4 * 256;
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

// PRE: the rows of all sequences over the shared tokens, `n_split` splits;
// partial sums only.  Otherwise a block of one sequence's rows.
template <int D, bool F16, bool TAB, int RW, int NW, bool PRE>
__global__ __launch_bounds__(64 * NW) void attend_wide_kernel(AttendArgs a, SplitSpace sp, int target, int min_chunk, int n_split) {
  using L = Wide<D, RW, NW>;
  constexpr int NT = L::NT, KS = D / 16, DB = D / 32;
  __shared__ __align__(16) char tiles[L::kLds];
  __shared__ ItemShared ish;
  __shared__ int qlim[2][NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hf = lane >> 5;
  const SeqCaches& kv = PRE ? a.pre : a.own;
  const int g = blockIdx.x % a.Hkv;
  int s, rb, split, splits, r0, R;
  if constexpr (PRE) {
    s = 0;
    split = (blockIdx.x / a.Hkv) % n_split;
    rb = blockIdx.x / a.Hkv / n_split;
    splits = n_split;
    r0 = row_start(a, 0);
    R = row_start(a, a.own.n_seq) - r0;
    if ((int64_t)rb * L::kRows >= (int64_t)R * a.group) return;
  } else {
    const Item it = find_item<NT, L::kRows>(a, blockIdx.x / a.Hkv, target, min_chunk, ish);
    if (it.s < 0) return;
    s = it.s;
    rb = it.rb;
    split = it.split;
    splits = it.n_split;
    r0 = row_start(a, s);
    R = row_start(a, s + 1) - r0;
  }
  const int n = seq_tokens(kv, s), pre_n = a.has_pre ? seq_tokens(a.pre, 0) : 0, base = PRE ? 0 : pre_n;
  const int n_rows = min(L::kRows, R * a.group - rb * L::kRows);

  // the lane's rows: their positions and queries
  int qp[RW];
  u32x4 qf[RW][KS];
  int qmin = INT_MAX, qmax = INT_MIN;
  const bool wave_on = wave * 32 * RW < n_rows;
#pragma unroll
  for (int w = 0; w < RW; ++w) {
    const int i = min((wave * RW + w) * 32 + c, n_rows - 1);
    const int rr = rb * L::kRows + i, p = rr / a.group, h = g * a.group + rr % a.group;
    if constexpr (PRE) {
      const int row = r0 + p;
      const int rs = max(row_seq(a, row), 0), f = row_start(a, rs);
      qp[w] = row_position(a, rs, f, row_start(a, rs + 1) - f, row - f, seq_tokens(a.own, rs), pre_n);
    } else {
      qp[w] = row_position(a, s, r0, R, p, n, base);
    }
    const uint16_t* qr = a.q + (int64_t)(r0 + p) * a.q_row_stride + (int64_t)h * a.q_head_stride;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[w][ks] = ldg_u4(qr + 16 * ks + 8 * hf);
    qmin = min(qmin, qp[w]);
    qmax = max(qmax, qp[w]);
  }
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
  for (int w = 0; w < NW; ++w) {
    bmin = min(bmin, qlim[0][w]);
    bmax = max(bmax, qlim[1][w]);
  }
  Range rg = seen_range(kv, s, n, base, bmin, bmax, a.window, a.n_sink);
  rg.ns = __builtin_amdgcn_readfirstlane(rg.ns);
  rg.shift = __builtin_amdgcn_readfirstlane(rg.shift);
  rg.cnt = __builtin_amdgcn_readfirstlane(rg.cnt);
  // tokens that every row of the wave sees: [full_lo, full_hi) and [0, full_ns)
  int full_lo, full_hi, full_ns;
  {
    const Range all = seen_range(kv, s, n, base, qmax, qmin, a.window, a.n_sink);   // window of the last, end of the first
    const bool joined = all.shift == 0;
    full_hi = __builtin_amdgcn_readfirstlane(joined ? all.cnt : all.cnt + all.shift);
    full_lo = __builtin_amdgcn_readfirstlane(joined ? 0 : all.ns + all.shift);
    full_ns = __builtin_amdgcn_readfirstlane(all.ns);
  }
  const int n_tiles = (rg.cnt + L::kTok - 1) / L::kTok;
  const int per_split = (n_tiles + splits - 1) / splits;
  const int tile0 = min(split * per_split, n_tiles), tile1 = min(tile0 + per_split, n_tiles);

  const uint32_t lds = lds_at(tiles), tab = lds + L::NBUF * 2 * L::kTileB + wave * 4 * 256;
  const int grp = lane / L::CH, ch = lane % L::CH;
  constexpr int kOwn = L::LOADS * L::LANES;               // tokens of a tile that the wave loads
  const int64_t head = g * kv.head_stride + (kv.slot ? 0 : s * kv.seq_stride);
  const char* kh = reinterpret_cast<const char*>(kv.k + head);
  const char* vh = reinterpret_cast<const char*>(kv.v + head);
  const int32_t* slots = kv.slot ? kv.slot + s * kv.slot_stride : nullptr;
  const int32_t* poss = kv.pos ? kv.pos + s * kv.pos_stride : nullptr;
  const int64_t row_bytes = kv.tok_stride * 2;
  auto token = [&](int tile, int r) { return rg.token(min(tile * L::kTok + r, rg.cnt - 1)); };
  auto load_tables = [&](int tile) {
    if constexpr (TAB) load_lds4(slots + token(tile, wave * kOwn + lane % kOwn), tab + (tile & 3) * 256);
  };
  auto load_tile = [&](int tile) {
    const uint32_t kb = lds + (tile % L::NBUF) * 2 * L::kTileB, vb = kb + L::kTileB;
    int rows[L::LOADS];
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) {
      if constexpr (TAB) {
        const auto* w = (const __attribute__((address_space(3))) int*)(uintptr_t)(tab + (tile & 3) * 256);
        rows[i] = (int)min((uint32_t)w[i * L::LANES + grp], (uint32_t)kv.pool_last);
      } else {
        rows[i] = token(tile, wave * kOwn + i * L::LANES + grp);
      }
    }
    wait_lds_reads();
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) {
      const int r = wave * kOwn + i * L::LANES + grp;
      const int64_t at = rows[i] * row_bytes;
      load_lds16(kh + at + ((ch ^ (r & (L::CH - 1))) << 4), kb + (wave * L::LOADS + i) * 1024);
      load_lds16(vh + at + ((ch ^ (2 * r & (L::CH - 1))) << 4), vb + (wave * L::LOADS + i) * 1024);
    }
  };

  f32x16 o[RW][DB];
  float m[RW], l[RW];
#pragma unroll
  for (int w = 0; w < RW; ++w) {
    m[w] = -INFINITY;
    l[w] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[w][db] = zero16();
  }
  bool hidden = false;          // some tile held tokens that not all rows see

  auto compute = [&](int tile) {
    const uint32_t kb = lds + (tile % L::NBUF) * 2 * L::kTileB, vb = kb + L::kTileB;
    f32x16 x[RW][2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
#pragma unroll
      for (int w = 0; w < RW; ++w) x[w][tb] = zero16();
      const int r = 32 * tb + c;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const u32x4 kf = lds_read16(kb + r * L::kRowB + (((2 * ks + hf) ^ (r & (L::CH - 1))) << 4));
#pragma unroll
        for (int w = 0; w < RW; ++w) x[w][tb] = mfma32<F16>(kf, qf[w][ks], x[w][tb]);
      }
    }
    const int u0 = tile * L::kTok, u1 = u0 + L::kTok - 1, ta = rg.token(u0), te = rg.token(u1);
    const bool full = u1 < rg.cnt && ((ta >= full_lo && te < full_hi) || te < full_ns);
    if (!full) {
      hidden = true;
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int u = u0 + 32 * tb + 8 * (r / 4) + 4 * hf + r % 4, t = rg.token(min(u, rg.cnt - 1));
          const int pt = poss ? poss[t] : base + t;
#pragma unroll
          for (int w = 0; w < RW; ++w)
            x[w][tb][r] = u < rg.cnt && sees(pt, qp[w], a.window, a.n_sink) ? x[w][tb][r] : -INFINITY;
        }
    }
    u32x4 ph[RW][4];
#pragma unroll
    for (int w = 0; w < RW; ++w) {
      float mx = -INFINITY;
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[w][tb][r]);
      mx = max32(mx) * a.sl2;
      if (__ballot(mx > m[w] + kLag || (m[w] == -INFINITY && mx > m[w])) != 0ull) {
        const float nm = mx > m[w] ? mx : m[w];
        const float al = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[w] - nm);
        l[w] *= al;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[w][db] *= al;
        m[w] = nm;
      }
      const float ref = m[w] == -INFINITY ? 0.f : m[w];
      float sum = 0.f;
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[w][tb][r], a.sl2, -ref));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[w][tb][r + 1], a.sl2, -ref));
          sum += p0 + p1;
          ph[w][2 * tb + r / 8][(r % 8) / 2] = pack2<F16>(p0, p1);
        }
      l[w] += sum;
    }
#pragma unroll
    for (int st = 0; st < 4; ++st)            // 16 tokens
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        u32x4 vf;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          const int r = 16 * st + 8 * part + 4 * hf + ((lane & 15) >> 2);
          const int chunk = 4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
          const s16x4 t = lds_read_tr(vb + r * L::kRowB + ((chunk ^ (2 * r & (L::CH - 1))) << 4) + 8 * (lane & 1));
          const uint2 x2 = __builtin_bit_cast(uint2, t);
          vf[2 * part] = x2.x;
          vf[2 * part + 1] = x2.y;
        }
#pragma unroll
        for (int w = 0; w < RW; ++w) o[w][db] = mfma32<F16>(vf, ph[w][st], o[w][db]);
      }
  };

  constexpr int KV = 2 * L::LOADS, T = TAB ? 1 : 0;
  if (tile0 < tile1) {
#pragma unroll
    for (int w = 0; w < RW; ++w) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[w][ks]));
      asm volatile("" : "+v"(qp[w]));
    }
    wait_loads<0>();
    load_tables(tile0);
    if (tile0 + 1 < tile1) {
      load_tables(tile0 + 1);
      wait_loads<T>();
    } else {
      wait_loads<0>();
    }
    load_tile(tile0);
    if (tile0 + 1 < tile1) {
      if (tile0 + 2 < tile1) {
        load_tables(tile0 + 2);
        wait_loads<KV + T>();
      } else {
        wait_loads<KV>();
      }
      load_tile(tile0 + 1);
    }
    for (int t = tile0; t < tile1; ++t) {
      // under way, oldest first: tile(t), tables(t + 2), tile(t + 1)
      if (t + 2 < tile1) wait_loads<T + KV>();
      else if (t + 1 < tile1) wait_loads<KV>();
      else wait_loads<0>();
      tile_barrier();             // tile t is there, and no wave reads tile t - 1 any more
      if (t + 2 < tile1) {
        if (t + 3 < tile1) {
          load_tables(t + 3);
          wait_loads<KV + T>();
        } else {
          wait_loads<KV>();
        }
        load_tile(t + 2);
      }
      if (wave_on) compute(t);
    }
  }
  wait_loads<0>();
  if (!wave_on) return;

#pragma unroll
  for (int w = 0; w < RW; ++w) {
    l[w] = sum32(l[w]);
    if (hidden) {
      // as in the few-rows kernel: values that are not finite under a weight of 0
      bool bad = !__builtin_isfinite(l[w]);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) bad |= !__builtin_isfinite(o[w][db][r]);
      if (__ballot(bad) != 0ull) {
#pragma unroll
        for (int db = 0; db < DB; ++db) o[w][db] = zero16();
        m[w] = -INFINITY;
        l[w] = 0.f;
        for (int u = tile0 * L::kTok; u < min(tile1 * L::kTok, rg.cnt); ++u) {
          const int t = rg.token(u);
          const int64_t at = (slots ? (int)min((uint32_t)slots[t], (uint32_t)kv.pool_last) : t) * row_bytes;
          float x = 0.f;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const u32x4 kk = ldg_u4(kh + at + (16 * ks + 8 * hf) * 2);
#pragma unroll
            for (int e = 0; e < 8; ++e) x = fmaf(elem<F16>(chunk_elem(kk, e)), elem<F16>(chunk_elem(qf[w][ks], e)), x);
          }
          x = sum32(x) * a.sl2;
          if (!sees(poss ? poss[t] : base + t, qp[w], a.window, a.n_sink)) continue;
          const float nm = fmaxf(m[w], x), ref = nm == -INFINITY ? 0.f : nm;
          const float al = __builtin_amdgcn_exp2f(m[w] - ref), p = __builtin_amdgcn_exp2f(x - ref);
          m[w] = nm;
          l[w] = l[w] * al + p;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              o[w][db][r] = fmaf(p, elem<F16>(reinterpret_cast<const uint16_t*>(vh + at)[32 * db + 8 * (r / 4) + 4 * hf + r % 4]),
                                 o[w][db][r] * al);
        }
      }
    }
    const int i = (wave * RW + w) * 32 + c;
    if (i >= n_rows) continue;
    if (!PRE && splits == 1 && !a.has_pre) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          store_row<D, F16>(a, r0, rb * L::kRows + i, g, 32 * db + 2 * r + 4 * hf,
                            f32x4{o[w][db][r], o[w][db][r + 1], o[w][db][r + 2], o[w][db][r + 3]}, m[w], l[w]);
    } else {
      const int64_t at = (int64_t)blockIdx.x * L::kRows + i;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *reinterpret_cast<f32x4*>(sp.o + at * D + 32 * db + 2 * r + 4 * hf) =
              f32x4{o[w][db][r], o[w][db][r + 1], o[w][db][r + 2], o[w][db][r + 3]};
      if (hf == 0) {
        sp.ml[at * 2] = m[w];
        sp.ml[at * 2 + 1] = l[w];
      }
    }
  }
}

// The splits of the many-rows kernel, and the shared tokens, joined: a
// workgroup takes one row block of a KV head (those that finished alone and
// share nothing are left).
template <int D, bool F16, int RB>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, SplitSpace sp, int target, int min_chunk, PrefixParts pp) {
  __shared__ ItemShared ish;
  const int g = blockIdx.x % a.Hkv;
  const Item it = find_item<256, RB>(a, blockIdx.x / a.Hkv, target, min_chunk, ish);
  if (it.s < 0 || it.split != 0 || (it.n_split == 1 && pp.n_split == 0)) return;
  const int r0 = row_start(a, it.s), R = row_start(a, it.s + 1) - r0;
  const int n_rows = min(RB, R * a.group - it.rb * RB);
  constexpr int TPR = D / 4;
  const int lead = (r0 - row_start(a, 0)) * a.group + it.rb * RB;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < n_rows * TPR; i += gridDim.y * 256) {
    const int row = i / TPR, w4 = (i % TPR) * 4;
    Joined j = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    for (int k = 0; k < it.n_split; ++k) {
      const int64_t at = ((int64_t)blockIdx.x + (int64_t)k * a.Hkv) * RB + row;
      j.add(sp.ml[at * 2], sp.ml[at * 2 + 1], *reinterpret_cast<const f32x4*>(sp.o + at * D + w4));
    }
    if (pp.n_split) add_prefix(a, pp, D, lead + row, g, w4, j);
    store_row<D, F16>(a, r0, it.rb * RB + row, g, w4, j.acc, j.m, j.l);
  }
}

constexpr int kRW = 1, kNW = 8, kRB = 32 * kRW * kNW;

}  // namespace

AttendPlan plan_wide(const AttendArgs& a, int64_t max_tokens, bool room) {
  AttendPlan p;
  p.rows = kRB;
  const int64_t n_seq = std::min(a.own.n_seq, a.n_rows);
  const int64_t blocks = (int64_t)a.n_rows * a.group / kRB + n_seq;     // row blocks of a KV head, at most
  p.target = 512;
  p.min_chunk = 256;
  int64_t e = p.target / a.Hkv + blocks + 1;
  if (!room || max_tokens <= p.min_chunk || blocks * a.Hkv >= p.target) {
    p.min_chunk = INT_MAX;                                              // no splits
    e = blocks;
  }
  p.items = e * a.Hkv;
  p.split = p.min_chunk != INT_MAX;
  return p;
}

PrefixPlan plan_prefix(const AttendArgs& a) {
  PrefixPlan p;
  p.rows = kRB;
  p.blocks = ((int64_t)a.n_rows * a.group + kRB - 1) / kRB;
  const int64_t tiles = std::max<int64_t>(1, (a.pre.max_tokens + 63) / 64);
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

#define CKV_WIDE(D, F16, TAB, PRE, GRID, K) \
  attend_wide_kernel<D, F16, TAB, kRW, kNW, PRE><<<GRID, 64 * kNW, 0, s>>>(a, sp, target, min_chunk, K)
#define CKV_WIDE3(D, F16, PRE, GRID, K) \
  if (tab) CKV_WIDE(D, F16, true, PRE, GRID, K); \
  else CKV_WIDE(D, F16, false, PRE, GRID, K)
#define CKV_WIDE2(PRE, GRID, K) \
  if (a.D == 64) { \
    if (a.f16) { CKV_WIDE3(64, true, PRE, GRID, K); } else { CKV_WIDE3(64, false, PRE, GRID, K); } \
  } else { \
    if (a.f16) { CKV_WIDE3(128, true, PRE, GRID, K); } else { CKV_WIDE3(128, false, PRE, GRID, K); } \
  }

hipError_t launch_attend_wide(const AttendArgs& a, const AttendPlan& p, const SplitSpace& sp, hipStream_t s) {
  const dim3 grid((unsigned)p.items);
  const bool tab = a.own.slot != nullptr;
  const int target = p.target, min_chunk = p.min_chunk;
  CKV_WIDE2(false, grid, 0)
  return hipGetLastError();
}

hipError_t launch_attend_prefix(const AttendArgs& a, const PrefixPlan& p, const SplitSpace& sp, hipStream_t s) {
  const dim3 grid((unsigned)(p.blocks * p.n_split * a.Hkv));
  const bool tab = a.pre.slot != nullptr;
  const int target = 0, min_chunk = 0;
  CKV_WIDE2(true, grid, p.n_split)
  return hipGetLastError();
}

hipError_t launch_attend_join(const AttendArgs& a, const AttendPlan& p, const SplitSpace& sp, const PrefixParts& pp,
                              hipStream_t s) {
  const dim3 grid((unsigned)p.items, 4);
#define CKV_JOIN(D, F16) attend_join_kernel<D, F16, kRB><<<grid, 256, 0, s>>>(a, sp, p.target, p.min_chunk, pp)
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
