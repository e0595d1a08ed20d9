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
constexpr int kAhead = 4;     // operands read from LDS ahead of their products

template <int D, int RW, int NW>
struct Wide {
  static constexpr int NT = 64 * NW, kRows = 32 * RW * NW, kTok = 64;
  static constexpr int CH = D / 8, LANES = 64 / CH;
  static constexpr int LOADS = kTok / LANES / NW;      // loads of a wave for a tile of K (or V)
  static constexpr int kRowB = 2 * D, kTileB = kTok * kRowB;
  static constexpr int kLds = 6 * kTileB + NW * 4 * 256;   // three tiles of K, three of V, four tables a wave
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

  const uint32_t lds = lds_at(tiles), tab = lds + 6 * L::kTileB + wave * 4 * 256;
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
  // K of tile kt and V of tile vt travel together (V is needed one step later)
  auto row_offset = [&](int tile, int i) -> int64_t {
    int row;
    if constexpr (TAB) {
      const auto* w = (const __attribute__((address_space(3))) int*)(uintptr_t)(tab + (tile & 3) * 256);
      row = (int)min((uint32_t)w[i * L::LANES + grp], (uint32_t)kv.pool_last);
    } else {
      row = token(tile, wave * kOwn + i * L::LANES + grp);
    }
    return row * row_bytes;
  };
  auto load_k = [&](int tile) {
    const uint32_t kb = lds + (tile % 3) * L::kTileB;
    int64_t at[L::LOADS];
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) at[i] = row_offset(tile, i);
    wait_lds_reads();
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) {
      const int r = wave * kOwn + i * L::LANES + grp;
      load_lds16(kh + at[i] + ((ch ^ (r & (L::CH - 1))) << 4), kb + (wave * L::LOADS + i) * 1024);
    }
  };
  auto load_v = [&](int tile) {
    const uint32_t vb = lds + (3 + tile % 3) * L::kTileB;
    int64_t at[L::LOADS];
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) at[i] = row_offset(tile, i);
    wait_lds_reads();
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) {
      const int r = wave * kOwn + i * L::LANES + grp;
      load_lds16(vh + at[i] + ((ch ^ (2 * r & (L::CH - 1))) << 4), vb + (wave * L::LOADS + i) * 1024);
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

  // Per-lane places of the operands inside a tile; the rest is a constant.
  // K: row 32 tb + c, chunk 2 ks + h.  V: token 16 st + 8 part + 4 h + l % 16 / 4,
  // chunk 4 db + 2 (l / 16 % 2) + l % 4 / 2, half a chunk l % 2.
  uint32_t ka[KS], va[DB];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) ka[ks] = lds + c * L::kRowB + (((2 * ks + hf) ^ (c & (L::CH - 1))) << 4);
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int r = 4 * hf + ((lane & 15) >> 2), chunk = 4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    va[db] = lds + 3 * L::kTileB + r * L::kRowB + ((chunk ^ (2 * r & (L::CH - 1))) << 4) + 8 * (lane & 1);
  }

  // scores of a tile (raw products)
  auto score = [&](int tile, f32x16 (&x)[RW][2]) {
    const uint32_t off = (tile % 3) * L::kTileB;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
#pragma unroll
      for (int w = 0; w < RW; ++w) x[w][tb] = zero16();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const u32x4 kf = lds_read16(ka[ks] + off, tb * 32 * L::kRowB);
#pragma unroll
        for (int w = 0; w < RW; ++w) x[w][tb] = mfma32<F16>(kf, qf[w][ks], x[w][tb]);
      }
    }
  };
  // hides what a row does not see
  auto mask = [&](int tile, f32x16 (&x)[RW][2]) {
    const int u0 = tile * L::kTok, u1 = u0 + L::kTok - 1, ta = rg.token(u0), te = rg.token(u1);
    if (u1 < rg.cnt && ((ta >= full_lo && te < full_hi) || te < full_ns)) return;
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
    // (vmcnt 0) the positions have arrived on every path: the compiler would
    // wait behind the branch otherwise, and drain the tiles under way each time
    __builtin_amdgcn_s_waitcnt(0x0F70);
  };
  auto largest = [&](const f32x16 (&x)[RW][2], float (&mx)[RW]) {
#pragma unroll
    for (int w = 0; w < RW; ++w) {
      mx[w] = -INFINITY;
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int r = 0; r < 16; r += 2) mx[w] = max3(mx[w], x[w][tb][r], x[w][tb][r + 1]);
    }
  };

  // One step: the weights of tile t from its scores x (largest one of a lane
  // mx), beside the scores of tile t + 1 (into y); then tile t's values beside
  // the largest of y.  A wave issues in order, so the vector work is written
  // between the products, and operands are read from LDS kAhead products early;
  // the fences keep the compiler from gathering either.
  auto step = [&](int t, f32x16 (&x)[RW][2], float (&mx)[RW], f32x16 (&y)[RW][2], float (&my)[RW]) {
    float ref[RW];
#pragma unroll
    for (int w = 0; w < RW; ++w) {
      const float top = max32(mx[w]) * a.sl2;
      if (__ballot(top > m[w] + kLag || (m[w] == -INFINITY && top > m[w])) != 0ull) {
        const float nm = top > m[w] ? top : m[w];
        const float al = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[w] - nm);
        l[w] *= al;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[w][db] *= al;
        m[w] = nm;
      }
      ref[w] = m[w] == -INFINITY ? 0.f : m[w];
    }
    u32x4 ph[RW][4];
    {
      // past the last tile: what an older tile left, used by nobody
      const uint32_t off = ((t + 1) % 3) * L::kTileB;
      u32x4 kf[kAhead];
      auto read = [&](int i) { return lds_read16(ka[i / 2] + off, (i % 2) * 32 * L::kRowB); };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = read(i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 2 * KS; ++i) {
#pragma unroll
        for (int w = 0; w < RW; ++w) y[w][i % 2] = mfma32<F16>(kf[i % kAhead], qf[w][i / 2], i < 2 ? zero16() : y[w][i % 2]);
        if (i + kAhead < 2 * KS) kf[i % kAhead] = read(i + kAhead);
        // the tile's 16 pairs of scores, over the 2 KS products
#pragma unroll
        for (int w = 0; w < RW; ++w)
#pragma unroll
          for (int e = i * 16 / (2 * KS); e < (i + 1) * 16 / (2 * KS); ++e) {
            const int tb = e / 8, r = 2 * (e % 8);
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[w][tb][r], a.sl2, -ref[w]));
            const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[w][tb][r + 1], a.sl2, -ref[w]));
            l[w] += p0 + p1;
            ph[w][e / 4][e % 4] = pack2<F16>(p0, p1);
          }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int w = 0; w < RW; ++w) {
        // keeps the weights here, beside the products
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(ph[w][i]));
        asm volatile("" : "+v"(l[w]));
      }
    }
    if (t + 1 < tile1) mask(t + 1, y);
    {
      const uint32_t off = (t % 3) * L::kTileB;
      u32x4 vf[kAhead];
      auto read = [&](int i) {                   // 16 tokens i / DB, widths 32 (i % DB) ..
        const uint2 p = __builtin_bit_cast(uint2, lds_read_tr(va[i % DB] + off, 16 * (i / DB) * L::kRowB));
        const uint2 q = __builtin_bit_cast(uint2, lds_read_tr(va[i % DB] + off, (16 * (i / DB) + 8) * L::kRowB));
        return u32x4{p.x, p.y, q.x, q.y};
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) vf[i] = read(i);
#pragma unroll
      for (int w = 0; w < RW; ++w) my[w] = -INFINITY;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i) {
#pragma unroll
        for (int w = 0; w < RW; ++w) o[w][i % DB] = mfma32<F16>(vf[i % kAhead], ph[w][i / DB], o[w][i % DB]);
        if (i + kAhead < 4 * DB) vf[i % kAhead] = read(i + kAhead);
#pragma unroll
        for (int w = 0; w < RW; ++w)
#pragma unroll
          for (int e = i * 16 / (4 * DB); e < (i + 1) * 16 / (4 * DB); ++e)
            my[w] = max3(my[w], y[w][e / 8][2 * (e % 8)], y[w][e / 8][2 * (e % 8) + 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  // A load step j brings V of tile j and K of tile j + 1; two steps are under way.
  constexpr int KV = 2 * L::LOADS, T = TAB ? 1 : 0;
  if (tile0 < tile1) {
#pragma unroll
    for (int w = 0; w < RW; ++w) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[w][ks]));
      asm volatile("" : "+v"(qp[w]));
    }
    wait_loads<0>();
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (tile0 + i < tile1) load_tables(tile0 + i);
    wait_loads<0>();
    load_k(tile0);
    if (tile0 + 1 < tile1) load_k(tile0 + 1);
    load_v(tile0);
    if (tile0 + 3 < tile1) load_tables(tile0 + 3);
    if (tile0 + 1 < tile1) {
      if (tile0 + 2 < tile1) load_k(tile0 + 2);
      load_v(tile0 + 1);
    }
    f32x16 xa[RW][2], xb[RW][2];
    float ma[RW], mb[RW];
    // under way, oldest first: step t, tables(t + 3), step t + 1
    auto turn = [&](int t, bool first, f32x16 (&x)[RW][2], float (&mx)[RW], f32x16 (&y)[RW][2], float (&my)[RW]) {
      if (t + 3 < tile1) wait_loads<T + KV>();
      else if (t + 2 < tile1) wait_loads<KV>();
      else if (t + 1 < tile1) wait_loads<L::LOADS>();
      else wait_loads<0>();
      tile_barrier();             // step t is there, and no wave reads step t - 1 any more
      if (first && wave_on) {
        score(t, x);
        mask(t, x);
        largest(x, mx);
      }
      if (first) tile_barrier();  // K of the first tile is read beside the others' next
      if (t + 2 < tile1) {
        if (t + 4 < tile1) {
          load_tables(t + 4);
          wait_loads<KV + T>();
        } else if (t + 3 < tile1) {
          wait_loads<KV>();
        }
        if (t + 3 < tile1) load_k(t + 3);
        load_v(t + 2);
      }
      if (wave_on) step(t, x, mx, y, my);
    };
    turn(tile0, true, xa, ma, xb, mb);
    for (int t = tile0 + 1; t < tile1; t += 2) {
      turn(t, false, xb, mb, xa, ma);
      if (t + 1 < tile1) turn(t + 1, false, xa, ma, xb, mb);
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
    j.template add_all<16>(it.n_split, [&](int k, float& m, float& l, f32x4& o) {
      const int64_t at = ((int64_t)blockIdx.x + (int64_t)k * a.Hkv) * RB + row;
      const float2 ml = *reinterpret_cast<const float2*>(sp.ml + at * 2);
      m = ml.x;
      l = ml.y;
      o = *reinterpret_cast<const f32x4*>(sp.o + at * D + w4);
    });
    if (pp.n_split) add_prefix(a, pp, D, lead + row, g, w4, j);
    store_row<D, F16>(a, r0, it.rb * RB + row, g, w4, j.acc, j.m, j.l);
  }
}

constexpr int kRW = 1, kNW = 8, kRB = 32 * kRW * kNW;

}  // namespace

AttendPlan plan_wide(const AttendArgs& a, int64_t max_tokens, bool room) {
  AttendPlan p;
  p.rows = kRB;
  p.wide = false;
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
  const int64_t tiles = std::max<int64_t>(1, (a.pre.max_tokens + 127) / 128);   // 128 tokens a split at least
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
