// Attention of a ragged batch over its resident caches: sliding window with
// first tokens that stay visible, and prefixes that a whole batch shares.
//
// Row r (position p) of sequence s and query head h:
//   x_t = scale q.k_t over the tokens with p_t <= p and (no window, or
//   p - p_t < window, or p_t < n_sink);  lse = log sum e^x;  o = sum e^(x - lse) v.
// Logits are carried in log2 units (scale * log2(e)).
#include "attend_device.h"

#include <algorithm>

namespace ckv {

namespace {

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
// its own two buffers of 32 tokens of K and V (128 KB of LDS a compute unit),
// filled by direct loads, without any barrier between waves; slots and positions of the tile after the next
// travel the same way (one load of 32 words each).  64 sequences with windows of
// 4096 tokens take 201 us (5.3 TB/s), two of 131072 tokens 192 (5.6; plain reads of
// 4 GiB reach 7.1, a 2 GiB copy 4.9).
//
// LDS: token r of a tile is row 4 (r % 8) + r / 8, so that a lane of load i
// (rows i, 8 + i, 16 + i, 24 + i) finds its slots in consecutive words.  The
// 16-byte chunks of a row are exchanged by XOR with the token (K: r, read 8
// tokens at a time; V: 2 (r % 8), read 4 tokens x 32 bytes at a time) against
// bank conflicts.
//
// Softmax weights are split into two values of the type (rounded weight and
// rounded rest), both multiplied: the matrix units have time for it, and the
// output keeps the precision of its own rounding.  fp16 has no values below 2^-25,
// and behind a dominant token many smaller weights make up the output: there they
// are formed 2^15 times as large, and those down to 2^-29 of the largest keep their
// bits (a smaller one is off by 2^-40 of it at most).
// ---------------------------------------------------------------------------
template <bool F16>
constexpr int kNarrowLog = F16 ? 15 : 0;            // weights are formed this many powers of two as large

template <int D, int NW_>
struct Narrow {
  static constexpr int NW = NW_, NT = 64 * NW;
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

template <int D, bool F16, bool TAB, int NW>
__global__ __launch_bounds__(64 * NW) void attend_narrow_kernel(AttendArgs a, SplitSpace sp, int target, int min_chunk, PrefixParts pp) {
  using L = Narrow<D, NW>;
  constexpr int NT = L::NT;
  __shared__ __align__(16) char tiles[NW * L::kWaveB];
  __shared__ ItemShared ish;
  __shared__ float sm[NW][16], sl[NW][16];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q = lane >> 4;
  const int g = blockIdx.x % a.Hkv;
  const Item it = find_item<NT, L::kRows>(a, blockIdx.x / a.Hkv, target, min_chunk, NW == 512 / D, ish);
  // (a block whose splits pass the grid, which rows out of order can make, is left
  // by all of them: none counts an arrival that the others do not)
  if (it.s < 0 || (it.e - it.split + it.n_split) * a.Hkv > gridDim.x) return;
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
  Range rg = seen_range(a.own, s, n, base, qmin, qmax, a.window, a.n_sink, !a.qpos && p_last == R - 1 && R <= n);
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
  bool large = false;                        // a row's m is: see kLargeRef
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
      large = any_large(m);
    }
    float ref = m == -INFINITY ? 0.f : m, sl2 = a.sl2;
    if (__builtin_expect(large, 0)) {
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[tb][r] = product(x[tb][r], sl2) - ref;
      ref = 0.f;
      sl2 = 1.f;
    }
    ref -= kNarrowLog<F16>;
    u32x4 ph, pl;
    float lt = 0.f;               // the tile's sum: small weights add up before they meet a large l
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tb][r], sl2, -ref));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tb][r + 1], sl2, -ref));
        lt += p0 + p1;
        const uint16_t h0 = to_elem<F16>(p0), h1 = to_elem<F16>(p1);
        ph[2 * tb + r / 2] = h0 | (uint32_t)h1 << 16;
        pl[2 * tb + r / 2] = to_elem<F16>(p0 - elem<F16>(h0)) | (uint32_t)to_elem<F16>(p1 - elem<F16>(h1)) << 16;
      }
    l += lt;
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
  if constexpr (kNarrowLog<F16> > 0) {
    constexpr float back = 1.f / (1 << kNarrowLog<F16>);
    l *= back;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) o[db] *= back;
  }

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
        x = product(sum_rows16(x), a.sl2);
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
  auto finish = [&](int row, int w4, Joined j) {
    const int rr = it.rb * L::kRows + row;
    if (pp.n_split) {
      const int first = row_start(a, 0), row = r0 + rr / a.group;     // (rows out of order may lie outside the prefix's)
      if (row >= first && row < row_start(a, a.own.n_seq)) add_prefix(a, pp, D, (r0 - first) * a.group + rr, g, w4, j);
    }
    store_row<D, F16>(a, r0, rr, g, w4, j.acc, j.m, j.l);
  };
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
      finish(row, w4, Joined{mm, ll, acc});
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
    Joined all = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    all.template add_all<16>(it.n_split, [&](int k, float& m, float& l, f32x4& o) {
      const int64_t at = (first + (int64_t)k * a.Hkv) * L::kRows + row;
      m = get_word(sp.ml + at * 2);
      l = get_word(sp.ml + at * 2 + 1);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = get_word(sp.o + at * D + w4 + e);
    });
    finish(row, w4, all);
  }
}

}  // namespace

AttendPlan plan_narrow(const AttendArgs& a, int64_t max_tokens, bool room) {
  AttendPlan p;
  p.rows = 16;
  const int64_t n_seq = std::min(a.own.n_seq, a.n_rows);
  const int64_t blocks = (int64_t)a.n_rows * a.group / 16 + n_seq;      // row blocks of a KV head, at most
  // Few row blocks: one round of equal splits on workgroups that have a compute
  // unit's LDS to themselves (512 / D waves): two 128K sequences 191 us, as below
  // 201; a window of 256 tokens 6.0 and 7.0.  More: half as large workgroups,
  // two a compute unit, so that one's prologue runs beside the other's loads;
  // lengths differ from block to block, and two rounds even them out.
  p.alone = blocks * a.Hkv <= 256;
  p.target = p.alone ? 256 : 1024;
  // A workgroup takes 17 us for 1000 tokens, and joining splits costs 5-7 us.
  // Four workgroups a block or more: short splits (one token of a 2048-token
  // cache 12 us, whole 27; of 4 caches of 4096 tokens 19, with splits of 2048
  // 31).  Fewer: what halves save the join takes (16 caches with about 500 tokens
  // in the window: whole 14.7, in halves 16.2 us).
  // (Of `blocks` about two thirds are there, so 10 sequences of 8 KV heads, 80
  // blocks, count as more than 96: 10 caches of 2000 tokens take 28.5 us whole, of
  // 2100 tokens in two splits 24.3, and 8 of 2000 in eight 19.1.)
  const bool small = blocks * a.Hkv <= 96;
  const int64_t seen = a.window ? std::min(max_tokens, (int64_t)a.window + a.n_sink + a.max_rows) : max_tokens;
  p.min_chunk = small ? 256 : 2048;
  int64_t e = p.target / a.Hkv + blocks + 1;
  if (!room || seen <= (small ? 512 : 2048) || blocks * a.Hkv >= 4 * p.target) {
    p.min_chunk = INT_MAX;                                              // no splits
    e = blocks;
  }
  p.items = p.grid = e * a.Hkv;
  p.split = p.min_chunk != INT_MAX;
  return p;
}

hipError_t launch_attend_narrow(const AttendArgs& a, const AttendPlan& p, const SplitSpace& sp, const PrefixParts& pp,
                                hipStream_t s) {
  const dim3 grid((unsigned)p.grid);
  const bool tab = a.own.slot || a.own.pos;
#define CKV_NARROW(D, F16, TAB) \
  if (p.alone) attend_narrow_kernel<D, F16, TAB, 512 / D><<<grid, 64 * 512 / D, 0, s>>>(a, sp, p.target, p.min_chunk, pp); \
  else attend_narrow_kernel<D, F16, TAB, 256 / D><<<grid, 64 * 256 / D, 0, s>>>(a, sp, p.target, p.min_chunk, pp)
#define CKV_NARROW2(D, F16) \
  if (tab) { CKV_NARROW(D, F16, true); } \
  else { CKV_NARROW(D, F16, false); }
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
