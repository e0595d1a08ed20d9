// Attention of ragged batches over caches in 4 bits (the row of
// include/commitkv.h), few rows at a time.  Row by row it is the attention of
// attend.hip, with keys and values that are the fp16 numbers the codes stand for.
#include "attend_device.h"
#include "packed_device.h"

namespace ckv {

namespace {

// ---------------------------------------------------------------------------
// A wave takes 16 query rows and its own tokens, 32 at a time, with the products
// S^T = K Q^T and O^T += V^T P^T of attend.hip (v_mfma_f32_16x16x32_f16; lane l:
// c = l % 16, q = l / 16), but its operands are made in registers from codes in LDS.
//
// K: a lane has token c of a block of 16, and of its row the contiguous widths
// D/4 q ..: one read of codes and one of their group's scale and base, eight
// widths an operand register set.  Which widths meet in one product does not
// matter as long as the queries have the same, so these are loaded that way.
//
// V^T: lane (c, q) needs, of widths that it may choose, the values of its eight
// tokens 4q ..3, 16 + 4q ..3 side by side.  It reads the same word of each token's
// codes (widths JW c .., JW = D/16), joins the halves of two tokens' words, and
// has two tokens' codes of one width in the two halves of a word: so the
// transposition costs one instruction per eight codes, and no lane exchange.
// Output register r of product j is width JW (4q + r) + j.
//
// bf16 queries become fp16 times a power of two of their row's own, which its logits
// are divided by again: the largest lies in [2^14, 2^15), elements keep their 8 bits down
// to 2^-31 of it, and smaller ones are off by 2^-39 of it at most.
//
// Bound: HBM, and latency where there are few tiles a wave.  A tile is 5 KB (16 KB in 16
// bits) and takes about 270 vector instructions, 1100 of the 2500 cycles or so in which its
// bytes arrive on a loaded device, so waves count more than bytes under way: two buffers
// and 12 waves a compute unit (LDS holds no more), 64 long ragged sequences 318 us, three
// buffers and 8 waves 337; the loads alone take 279 either way, past the caches 251, and
// then the whole 283 (5.3 TB/s; in 16 bits 862 us).
// ---------------------------------------------------------------------------
template <int D, int NW_>
struct PackedNarrow {
  using R = PackedRow<D>;
  static constexpr int NW = NW_, NT = 64 * NW;
  static constexpr int kTok = 32, kBuf = 2;
  static constexpr int kTileB = kTok * R::kBytes, kChunks = kTileB / 16;
  static constexpr int LOADS = (kChunks + 63) / 64;     // loads of a tile
  static constexpr int kWaveB = kBuf * kTileB + 4 * 256;   // two buffers, four of slots and positions
};

template <int D, bool F16, bool TAB, int NW>
__global__ __launch_bounds__(64 * NW, 3) void attend_packed_narrow_kernel(AttendArgs a, SplitSpace sp, int target, int min_chunk, bool one_round) {
  using L = PackedNarrow<D, NW>;
  using R = PackedRow<D>;
  constexpr int NT = L::NT, KS = D / 32, JW = D / 16;
  __shared__ __align__(16) char tiles[NW * L::kWaveB];
  __shared__ ItemShared ish;
  __shared__ float sm[NW][kNarrowRows], sl[NW][kNarrowRows];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q = lane >> 4;
  const int g = blockIdx.x % a.Hkv;
  const Item it = find_item<NT, kNarrowRows>(a, blockIdx.x / a.Hkv, target, min_chunk, one_round, ish);
  // (a block whose splits pass the grid, which rows out of order can make, is left
  // by all of them: none counts an arrival that the others do not)
  if (it.s < 0 || (it.e - it.split + it.n_split) * a.Hkv > gridDim.x) return;
  const int s = it.s, n = seq_tokens(a.own, s);
  const int r0 = row_start(a, s), Rs = row_start(a, s + 1) - r0;
  const int n_rows = min(kNarrowRows, Rs * a.group - it.rb * kNarrowRows);
  const int p_first = it.rb * kNarrowRows / a.group, p_last = (it.rb * kNarrowRows + n_rows - 1) / a.group;

  // this lane's row
  const int rr = it.rb * kNarrowRows + min(c, n_rows - 1);
  const int p = rr / a.group, h = g * a.group + rr % a.group;
  int qp = row_position(a, s, r0, Rs, p, n, 0);
  u32x4 qf[KS];
  {
    const uint16_t* qr = a.q + (int64_t)(r0 + p) * a.q_row_stride + (int64_t)h * a.q_head_stride;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = ldg_u4(qr + D / 4 * q + 8 * ks);
  }
  float row_sl2 = a.sl2;
  if constexpr (!F16) {
    float most = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) most = largest_finite(qf[ks], most);
    const PowerOfTwo f = factor_of(max_rows16(most));
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = to_f16(qf[ks], f.mul);
    row_sl2 *= f.back;
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
  Range rg = seen_range(a.own, s, n, 0, qmin, qmax, a.window, a.n_sink, !a.qpos && p_last == Rs - 1 && Rs <= n);
  rg.ns = __builtin_amdgcn_readfirstlane(rg.ns);
  rg.shift = __builtin_amdgcn_readfirstlane(rg.shift);
  rg.cnt = __builtin_amdgcn_readfirstlane(rg.cnt);
  // the split's tokens, and the wave's among them: every NW-th tile, so that what
  // the workgroup reads at a time lies together
  const int n_tiles = (rg.cnt + L::kTok - 1) / L::kTok;
  const int per_split = (n_tiles + it.n_split - 1) / it.n_split;
  const int t_begin = min(it.split * per_split, n_tiles), t_end = min(t_begin + per_split, n_tiles);
  const int tile0 = t_begin + wave, my_tiles = max(t_end - tile0 + NW - 1, 0) / NW;

  const uint32_t my = lds_at(tiles) + wave * L::kWaveB, tab = my + L::kBuf * L::kTileB;
  const char* rows_of = reinterpret_cast<const char*>(
      uniform((long long)(uintptr_t)(a.own.k + g * a.own.head_stride + (a.own.slot ? 0 : s * a.own.seq_stride))));
  const int32_t* slots = a.own.slot ? a.own.slot + s * a.own.slot_stride : nullptr;
  const int32_t* poss = a.own.pos ? a.own.pos + s * a.own.pos_stride : nullptr;
  const int64_t row_bytes = a.own.tok_stride * 2;
  // rows that 32-bit offsets reach (24-bit products) take one instruction each
  const int last_row = slots ? a.own.pool_last : max(n - 1, 0);
  const bool near = (uint64_t)last_row * row_bytes + row_bytes < (1ull << 32) && last_row < (1 << 24) && row_bytes < (1 << 24);
  auto token = [&](int tile, int r) { return rg.token(min(tile * L::kTok + r, rg.cnt - 1)); };
  auto word_at = [](uint32_t at) { return *(const __attribute__((address_space(3))) uint32_t*)(uintptr_t)at; };
  // slots (lanes 0-31) and positions (lanes 32-63) of a tile; without one of the tables its lanes read the other
  auto load_tables = [&](int i) {
    if constexpr (TAB) {
      const int tile = tile0 + i * NW;
      const int32_t* from = lane < 32 ? (slots ? slots : poss) : (poss ? poss : slots);
      load_lds4(from + token(tile, lane & 31), tab + (i & 3) * 256);
    }
  };
  // 16-byte chunk x = 64 j + lane of a tile is chunk x % CH of token x / CH: its
  // token's place in a table, and where in the row it lies (opaque, or both are worked out again for each tile)
  uint32_t place[L::LOADS];
#pragma unroll
  for (int j = 0; j < L::LOADS; ++j) {
    const int x = min(64 * j + lane, L::kChunks - 1);
    place[j] = (uint32_t)(x / R::CH * 4) << 16 | (uint32_t)(x % R::CH * 16);
    asm volatile("" : "+v"(place[j]));
  }
  auto load_tile = [&](int i) {
    const int tile = tile0 + i * NW;
    const uint32_t to = my + i % L::kBuf * L::kTileB, words = tab + (i & 3) * 256;
    int rows[L::LOADS];
#pragma unroll
    for (int j = 0; j < L::LOADS; ++j) {
      if (TAB && slots) rows[j] = (int)min(word_at(words + (place[j] >> 16)), (uint32_t)a.own.pool_last);
      else rows[j] = token(tile, (int)(place[j] >> 18));
    }
    wait_lds_reads();
    auto all = [&](auto load) {
#pragma unroll
      for (int j = 0; j < L::LOADS; ++j)
        if (L::kChunks % 64 == 0 || 64 * j + lane < L::kChunks) load(j, place[j] & 0xFFFFu);
    };
    if (near) all([&](int j, uint32_t in) { load_lds16_near_once(rows_of, __umul24(rows[j], (uint32_t)row_bytes) + in, to + j * 1024); });
    else all([&](int j, uint32_t in) { load_lds16_once(rows_of + (rows[j] * row_bytes + in), to + j * 1024); });
  };

  f32x4 o[JW];
#pragma unroll
  for (int j = 0; j < JW; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  bool large = false;                        // a row's m is: see kLargeRef
  auto compute = [&](int i) {
    const int tile = tile0 + i * NW;
    const uint32_t buf = my + i % L::kBuf * L::kTileB;
    f32x4 x[2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
      x[tb] = f32x4{0.f, 0.f, 0.f, 0.f};
      const uint32_t row = buf + (16 * tb + c) * R::kBytes;
      uint32_t w[KS];
      if constexpr (D == 128) {
        const u32x4 t = lds_read16(row + 16 * q);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) w[ks] = t[ks];
      } else {
        w[0] = word_at(row + 8 * q);
        w[1] = word_at(row + 8 * q + 4);
      }
      const Scale sc = scale_of(word_at(row + R::kParams + D / 4 * q / 32 * 4));
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x[tb] = mfma16<true>(eight_values(w[ks], sc), qf[ks], x[tb]);
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
            if (TAB && poss) pt = (int)word_at(tab + (i & 3) * 256 + 128 + (16 * tb + 4 * q + r) * 4);
            else pt = rg.token(min(u, rg.cnt - 1));
            vis = vis && sees(pt, qp, a.window, a.n_sink);
          }
          x[tb][r] = vis ? x[tb][r] : -INFINITY;
          mx = fmaxf(mx, x[tb][r]);
        }
    }
    mx = max_rows16(mx) * row_sl2;
    if (__ballot(mx > m) != 0ull) {
      const float nm = fmaxf(mx, m);
      const float al = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - nm);
      l *= al;
#pragma unroll
      for (int j = 0; j < JW; ++j) o[j] *= al;
      m = nm;
      large = any_large(m);
    }
    float ref = m == -INFINITY ? 0.f : m, sl2 = row_sl2;
    if (__builtin_expect(large, 0)) {
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[tb][r] = product(x[tb][r], sl2) - ref;
      ref = 0.f;
      sl2 = 1.f;
    }
    ref -= kNarrowLog<true>;
    // fp16 weights have 3 bits more than a bf16 output: only an fp16 one needs their rest
    u32x4 ph, pl;
    float lt = 0.f;               // the tile's sum: small weights add up before they meet a large l
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tb][r], sl2, -ref));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tb][r + 1], sl2, -ref));
        lt += p0 + p1;
        const uint32_t w = pack2<true>(p0, p1);
        ph[2 * tb + r / 2] = w;
        if constexpr (F16) pl[2 * tb + r / 2] = pack2<true>(p0 - half_of(w, 0), p1 - half_of(w, 1));
      }
    l += lt;
    // words of two tokens: codes of even widths (lo) and of odd ones (hi)
    uint32_t lo[4], hi[4];
    Scale sc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t0 = 16 * (i / 2) + 4 * q + 2 * (i % 2);
      const uint32_t at = buf + t0 * R::kBytes + R::kValue + JW * c / 8 * 4, par = buf + t0 * R::kBytes + R::kValueParams + JW * c / 32 * 4;
      const uint32_t w0 = word_at(at), w1 = word_at(at + R::kBytes);
      lo[i] = __builtin_amdgcn_perm(w1, w0, 0x05040100u);
      hi[i] = __builtin_amdgcn_perm(w1, w0, 0x07060302u);
      if constexpr (JW == 4) {                       // half a word a lane
        lo[i] >>= 8 * (c & 1);
        hi[i] >>= 8 * (c & 1);
      }
      sc[i] = scale_of(word_at(par), word_at(par + R::kBytes));
    }
    auto value = [&](auto P) {
      constexpr int pp = decltype(P)::value;
      auto values = [&](const uint32_t (&w)[4]) {
        return values_of(two_codes<pp>(w[0]), two_codes<pp>(w[1]), two_codes<pp>(w[2]), two_codes<pp>(w[3]), sc[0], sc[1], sc[2], sc[3]);
      };
      const u32x4 even = values(lo), odd = values(hi);
      o[2 * pp] = mfma16<true>(even, ph, o[2 * pp]);
      o[2 * pp + 1] = mfma16<true>(odd, ph, o[2 * pp + 1]);
      if constexpr (F16) {
        o[2 * pp] = mfma16<true>(even, pl, o[2 * pp]);
        o[2 * pp + 1] = mfma16<true>(odd, pl, o[2 * pp + 1]);
      }
    };
    value(Int<0>{});
    value(Int<1>{});
    if constexpr (JW == 8) {
      value(Int<2>{});
      value(Int<3>{});
    }
  };

  // tile i + 1 and the table of tile i + 2 are loaded during tile i
  constexpr int KV = L::LOADS, T = TAB ? 1 : 0;
  if (my_tiles) {
    // From here on the wave counts its loads itself: what the compiler loaded
    // has to have arrived, or its own waits inside the loop would drain them.
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
    asm volatile("" : "+v"(qp), "+v"(row_sl2));
    wait_loads<0>();
    load_tables(0);
    if (1 < my_tiles) load_tables(1);
    if (TAB) wait_loads<0>();
    load_tile(0);
    for (int i = 0; i < my_tiles; ++i) {
      // Under way, oldest first: tables(i + 1), tile(i).
      if (i + 1 < my_tiles) {
        if (i + 2 < my_tiles) {
          load_tables(i + 2);
          wait_loads<KV + T>();
        } else {
          wait_loads<KV>();
        }
        load_tile(i + 1);
        if (i + 2 < my_tiles) wait_loads<KV + T>();
        else wait_loads<KV>();
      } else {
        wait_loads<0>();
      }
      compute(i);
    }
  }
  wait_loads<0>();
  wait_lds_reads();
  {
    constexpr float back = 1.f / (1 << kNarrowLog<true>);
    l *= back;
#pragma unroll
    for (int j = 0; j < JW; ++j) o[j] *= back;
  }

  // A token that only some rows of the block see has weight 0 in the others,
  // and 0 times a value that is not finite is NaN: then the wave's tokens are
  // taken again one by one, each by the rows that see it.
  if (!one) {
    bool bad = !__builtin_isfinite(l);
#pragma unroll
    for (int j = 0; j < JW; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) bad |= !__builtin_isfinite(o[j][r]);
    if (__ballot(bad) != 0ull) {
#pragma unroll
      for (int j = 0; j < JW; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      m = -INFINITY;
      l = 0.f;
      for (int v = 0; v < my_tiles * L::kTok; ++v) {
        const int u = (tile0 + v / L::kTok * NW) * L::kTok + v % L::kTok;
        if (u >= rg.cnt) break;
        const int t = rg.token(u);
        const char* row = rows_of + (slots ? (int)min((uint32_t)slots[t], (uint32_t)a.own.pool_last) : t) * row_bytes;
        float x = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const u32x4 kk = row_values<D>(row, false, KS * q + ks);
#pragma unroll
          for (int e = 0; e < 8; ++e) x = fmaf(elem<true>(chunk_elem(kk, e)), elem<true>(chunk_elem(qf[ks], e)), x);
        }
        x = product(sum_rows16(x), row_sl2);
        if (!sees(poss ? poss[t] : t, qp, a.window, a.n_sink)) continue;
        const float nm = fmaxf(m, x), ref = nm == -INFINITY ? 0.f : nm;
        const float al = __builtin_amdgcn_exp2f(m - ref), w = __builtin_amdgcn_exp2f(x - ref);
        m = nm;
        l = l * al + (q == 0 ? w : 0.f);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const u32x4 y = row_values<D>(row, true, JW * (4 * q + r) / 8);
#pragma unroll
          for (int j = 0; j < JW; ++j) o[j][r] = fmaf(w, half_of(y[(JW * r % 8 + j) / 2], j % 2), o[j][r] * al);
        }
      }
    }
  }

  // a row's sums over the wave's tokens; then over the waves, through LDS
  l = sum_rows16(l);
  float* wo = reinterpret_cast<float*>(tiles + wave * L::kWaveB);          // [16][D + 4]
  static_assert(kNarrowRows * (D + 4) * 4 <= L::kWaveB);
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < JW; j += 4)
      *reinterpret_cast<f32x4*>(wo + c * (D + 4) + JW * (4 * q + r) + j) = f32x4{o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]};
  if (q == 0) {
    sm[wave][c] = m;
    sl[wave][c] = l;
  }
  finish_block<D, F16, NW, true>(a, sp, PrefixParts{nullptr, nullptr, 0, 1}, it, r0, n_rows, g, tiles, L::kWaveB, sm, sl, last);
}

}  // namespace

hipError_t launch_packed_narrow(const AttendArgs& a, const AttendPlan& p, const SplitSpace& sp, hipStream_t s) {
  const dim3 grid((unsigned)p.grid);
  const bool tab = a.own.slot || a.own.pos;
#define CKV_NARROW(D, F16, TAB) \
  if (p.alone) attend_packed_narrow_kernel<D, F16, TAB, 12><<<grid, 768, 0, s>>>(a, sp, p.target, p.min_chunk, true); \
  else attend_packed_narrow_kernel<D, F16, TAB, 4><<<grid, 256, 0, s>>>(a, sp, p.target, p.min_chunk, false)
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
