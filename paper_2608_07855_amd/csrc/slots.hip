// Block tables and slot tables of a batch from its lengths (ckv_build_slots).
//
// With B rows a block, sequence s holds blocks(n) = ceil(n / B) blocks for n
// tokens.  It gives back(s) = blocks(old) of them when it ends, or takes
// need(s) = blocks(old + new) - blocks(old) for fresh(s) = new tokens, which
// fall into pieces(s) blocks (need(s), and the one that old left open).  The
// free stack after the returns is F = free[0 .. n_free) followed by the
// returned blocks in the order of sequences; the k-th new block of the batch
// is F[top - 1 - k].  So every word of the result follows from the prefix sums
// of these counts over the sequences, and from words that the step does not
// change: blocks that are taken have an index in F of at least the new top,
// blocks that are stored below it, and entries of F past n_free are read from
// the ended sequences' own tables, which stay.  One launch does it all, without
// any order between its workgroups: each forms the prefix sums for itself (a
// few thousand lengths, from L2) and takes a share of the pieces, returned
// blocks and sequences.  A thread writes a piece's tokens, up to four words a
// store (1024 prompts, 920K tokens, 13.5 us; a thread per token spent its time
// finding each token's sequence: 16.6).
//
// Bound: latency (a decoding step of 64 sequences 5.4 us), and with many new
// tokens the stores: a step reads two counts a sequence, moves two words a block
// and writes four words a token, a lane's run of 64 bytes apart from its
// neighbour's in each of four arrays (most of what the 13.5 us above have over the 5.4).
#include "ckv_device.h"
#include "ckv_kernels.h"

#include "commitkv.h"

#include <algorithm>
#include <climits>

namespace ckv {

namespace {

constexpr int kNT = 256;
constexpr int kUnits = 2048;   // prefix sums kept in LDS, one for every `unit` sequences

enum { kNeed, kBack, kFresh, kPieces, kLists };

struct Counts {
  long long n[kLists];
};

struct Shared {
  int sum[kLists][kUnits];     // sums before each unit
  int old[kUnits];             // n_tokens, where a unit is one sequence
  long long wave[kNT / 64][kLists];
  int status;
};

// Blocks of `tokens` rows: shift >= 0 where B is a power of two.  32-bit
// (lengths are below 2^31, so tokens stay below 2^32).
__device__ __forceinline__ unsigned blocks_of(unsigned tokens, int B, int shift) {
  if (shift >= 0) return (tokens >> shift) + ((tokens & (unsigned)(B - 1)) != 0);
  return tokens ? (tokens - 1) / (unsigned)B + 1 : 0u;
}
// blocks that are full
__device__ __forceinline__ unsigned full_of(unsigned tokens, int B, int shift) {
  return shift >= 0 ? tokens >> shift : tokens / (unsigned)B;
}

__device__ __forceinline__ Counts counts_of(int old, int nn, int B, int shift) {
  Counts c = {{0, 0, 0, 0}};
  if (old < 0 || nn < -1) return c;
  const unsigned have = blocks_of((unsigned)old, B, shift);
  if (nn < 0) {
    c.n[kBack] = have;
  } else {
    const unsigned now = blocks_of((unsigned)old + (unsigned)nn, B, shift);
    c.n[kNeed] = now - have;
    c.n[kFresh] = nn;
    if (nn > 0) c.n[kPieces] = now - full_of((unsigned)old, B, shift);
  }
  return c;
}

struct Step {
  const SlotArgs& a;
  const Shared& sh;
  int unit, n_units, nf, top;   // top: entries of F
  int shift;

  __device__ __forceinline__ Counts counts(int s) const {
    return counts_of(a.n_tokens[s], a.n_new[s], a.block_size, shift);
  }

  // Sequence of element i of a list, and i's place inside it: the last unit
  // with sum <= i, then the sequences of the unit one by one.
  __device__ __forceinline__ int find(int list, int i, int& at) const {
    const int* pre = sh.sum[list];
    int lo = 0, hi = n_units;
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (pre[m] <= i) lo = m;
      else hi = m;
    }
    at = i - pre[lo];
    int s = lo * unit;
    if (unit > 1)
      for (; s < a.n_seq - 1; ++s) {
        const int n = (int)counts(s).n[list];
        if (at < n) break;
        at -= n;
      }
    return s;
  }

  // sum of a list before sequence s
  __device__ __forceinline__ int before(int list, int s) const {
    if (unit == 1) return sh.sum[list][s];
    const int u = s / unit;
    int n = sh.sum[list][u];
    for (int t = u * unit; t < s; ++t) n += (int)counts(t).n[list];
    return n;
  }

  __device__ __forceinline__ int held(int s, int64_t i) const {
    return a.block_table ? a.block_table[s * a.block_stride + i] : a.slot[s * a.slot_stride + i];
  }

  // F[i]
  __device__ __forceinline__ int stacked(int i) const {
    if (i < nf) return a.free_blocks[i];
    int at;
    const int s = find(kBack, i - nf, at);
    return held(s, at);
  }
};

// n words x, x + 1, ... at p
__device__ __forceinline__ void store_run(int32_t* p, int x, int n) {
  typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));
  int i = 0;
  for (; i + 4 <= n; i += 4) *reinterpret_cast<i32x4*>(p + i) = i32x4{x + i, x + i + 1, x + i + 2, x + i + 3};
  for (; i < n; ++i) p[i] = x + i;
}

__global__ __launch_bounds__(kNT) void slots_kernel(SlotArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = a.block_size;
  const int unit = max((a.n_seq + kUnits - 1) / kUnits, 1);
  const int n_units = (a.n_seq + unit - 1) / unit;
  const int per = (n_units + kNT - 1) / kNT;           // units of a thread
  const int u0 = min(tid * per, n_units), u1 = min(u0 + per, n_units);
  const int64_t cols = a.block_table ? a.block_cols : a.slot_cols;
  const int shift = (B & (B - 1)) == 0 ? __ffs(B) - 1 : -1;
  if (tid == 0) sh.status = CKV_SLOTS_OK;
  const int nf = *a.n_free;

  Counts mine = {{0, 0, 0, 0}};
  int bad = CKV_SLOTS_OK;
  auto check = [&](int old, int nn) {
    if (old < 0 || nn < -1) {
      bad = CKV_SLOTS_BAD_COUNT;
      return;
    }
    const unsigned now = (unsigned)old + (unsigned)max(nn, 0);
    if (now > a.slot_cols || blocks_of(now, B, shift) > cols) bad = max(bad, CKV_SLOTS_TABLE);
  };
  if (unit == 1) {
    // lengths to LDS, eight loads of a thread under way; then each thread sums
    // its run of sequences from there (n_new waits where a sum will be)
    for (int s0 = tid; s0 < a.n_seq; s0 += 4 * kNT) {
      int o[4], w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = min(s0 + k * kNT, a.n_seq - 1);
        o[k] = a.n_tokens[s];
        w[k] = a.n_new[s];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int s = s0 + k * kNT;
        if (s >= a.n_seq) break;
        check(o[k], w[k]);
        sh.old[s] = o[k];
        sh.sum[kFresh][s] = w[k];
      }
    }
    __syncthreads();
    for (int u = u0; u < u1; ++u) {
      const Counts c = counts_of(sh.old[u], sh.sum[kFresh][u], B, shift);
#pragma unroll
      for (int i = 0; i < kLists; ++i) {
        sh.sum[i][u] = (int)mine.n[i];
        mine.n[i] += c.n[i];
      }
    }
  } else {
    for (int s = u0 * unit; s < min(u1 * unit, a.n_seq); ++s) {
      const int old = a.n_tokens[s], nn = a.n_new[s];
      check(old, nn);
      const Counts c = counts_of(old, nn, B, shift);
#pragma unroll
      for (int i = 0; i < kLists; ++i) mine.n[i] += c.n[i];
    }
  }
  long long v[kLists], total[kLists];
#pragma unroll
  for (int i = 0; i < kLists; ++i) {
    v[i] = mine.n[i];
    for (int off = 1; off < 64; off <<= 1) {
      const long long x = __shfl_up(v[i], off, 64);
      if (lane >= off) v[i] += x;
    }
    if (lane == 63) sh.wave[wave][i] = v[i];
  }
  __syncthreads();
  if (bad) atomicMax(&sh.status, bad);
#pragma unroll
  for (int i = 0; i < kLists; ++i) {
    total[i] = 0;
    v[i] -= mine.n[i];
#pragma unroll
    for (int w = 0; w < kNT / 64; ++w) {
      if (w < wave) v[i] += sh.wave[w][i];
      total[i] += sh.wave[w][i];
    }
  }
  // sums before each of the thread's units (they fit 32 bits if the step is done)
  for (int u = u0; u < u1; ++u) {
    if (unit == 1) {
#pragma unroll
      for (int i = 0; i < kLists; ++i) sh.sum[i][u] += (int)v[i];
      continue;
    }
#pragma unroll
    for (int i = 0; i < kLists; ++i) sh.sum[i][u] = (int)v[i];
    for (int s = u * unit; s < min((u + 1) * unit, a.n_seq); ++s) {
      const Counts c = counts_of(a.n_tokens[s], a.n_new[s], B, shift);
#pragma unroll
      for (int i = 0; i < kLists; ++i) v[i] += c.n[i];
    }
  }
  __syncthreads();
  int status = sh.status;
  if (total[kNeed] > nf + total[kBack]) status = max(status, CKV_SLOTS_NO_BLOCKS);
  if (total[kFresh] > a.max_new) status = max(status, CKV_SLOTS_MAX_NEW);
  if (nf < 0 || nf > a.n_blocks || nf + total[kBack] > a.n_blocks) status = CKV_SLOTS_BAD_COUNT;
  const bool ok = status == CKV_SLOTS_OK;
  const Step st = {a, sh, unit, n_units, nf, (int)(nf + total[kBack]), shift};
  const int g = blockIdx.x * kNT + tid, stride = gridDim.x * kNT;

  // pieces of new tokens, and the new blocks' words in the table
  if (ok) {
    for (int64_t i = g; i < total[kPieces]; i += stride) {
      int c;
      const int s = st.find(kPieces, (int)i, c);
      const int old = unit == 1 ? sh.old[s] : a.n_tokens[s], end = old + a.n_new[s];
      const int col = (int)full_of((unsigned)old, B, shift) + c, have = (int)blocks_of((unsigned)old, B, shift);
      const int first = a.next_pos ? a.next_pos[s] : old;
      const bool taken = col >= have;
      const int b = taken ? st.stacked(st.top - 1 - (st.before(kNeed, s) + col - have)) : st.held(s, col);
      if (taken && a.block_table) a.block_table[s * a.block_stride + col] = b;
      const int t0 = max(old, col * B), n = (int)min((unsigned)end, (unsigned)col * B + B) - t0;
      const int row = (int)min((uint32_t)b, (uint32_t)(a.n_blocks - 1)) * B + (t0 - col * B);
      const int at = st.before(kFresh, s) + t0 - old, p = first + t0 - old;
      store_run(a.slot + s * a.slot_stride + t0, row, n);
      store_run(a.new_row + at, row, n);
      if (a.pos) store_run(a.pos + s * a.slot_stride + t0, p, n);
      if (a.new_pos) store_run(a.new_pos + at, p, n);
    }
    // returned blocks that stay on the stack
    for (int64_t i = (int64_t)nf + g; i < st.top - total[kNeed]; i += stride) a.free_blocks[i] = st.stacked((int)i);
  }
  for (int s = g; s < a.n_seq; s += stride) {
    const int old = unit == 1 ? sh.old[s] : a.n_tokens[s], nn = a.n_new[s];
    a.n_tokens_out[s] = !ok ? old : nn < 0 ? 0 : old + nn;
    a.cu_new[s] = ok ? st.before(kFresh, s) : 0;
  }
  if (g == 0) {
    *a.status = status;
    *a.n_free_out = ok ? (int)(st.top - total[kNeed]) : nf;
    a.cu_new[a.n_seq] = ok ? (int)total[kFresh] : 0;
  }
}

}  // namespace

hipError_t launch_slots(const SlotArgs& a, hipStream_t s) {
  // a thread per piece of the largest step that the lists have room for, as far
  // as the device holds the workgroups at once
  const int64_t want = (int64_t)a.max_new / a.block_size + a.n_seq;
  const int grid = (int)std::min<int64_t>(std::max<int64_t>((want + kNT - 1) / kNT, 1), 768);
  slots_kernel<<<dim3((unsigned)grid), kNT, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ckv
