// Block tables and slot tables of a batch from its lengths (ckv_build_slots).
//
// With B rows a block, sequence s holds blocks(n) = ceil(n / B) blocks for n
// tokens.  It gives back(s) = blocks(old) of them when it ends, or takes
// need(s) = blocks(old + new) - blocks(old) for fresh(s) = new tokens.  The
// free stack after the returns is F = free[0 .. n_free) followed by the
// returned blocks in the order of sequences; the k-th new block of the batch
// is F[top - 1 - k].  So every word of the result follows from the prefix
// sums of need, back and fresh over the sequences, and from words that the
// step does not change: blocks that are taken have an index in F of at least
// the new top, blocks that are stored below it, and entries of F past n_free
// are read from the ended sequences' own tables, which stay.  One launch does
// it all, without any order between its workgroups: each forms the prefix
// sums for itself (a few thousand lengths, from L2) and takes a share of the
// tokens, blocks and sequences.
//
// Bound: latency.  A step reads two counts a sequence, moves two words a
// block and writes four words a token.
#include "ckv_device.h"
#include "ckv_kernels.h"

#include "commitkv.h"

#include <algorithm>
#include <climits>

namespace ckv {

namespace {

constexpr int kNT = 256;
constexpr int kUnits = 4096;   // prefix sums kept in LDS, one for every `unit` sequences

struct Counts {
  long long need, back, fresh;
};

__device__ __forceinline__ long long blocks_of(long long tokens, int b) {
  return (long long)(((unsigned long long)tokens + (unsigned)b - 1) / (unsigned)b);
}

__device__ __forceinline__ Counts counts_of(int old, int nn, int B) {
  Counts c = {0, 0, 0};
  if (old < 0 || nn < -1) return c;
  // 32-bit division: old + new + B stays below 2^32 (lengths below 2^31, B at most 2^31)
  const unsigned b = (unsigned)B, have = old ? ((unsigned)old - 1) / b + 1 : 0u;
  if (nn < 0) {
    c.back = have;
  } else {
    const unsigned now = (unsigned)old + (unsigned)nn;
    c.need = (now ? (now - 1) / b + 1 : 0u) - have;
    c.fresh = nn;
  }
  return c;
}

struct Shared {
  int need[kUnits + 1], back[kUnits + 1], fresh[kUnits + 1];   // sums before each unit, and the totals
  long long wave[kNT / 64][3];
  int status;
};

// the unit that holds element i of the list whose sums are `pre`: the last u with pre[u] <= i
__device__ __forceinline__ int find_unit(const int* pre, int n_units, int i) {
  int lo = 0, hi = n_units;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (pre[m] <= i) lo = m;
    else hi = m;
  }
  return lo;
}

struct Step {
  const SlotArgs& a;
  const Shared& sh;
  int unit, n_units, nf, top;   // top: entries of F

  // sequence of element i of a list, and i's place inside it
  template <int Counts32>
  __device__ __forceinline__ int find(int i, int& at) const {
    const int* pre = Counts32 == 0 ? sh.need : Counts32 == 1 ? sh.back : sh.fresh;
    const int u = find_unit(pre, n_units, i);
    at = i - pre[u];
    int s = u * unit;
    if (unit > 1) {
      for (; s < a.n_seq - 1; ++s) {
        const Counts c = counts_of(a.n_tokens[s], a.n_new[s], a.block_size);
        const int n = (int)(Counts32 == 0 ? c.need : Counts32 == 1 ? c.back : c.fresh);
        if (at < n) break;
        at -= n;
      }
    }
    return s;
  }

  // sum of need before sequence s (its unit's, plus the sequences between)
  __device__ __forceinline__ int need_before(int s) const {
    const int u = s / unit;
    int n = sh.need[u];
    for (int t = u * unit; t < s; ++t) n += (int)counts_of(a.n_tokens[t], a.n_new[t], a.block_size).need;
    return n;
  }

  __device__ __forceinline__ int held(int s, int64_t i) const {
    return a.block_table ? a.block_table[s * a.block_stride + i] : a.slot[s * a.slot_stride + i];
  }

  // F[i]
  __device__ __forceinline__ int stacked(int i) const {
    if (i < nf) return a.free_blocks[i];
    int at;
    const int s = find<1>(i - nf, at);
    return held(s, at);
  }
};

__global__ __launch_bounds__(kNT) void slots_kernel(SlotArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = a.block_size;
  const int unit = (a.n_seq + kUnits - 1) / kUnits > 1 ? (a.n_seq + kUnits - 1) / kUnits : 1;
  const int n_units = a.n_seq > 0 ? (a.n_seq + unit - 1) / unit : 0;
  const int per = (n_units + kNT - 1) / kNT;           // units of a thread
  const int u0 = min(tid * per, n_units), u1 = min(u0 + per, n_units);
  const int64_t cols = a.block_table ? a.block_stride : a.slot_stride;
  if (tid == 0) sh.status = CKV_SLOTS_OK;
  const int nf = *a.n_free;

  Counts mine = {0, 0, 0};
  int bad = CKV_SLOTS_OK;
  for (int s = u0 * unit; s < min(u1 * unit, a.n_seq); ++s) {
    const int old = a.n_tokens[s], nn = a.n_new[s];
    if (old < 0 || nn < -1) {
      bad = CKV_SLOTS_BAD_COUNT;
      continue;
    }
    const long long now = (long long)old + max(nn, 0);
    if (now > a.slot_stride || blocks_of(now, B) > cols) bad = max(bad, CKV_SLOTS_TABLE);
    const Counts c = counts_of(old, nn, B);
    mine.need += c.need;
    mine.back += c.back;
    mine.fresh += c.fresh;
  }
  long long v[3] = {mine.need, mine.back, mine.fresh};
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    for (int off = 1; off < 64; off <<= 1) {
      const long long x = __shfl_up(v[i], off, 64);
      if (lane >= off) v[i] += x;
    }
    if (lane == 63) sh.wave[wave][i] = v[i];
  }
  __syncthreads();
  if (bad) atomicMax(&sh.status, bad);
  long long total[3] = {0, 0, 0};
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int w = 0; w < kNT / 64; ++w) {
      if (w < wave) v[i] += sh.wave[w][i];
      total[i] += sh.wave[w][i];
    }
  // sums before each of the thread's units (they fit 32 bits if the step is done)
  {
    long long x[3] = {v[0] - mine.need, v[1] - mine.back, v[2] - mine.fresh};
    for (int u = u0; u < u1; ++u) {
      sh.need[u] = (int)x[0];
      sh.back[u] = (int)x[1];
      sh.fresh[u] = (int)x[2];
      for (int s = u * unit; s < min((u + 1) * unit, a.n_seq); ++s) {
        const Counts c = counts_of(a.n_tokens[s], a.n_new[s], B);
        x[0] += c.need;
        x[1] += c.back;
        x[2] += c.fresh;
      }
    }
  }
  __syncthreads();
  int status = sh.status;
  if (total[0] > nf + total[1]) status = max(status, CKV_SLOTS_NO_BLOCKS);
  if (total[2] > a.max_new) status = max(status, CKV_SLOTS_MAX_NEW);
  if (nf < 0 || nf > a.n_blocks || nf + total[1] > a.n_blocks) status = CKV_SLOTS_BAD_COUNT;
  const bool ok = status == CKV_SLOTS_OK;
  const int g = blockIdx.x * kNT + tid, stride = gridDim.x * kNT;
  if (g == 0) {
    *a.status = status;
    *a.n_free_out = ok ? (int)(nf + total[1] - total[0]) : nf;
    a.cu_new[a.n_seq] = ok ? (int)total[2] : 0;
  }
  const Step st = {a, sh, unit, n_units, nf, (int)(nf + total[1])};
  for (int s = g; s < a.n_seq; s += stride) {
    const int old = a.n_tokens[s], nn = a.n_new[s];
    a.n_tokens_out[s] = !ok ? old : nn < 0 ? 0 : old + nn;
    int before = 0;
    if (ok) {
      const int u = s / unit;
      before = sh.fresh[u];
      for (int t = u * unit; t < s; ++t) before += max(a.n_new[t], 0);
    }
    a.cu_new[s] = before;
  }
  if (!ok) return;
  // returned blocks that stay on the stack
  for (int i = nf + g; i < st.top - (int)total[0]; i += stride) a.free_blocks[i] = st.stacked(i);
  // new blocks (their words in the table; with B = 1 and no table the tokens below write them)
  if (a.block_table) {
    for (int k = g; k < (int)total[0]; k += stride) {
      int at;
      const int s = st.find<0>(k, at);
      a.block_table[s * a.block_stride + blocks_of(a.n_tokens[s], B) + at] = st.stacked(st.top - 1 - k);
    }
  }
  // new tokens
  for (int i = g; i < (int)total[2]; i += stride) {
    int j;
    const int s = st.find<2>(i, j);
    const int old = a.n_tokens[s], t = old + j;
    const int col = (int)((unsigned)t / (unsigned)B), have = (int)blocks_of(old, B);
    const int b = col < have ? st.held(s, col) : st.stacked(st.top - 1 - (st.need_before(s) + col - have));
    const int row = (int)min((uint32_t)b, (uint32_t)(a.n_blocks - 1)) * B + (t - col * B);
    const int64_t at = s * a.slot_stride + t;
    a.slot[at] = row;
    a.new_row[i] = row;
    if (a.pos || a.new_pos) {
      const int p = (a.next_pos ? a.next_pos[s] : old) + j;
      if (a.pos) a.pos[at] = p;
      if (a.new_pos) a.new_pos[i] = p;
    }
  }
}

}  // namespace

hipError_t launch_slots(const SlotArgs& a, hipStream_t s) {
  // a thread takes up to 8 tokens of the largest step the lists have room for
  const int64_t want = std::max<int64_t>((int64_t)a.max_new / 8, a.n_seq);
  const int grid = (int)std::min<int64_t>(std::max<int64_t>((want + kNT - 1) / kNT, 1), 512);
  slots_kernel<<<dim3((unsigned)grid), kNT, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ckv
