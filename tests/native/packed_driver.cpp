// Host-side exercise of the 4-bit calls (ckv_pack_tokens, ckv_unpack_tokens,
// ckv_attend_packed) for sanitizer builds, beside serving_driver.cpp: tokens
// packed, read back and attended to in both kernels, workspace growth and limit,
// a captured step and the argument-error paths.  Results are compared by the
// parity tests; here return codes and the sanitizers count, and that what is read
// back lies within half a step of what was packed.
//
// Exit status 0 when every call returned what it should.
#include "commitkv.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

namespace {

int g_fail = 0;

void expect(int rc, int want, const char* what, ckv_ctx* c) {
  if (rc != want) {
    std::fprintf(stderr, "[driver] %s: returned %d, expected %d (%s)\n", what, rc, want, c ? ckv_last_error(c) : "");
    ++g_fail;
  }
}

void expect(hipError_t rc, const char* what) {
  if (rc != hipSuccess) {
    std::fprintf(stderr, "[driver] %s: %s\n", what, hipGetErrorString(rc));
    ++g_fail;
  }
}

std::vector<void*> g_held;

template <class T>
T* dev(const std::vector<T>& h) {
  void* d = nullptr;
  expect(hipMalloc(&d, std::max<size_t>(h.size(), 1) * sizeof(T)), "hipMalloc");
  if (!h.empty()) expect(hipMemcpy(d, h.data(), h.size() * sizeof(T), hipMemcpyHostToDevice), "hipMemcpy");
  g_held.push_back(d);
  return static_cast<T*>(d);
}

float number(uint16_t bits) {
  const uint32_t b = (uint32_t)bits << 16;
  float f;
  __builtin_memcpy(&f, &b, 4);
  return f;
}

// bf16 bits of multiples of 1/8 from -1 to 7/8
std::vector<uint16_t> values(size_t n, uint32_t seed) {
  std::vector<uint16_t> out(n);
  for (auto& x : out) {
    seed = seed * 1664525u + 1013904223u;
    const float f = ((int)(seed >> 28) - 8) / 8.f;
    uint32_t b;
    __builtin_memcpy(&b, &f, 4);
    x = (uint16_t)(b >> 16);
  }
  return out;
}

}  // namespace

int main() {
  hipStream_t stream = nullptr;
  expect(hipStreamCreate(&stream), "hipStreamCreate");
  ckv_ctx* c = nullptr;
  expect(ckv_create(&c, 0, stream), CKV_OK, "ckv_create", nullptr);
  if (!c) return 1;

  const int N = 2, H = 2, Hq = 8, D = 128, most = 3000, n = N * most, pool_rows = n + 7, rows = 200;
  const std::vector<uint16_t> kv = values((size_t)n * H * D, 3);
  ckv_kv_rows in{};
  in.k = dev(kv);
  in.v = dev(kv);
  in.tok_stride = H * D;
  in.head_stride = D;
  in.dtype = CKV_BF16;
  std::vector<int32_t> row(n), slot(n);
  for (int t = 0; t < n; ++t) slot[t] = row[t] = (int)((int64_t)t * 101 % n);
  const int32_t *d_row = dev(row), *d_slot = dev(slot), *live = dev(std::vector<int32_t>{n}), *lens = dev(std::vector<int32_t>{most, 17});
  ckv_packed_pool pool{};
  pool.data = dev(std::vector<uint8_t>((size_t)H * pool_rows * CKV_PACKED_ROW_BYTES(D)));
  pool.row_stride = CKV_PACKED_ROW_BYTES(D);
  pool.head_stride = (int64_t)pool_rows * pool.row_stride;
  pool.pool_rows = pool_rows;
  pool.n_kv_heads = H;
  pool.head_dim = D;
  expect(ckv_pack_tokens(c, &in, d_row, n, live, &pool), CKV_OK, "pack", c);
  expect(ckv_pack_tokens(c, &in, d_row, 5, nullptr, &pool), CKV_OK, "pack a few", c);
  expect(ckv_pack_tokens(c, &in, d_row, 0, nullptr, &pool), CKV_OK, "pack none", c);

  ckv_packed_view view{};
  view.data = pool.data;
  view.head_stride = pool.head_stride;
  view.row_stride = pool.row_stride;
  view.slot = d_slot;
  view.slot_stride = most;
  view.n_tokens = lens;
  view.n_seq = N;
  view.max_tokens = most;
  view.pool_rows = pool_rows;
  view.n_kv_heads = H;
  view.head_dim = D;
  ckv_kv_rows out{};
  const size_t wide = (size_t)N * H * most * D;
  out.k = dev(std::vector<uint16_t>(wide));
  out.v = dev(std::vector<uint16_t>(wide));
  out.seq_stride = (int64_t)H * most * D;
  out.head_stride = (int64_t)most * D;
  out.tok_stride = D;
  out.dtype = CKV_BF16;
  expect(ckv_unpack_tokens(c, &view, &out), CKV_OK, "unpack", c);
  expect(ckv_sync(c), CKV_OK, "sync", c);
  std::vector<uint16_t> back(wide);
  expect(hipMemcpy(back.data(), out.k, wide * 2, hipMemcpyDeviceToHost), "copy");
  // (steps of 1/8: a half is 1/16, and 2^-7 of rounding to spare)
  for (int g = 0; g < H; ++g)
    for (int t = 0; t < most; t += 97)
      for (int e = 0; e < D; ++e)
        if (std::fabs(number(back[((size_t)g * most + t) * D + e]) - number(kv[((size_t)t * H + g) * D + e])) > 0.0625f + 0.0078125f) {
          std::fprintf(stderr, "[driver] token %d, head %d, width %d is off\n", t, g, e);
          return 1;
        }

  ckv_query_view q{};
  q.q = dev(values((size_t)rows * Hq * D, 9));
  q.row_stride = Hq * D;
  q.head_stride = D;
  q.n_q_heads = Hq;
  uint16_t* o = dev(std::vector<uint16_t>((size_t)rows * Hq * D));
  float* lse = dev(std::vector<float>((size_t)rows * Hq));
  const int32_t *one = dev(std::vector<int32_t>{0, 1, 2}), *many = dev(std::vector<int32_t>{0, 190, rows});
  for (int pass = 0; pass < 2; ++pass) {
    q.cu_rows = pass ? many : one;
    q.n_rows = pass ? rows : 2;
    q.max_rows = pass ? 190 : 1;
    expect(ckv_attend_packed(c, &view, &q, CKV_BF16, 0, 0, o, lse), CKV_OK, "attend", c);
    expect(ckv_attend_packed(c, &view, &q, CKV_BF16, 500, 4, o, nullptr), CKV_OK, "attend, window", c);
    expect(ckv_sync(c), CKV_OK, "sync", c);
    // captured, and replayed behind larger eager work
    hipGraph_t graph = nullptr;
    hipGraphExec_t exec = nullptr;
    expect(hipStreamBeginCapture(stream, hipStreamCaptureModeThreadLocal), "capture");
    expect(ckv_pack_tokens(c, &in, d_row, n, live, &pool), CKV_OK, "captured pack", c);
    expect(ckv_attend_packed(c, &view, &q, CKV_BF16, 0, 0, o, lse), CKV_OK, "captured attend", c);
    expect(hipStreamEndCapture(stream, &graph), "end of capture");
    expect(hipGraphInstantiate(&exec, graph, nullptr, nullptr, 0), "instantiate");
    for (int i = 0; i < 3; ++i) {
      expect(hipGraphLaunch(exec, stream), "launch");
      expect(ckv_sync(c), CKV_OK, "sync", c);
    }
    expect(hipGraphExecDestroy(exec), "destroy");
    expect(hipGraphDestroy(graph), "destroy");
  }
  expect(ckv_set_workspace_limit(c, 1), CKV_OK, "limit", c);
  expect(ckv_attend_packed(c, &view, &q, CKV_BF16, 0, 0, o, lse), CKV_OK, "attend under a limit", c);
  expect(ckv_set_workspace_limit(c, 0), CKV_OK, "limit", c);

  // refusals
  expect(ckv_pack_tokens(nullptr, &in, d_row, n, nullptr, &pool), CKV_ERR_ARG, "pack, no context", nullptr);
  expect(ckv_pack_tokens(c, nullptr, d_row, n, nullptr, &pool), CKV_ERR_ARG, "pack, no tokens", c);
  expect(ckv_pack_tokens(c, &in, nullptr, n, nullptr, &pool), CKV_ERR_ARG, "pack, no rows", c);
  expect(ckv_pack_tokens(c, &in, d_row, n, nullptr, nullptr), CKV_ERR_ARG, "pack, no pool", c);
  expect(ckv_pack_tokens(c, &in, d_row, -1, nullptr, &pool), CKV_ERR_SHAPE, "pack, negative count", c);
  expect(ckv_pack_tokens(c, &in, d_row, INT32_MAX, nullptr, &pool), CKV_ERR_SHAPE, "pack, a count too large", c);
  ckv_packed_pool p2 = pool;
  p2.head_dim = 96;
  expect(ckv_pack_tokens(c, &in, d_row, n, nullptr, &p2), CKV_ERR_SHAPE, "pack, width", c);
  p2 = pool;
  p2.row_stride = 152;
  expect(ckv_pack_tokens(c, &in, d_row, n, nullptr, &p2), CKV_ERR_ARG, "pack, stride", c);
  ckv_kv_rows bad = in;
  bad.dtype = 9;
  expect(ckv_pack_tokens(c, &bad, d_row, n, nullptr, &pool), CKV_ERR_ARG, "pack, type", c);
  expect(ckv_unpack_tokens(c, nullptr, &out), CKV_ERR_ARG, "unpack, no view", c);
  expect(ckv_unpack_tokens(c, &view, nullptr), CKV_ERR_ARG, "unpack, no output", c);
  bad = out;
  bad.v = bad.k;
  expect(ckv_unpack_tokens(c, &view, &bad), CKV_ERR_ARG, "unpack, outputs overlap", c);
  bad = out;
  bad.tok_stride = 64;
  expect(ckv_unpack_tokens(c, &view, &bad), CKV_ERR_SHAPE, "unpack, rows overlap", c);
  ckv_packed_view v2 = view;
  v2.n_tokens = nullptr;
  expect(ckv_attend_packed(c, &v2, &q, CKV_BF16, 0, 0, o, lse), CKV_ERR_ARG, "attend, no lengths", c);
  v2 = view;
  v2.max_tokens = INT32_MAX;
  expect(ckv_attend_packed(c, &v2, &q, CKV_BF16, 0, 0, o, lse), CKV_ERR_SHAPE, "attend, room", c);
  expect(ckv_attend_packed(c, nullptr, &q, CKV_BF16, 0, 0, o, lse), CKV_ERR_ARG, "attend, no view", c);
  expect(ckv_attend_packed(c, &view, nullptr, CKV_BF16, 0, 0, o, lse), CKV_ERR_ARG, "attend, no queries", c);
  expect(ckv_attend_packed(c, &view, &q, 2, 0, 0, o, lse), CKV_ERR_ARG, "attend, type", c);
  expect(ckv_attend_packed(c, &view, &q, CKV_BF16, -1, 0, o, lse), CKV_ERR_ARG, "attend, window", c);

  expect(ckv_sync(c), CKV_OK, "last sync", c);
  expect(ckv_destroy(c), CKV_OK, "ckv_destroy", nullptr);
  for (void* p : g_held) expect(hipFree(p), "hipFree");
  expect(hipStreamDestroy(stream), "hipStreamDestroy");
  if (g_fail) return 1;
  std::printf("[driver] ok\n");
  return 0;
}
