// Host-side exercise of the serving calls (ckv_build_slots, ckv_attend_window,
// ckv_attend_shared) for sanitizer builds, beside abi_driver.cpp: steps of a
// small server with workspace growth, a workspace limit, a captured step and
// the argument-error paths.  Results are compared by the parity tests; here
// return codes and the sanitizers count, and that every output is finite.
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

// bf16 bits of small multiples of 1/8
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

  const int N = 3, Hkv = 2, Hq = 8, D = 64, B = 16, blocks = 600, pool = B * blocks, most = 4096, rows = 400;
  const std::vector<uint16_t> kv = values((size_t)Hkv * pool * D, 7);
  uint16_t *k = dev(kv), *v = dev(kv), *q = dev(values((size_t)rows * Hq * D, 9)), *o = dev(std::vector<uint16_t>((size_t)rows * Hq * D));
  float* lse = dev(std::vector<float>((size_t)rows * Hq));

  // tables
  std::vector<int32_t> stack(blocks);
  for (int i = 0; i < blocks; ++i) stack[i] = (i * 7) % blocks;
  ckv_slot_step st{};
  st.n_seq = N;
  st.block_size = B;
  st.n_blocks = blocks;
  st.max_new = 8192;
  int32_t* len = dev(std::vector<int32_t>(N));
  int32_t* n_new = dev(std::vector<int32_t>{130, 3000, 1});
  int32_t* n_free = dev(std::vector<int32_t>{blocks});
  st.n_tokens = len;
  st.n_new = n_new;
  st.n_free = n_free;
  st.free_blocks = dev(stack);
  st.block_stride = st.block_cols = most / B;
  st.block_table = dev(std::vector<int32_t>(N * most / B));
  st.slot_stride = st.slot_cols = most;
  st.slot = dev(std::vector<int32_t>(N * most));
  st.pos = dev(std::vector<int32_t>(N * most));
  st.n_tokens_out = dev(std::vector<int32_t>(N));
  st.n_free_out = dev(std::vector<int32_t>(1));
  st.cu_new = dev(std::vector<int32_t>(N + 1));
  st.new_row = dev(std::vector<int32_t>(8192));
  st.new_pos = dev(std::vector<int32_t>(8192));
  st.status = dev(std::vector<int32_t>(1));
  expect(ckv_build_slots(c, &st), CKV_OK, "build_slots", c);
  expect(ckv_sync(c), CKV_OK, "sync", c);
  int32_t status = -1;
  expect(hipMemcpy(&status, st.status, 4, hipMemcpyDeviceToHost), "status");
  expect(status, CKV_SLOTS_OK, "slot status", nullptr);

  ckv_batch_view b{};
  b.k = k;
  b.v = v;
  b.head_stride = (int64_t)pool * D;
  b.tok_stride = D;
  b.slot = st.slot;
  b.slot_stride = most;
  b.pos = st.pos;
  b.pos_stride = most;
  b.n_tokens = st.n_tokens_out;
  b.n_seq = N;
  b.max_tokens = most;
  b.pool_rows = pool;
  b.n_kv_heads = Hkv;
  b.head_dim = D;
  b.dtype = CKV_BF16;
  ckv_query_view w{};
  w.q = q;
  w.row_stride = Hq * D;
  w.head_stride = D;
  w.n_q_heads = Hq;
  int32_t *one = dev(std::vector<int32_t>{0, 1, 2, 3}), *many = dev(std::vector<int32_t>{0, 130, 399, 400});
  ckv_batch_view pre = b;
  pre.n_seq = 1;
  pre.pos = nullptr;
  pre.slot = nullptr;
  pre.n_tokens = dev(std::vector<int32_t>{2500});
  pre.max_tokens = 2500;
  b.pos = nullptr;
  auto finite = [&](int n, const char* what) {
    std::vector<float> h((size_t)n * Hq);
    expect(hipMemcpy(h.data(), lse, h.size() * 4, hipMemcpyDeviceToHost), "lse");
    for (float x : h)
      if (!std::isfinite(x)) {
        std::fprintf(stderr, "[driver] %s: lse %f\n", what, x);
        ++g_fail;
        break;
      }
  };
  auto calls = [&](const char* what) {
    for (int few = 1; few >= 0; --few) {
      w.cu_rows = few ? one : many;
      w.n_rows = few ? 3 : 400;
      w.max_rows = few ? 1 : 269;
      expect(ckv_attend_window(c, &b, &w, 0, 0, o, lse), CKV_OK, what, c);
      expect(ckv_attend_window(c, &b, &w, 100, 4, o, lse), CKV_OK, what, c);
      expect(ckv_sync(c), CKV_OK, what, c);
      finite(w.n_rows, what);
      expect(ckv_attend_shared(c, &pre, &b, &w, o, lse), CKV_OK, what, c);
      expect(ckv_attend_shared(c, &pre, &b, &w, o, nullptr), CKV_OK, what, c);
      expect(ckv_sync(c), CKV_OK, what, c);
      finite(w.n_rows, what);
    }
  };
  calls("growing workspace");
  calls("again");
  expect(ckv_set_workspace_limit(c, 1 << 20), CKV_OK, "limit", c);
  calls("kept workspace under a limit");
  {
    ckv_ctx* d = nullptr;
    expect(ckv_create(&d, 0, stream), CKV_OK, "ckv_create", nullptr);
    std::swap(c, d);
    expect(ckv_set_workspace_limit(c, 4096), CKV_OK, "limit", c);
    calls("no workspace");
    expect(ckv_destroy(c), CKV_OK, "ckv_destroy", nullptr);
    expect(ckv_create(&c, 0, stream), CKV_OK, "ckv_create", nullptr);
    // growth inside a capture is refused, and the capture goes on without it
    w.cu_rows = one;
    w.n_rows = 3;
    w.max_rows = 1;
    hipGraph_t g = nullptr;
    expect(hipStreamBeginCapture(stream, hipStreamCaptureModeThreadLocal), "capture");
    expect(ckv_attend_window(c, &b, &w, 0, 0, o, lse), CKV_ERR_NOMEM, "growth in a capture", c);
    expect(ckv_build_slots(c, &st), CKV_OK, "build_slots in a capture", c);
    expect(hipStreamEndCapture(stream, &g), "end of the capture");
    if (g) expect(hipGraphDestroy(g), "hipGraphDestroy");
    expect(ckv_destroy(c), CKV_OK, "ckv_destroy", nullptr);
    std::swap(c, d);
  }
  // a captured step, replayed
  hipGraph_t g = nullptr;
  hipGraphExec_t x = nullptr;
  expect(hipStreamBeginCapture(stream, hipStreamCaptureModeThreadLocal), "capture");
  expect(ckv_attend_window(c, &b, &w, 0, 0, o, lse), CKV_OK, "captured", c);
  expect(ckv_attend_shared(c, &pre, &b, &w, o, lse), CKV_OK, "captured", c);
  expect(hipStreamEndCapture(stream, &g), "end of the capture");
  expect(hipGraphInstantiate(&x, g, nullptr, nullptr, 0), "hipGraphInstantiate");
  for (int i = 0; i < 3 && x; ++i) expect(hipGraphLaunch(x, stream), "hipGraphLaunch");
  expect(ckv_sync(c), CKV_OK, "replays", c);
  finite(3, "replays");
  if (x) expect(hipGraphExecDestroy(x), "hipGraphExecDestroy");
  if (g) expect(hipGraphDestroy(g), "hipGraphDestroy");

  // refusals
  expect(ckv_attend_window(nullptr, &b, &w, 0, 0, o, lse), CKV_ERR_ARG, "no context", nullptr);
  expect(ckv_attend_window(c, nullptr, &w, 0, 0, o, lse), CKV_ERR_ARG, "no caches", c);
  expect(ckv_attend_window(c, &b, nullptr, 0, 0, o, lse), CKV_ERR_ARG, "no queries", c);
  expect(ckv_attend_window(c, &b, &w, -1, 0, o, lse), CKV_ERR_ARG, "window", c);
  expect(ckv_attend_window(c, &b, &w, 0, 0, nullptr, lse), CKV_ERR_ARG, "no output", c);
  expect(ckv_attend_shared(c, &b, &b, &w, o, lse), CKV_ERR_SHAPE, "prefix of several sequences", c);
  {
    ckv_batch_view bad = b;
    bad.head_dim = 80;
    expect(ckv_attend_window(c, &bad, &w, 0, 0, o, lse), CKV_ERR_SHAPE, "head_dim", c);
    ckv_slot_step s = st;
    s.block_size = 0;
    expect(ckv_build_slots(c, &s), CKV_ERR_ARG, "block_size", c);
    s = st;
    s.n_tokens_out = len;
    expect(ckv_build_slots(c, &s), CKV_ERR_ARG, "output over an input", c);
    expect(ckv_build_slots(c, nullptr), CKV_ERR_ARG, "no step", c);
  }

  expect(ckv_sync(c), CKV_OK, "final sync", c);
  expect(ckv_destroy(c), CKV_OK, "ckv_destroy", nullptr);
  for (void* p : g_held) (void)hipFree(p);
  (void)hipStreamDestroy(stream);
  std::printf("[driver] %s (%d failed checks)\n", g_fail ? "FAILED" : "ok", g_fail);
  return g_fail ? 1 : 0;
}
