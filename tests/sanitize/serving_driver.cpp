// Drives the argument checks of the cache, attention and logits entry points (include/c2t.h) with the library's host code built under
// -fsanitize=address,undefined (tests/test_serving_host.py; CPU only: every call is refused before anything is enqueued, or fails cleanly at
// the launch): sizes and strides at and past their limits, where a product could leave its type.
#include "../../include/c2t.h"

#include <cstdio>
#include <cstring>

#define EXPECT(cond) do { if (!(cond)) { std::printf("serving driver: %s failed at line %d\n", #cond, __LINE__); return 1; } } while (0)

static c2t_cache base() {
  c2t_cache c;
  std::memset(&c, 0, sizeof c);
  c.batch = 2; c.layers = 3; c.pages = 40; c.page_size = 16; c.kv_heads = 2; c.head_dim = 64; c.max_pages = 8; c.dtype = C2T_BF16;
  void* p = (void*)(uintptr_t)0x10000000;                    // never dereferenced on the host
  c.k = c.v = p; c.page_table = c.length = c.refcount = (int32_t*)p; c.status = (uint32_t*)p;
  return c;
}

static bool refused_or_launched(int rc) { return rc == C2T_OK || rc == C2T_ERR_HIP || rc == C2T_ERR_INVALID_ARG || rc == C2T_ERR_UNSUPPORTED || rc == C2T_ERR_WORKSPACE; }

int main() {
  void* const p = (void*)(uintptr_t)0x10000000;
  int32_t* const ip = (int32_t*)p;
  const int32_t odd[] = {INT32_MIN, -1, 0, 1, 2, 16, 64, 256, 1024, 1025, 4096, 65536, 1 << 24, 1 << 30, INT32_MAX};
  const int64_t odd64[] = {INT64_MIN, -8, 0, 8, 64, 128, 256, (int64_t)1 << 40, ((int64_t)1 << 40) + 8, INT64_MAX - 7};
  size_t need = 0;
  for (int32_t x : odd) {
    for (int field = 0; field < 8; ++field) {
      c2t_cache c = base();
      int32_t* f[] = {&c.batch, &c.layers, &c.pages, &c.page_size, &c.kv_heads, &c.head_dim, &c.max_pages, &c.dtype};
      *f[field] = x;
      const int rc = c2t_cache_workspace_bytes(&c, &need);
      EXPECT(refused_or_launched(rc) && rc != C2T_ERR_HIP);
      for (int32_t tokens : odd) for (int32_t heads : {-1, 0, 2, 6, 2048, INT32_MAX}) {
        c2t_attention a;
        std::memset(&a, 0, sizeof a);
        a.tokens = tokens; a.q_heads = heads; a.nodes = tokens > 4 ? 3 : 0;
        EXPECT(refused_or_launched(c2t_attention_workspace_bytes(&c, &a, &need)));
      }
    }
  }
  c2t_cache c = base();
  for (int64_t s : odd64) for (int64_t t : odd64) {
    c2t_attention a;
    std::memset(&a, 0, sizeof a);
    a.q = a.out = p; a.tokens = 4; a.q_heads = 4; a.scale = 1.f;
    a.q_batch_stride = s; a.q_token_stride = t; a.out_batch_stride = t; a.out_token_stride = s;
    EXPECT(c2t_cache_attention(&c, &a, nullptr, 0, nullptr) != C2T_OK);
    if (s < 0 || t < 0 || t > ((int64_t)1 << 40)) EXPECT(c2t_cache_write(&c, 0, p, p, s, t, 4, nullptr, nullptr) < 0);
    c2t_adjustments j;
    std::memset(&j, 0, sizeof j);
    j.tokens = ip; j.n_tokens = ip; j.token_stride = s; j.allowed = (uint32_t*)p; j.allowed_row_stride = t; j.allowed_batch_stride = s;
    EXPECT(refused_or_launched(c2t_adjust_tree_logits(&j, 0, 100, 3, C2T_F32, ip, ip, ip, p, s, p, t, nullptr)));
    std::memset(&j, 0, sizeof j);
    if (s < 100 || s > ((int64_t)1 << 40) || s != t) EXPECT(c2t_adjust_tree_logits(&j, 1, 100, 3, C2T_F32, ip, ip, ip, p, s, p, t, nullptr) < 0);
  }
  for (int32_t x : odd) {
    c2t_adjustments j;
    std::memset(&j, 0, sizeof j);
    if (x <= 0 || x > C2T_MAX_BIAS) { j.bias = (float*)p; j.bias_tokens = ip; j.bias_stride = x; EXPECT(c2t_adjust_tree_logits(&j, 1, 100, 3, C2T_F32, ip, ip, ip, p, 128, p, 128, nullptr) < 0); }
    std::memset(&j, 0, sizeof j);
    if (x <= 0 || x > 65535) EXPECT(c2t_adjust_tree_logits(&j, x, 100, 3, C2T_F32, ip, ip, ip, p, 128, p, 128, nullptr) < 0);
    if (x < 0 || x > C2T_MAX_BUDGET) EXPECT(c2t_adjust_tree_logits(&j, 1, 100, x, C2T_F32, ip, ip, ip, p, 128, p, 128, nullptr) < 0);
    if (x <= 0 || x > C2T_MAX_PATH) EXPECT(c2t_cache_commit(&c, ip, x, ip, nullptr) < 0);
    if (x <= 0 || x > C2T_MAX_CACHE_BATCH) EXPECT(c2t_cache_fork(&c, ip, ip, x, nullptr) < 0);
    if (x < 0) EXPECT(c2t_cache_truncate(&c, nullptr, x, nullptr) < 0);
  }
  uint64_t id = 7;
  EXPECT(c2t_stream_capture_id(nullptr, nullptr) == C2T_ERR_INVALID_ARG && c2t_stream_capture_id(nullptr, &id) == C2T_OK && id == 0);
  std::printf("serving driver ok\n");
  return 0;
}
