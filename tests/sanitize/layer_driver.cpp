// Drives the argument checks of the norm, append and prompt entry points (include/c2t.h) with the library's host code built under
// -fsanitize=address,undefined (tests/test_layer_host.py; CPU only: every call is refused before anything is enqueued, or fails cleanly at
// the launch): sizes and strides at and past their limits, where a product could leave its type.
#include "../../include/c2t.h"

#include <cstdio>
#include <cstring>

#define EXPECT(cond) do { if (!(cond)) { std::printf("layer driver: %s failed at line %d\n", #cond, __LINE__); return 1; } } while (0)

static bool known(int rc) { return rc == C2T_OK || rc == C2T_ERR_HIP || rc == C2T_ERR_INVALID_ARG || rc == C2T_ERR_UNSUPPORTED; }

int main() {
  char* const p = (char*)(uintptr_t)0x10000000;              // never dereferenced on the host
  const int32_t odd[] = {INT32_MIN, -1, 0, 1, 3, 8, 16, 32, 64, 128, 1024, 4096, 65536, 1 << 24, 1 << 30, INT32_MAX};
  const int64_t odd64[] = {INT64_MIN, -8, 0, 8, 64, 256, 1 << 24, (int64_t)1 << 40, ((int64_t)1 << 40) + 8, INT64_MAX - 7};
  for (int32_t x : odd) for (int32_t y : odd) for (int64_t s : odd64) for (int64_t t : odd64) {
    c2t_norm n;
    std::memset(&n, 0, sizeof n);
    n.x = p; n.weight = p; n.residual = p + 64; n.residual_out = p + 128; n.out = p + 192; n.scales = (float*)(p + 256);
    n.x_stride = s; n.residual_stride = t; n.residual_out_stride = s; n.out_stride = t; n.scales_stride = s;
    n.rows = x; n.width = y; n.dtype = C2T_BF16; n.weight_dtype = C2T_F32; n.residual_dtype = C2T_F32; n.out_dtype = C2T_E4M3; n.scale_block = y; n.eps = 1e-5f;
    EXPECT(known(c2t_rms_norm(&n, nullptr)));
    if (x < 0 || y <= 0 || s < y || t < y || s > ((int64_t)1 << 40)) EXPECT(c2t_rms_norm(&n, nullptr) < 0);
    n.scale_block = x; n.rows = 5;
    EXPECT(known(c2t_rms_norm(&n, nullptr)));

    c2t_cache c;
    std::memset(&c, 0, sizeof c);
    c.batch = 2; c.layers = 3; c.pages = 40; c.page_size = 16; c.kv_heads = 2; c.head_dim = 64; c.max_pages = 8; c.dtype = C2T_BF16;
    c.k = c.v = p; c.page_table = c.length = c.refcount = (int32_t*)p; c.status = (uint32_t*)p;
    c2t_append a;
    std::memset(&a, 0, sizeof a);
    a.q = p; a.k = p + 64; a.v = p + 128; a.q_out = p + 192; a.k_out = p + 256; a.turns = (uint64_t*)p; a.magnitude = 1.f;
    a.q_batch_stride = s; a.q_token_stride = t; a.kv_batch_stride = t; a.kv_token_stride = s; a.q_out_batch_stride = t; a.q_out_token_stride = s; a.k_out_batch_stride = s;
    a.k_out_token_stride = t; a.tokens = x; a.q_heads = y; a.pairs = 32;
    EXPECT(known(c2t_cache_append(&c, &a, nullptr)));
    if (x < 0 || y <= 0 || s < 0 || t < 0 || s > ((int64_t)1 << 40)) EXPECT(c2t_cache_append(&c, &a, nullptr) < 0);
    a.starts = (int32_t*)p; a.q_heads = 2; a.pairs = y;
    EXPECT(known(c2t_cache_append(&c, &a, nullptr)));
    a.starts = nullptr; a.pairs = 32; a.nodes = y; a.position = (int32_t*)p;
    EXPECT(known(c2t_cache_append(&c, &a, nullptr)));

    c2t_prompt q;
    std::memset(&q, 0, sizeof q);
    q.q = p; q.k = p + 64; q.v = p + 128; q.out = p + 192; q.starts = (int32_t*)p; q.q_stride = s; q.k_stride = t; q.v_stride = s; q.out_stride = t;
    q.rows = x; q.sequences = y; q.q_heads = 4; q.kv_heads = 2; q.head_dim = 64; q.dtype = C2T_BF16; q.scale = 1.f;
    EXPECT(known(c2t_prompt_attention(&q, nullptr)));
    if (x < 0 || y <= 0 || y > C2T_MAX_CACHE_BATCH || s < 256 || t < 256 || s > 1 << 24 || t > 1 << 24) EXPECT(c2t_prompt_attention(&q, nullptr) < 0);
    q.sequences = 3; q.q_heads = y; q.kv_heads = x; q.rows = 1 << 24;
    EXPECT(known(c2t_prompt_attention(&q, nullptr)));
  }
  std::printf("layer driver ok\n");
  return 0;
}
