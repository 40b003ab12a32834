// Checks on the host that a query head's place in its token's row (paper_2502_13652_amd/csrc/k_paged.h) is right for as many heads as a call may
// have: past 31 bits of bytes, and past 31 bits of elements.
#include "../../paper_2502_13652_amd/csrc/k_paged.h"

#include <cstdio>

using namespace c2t;

#define EXPECT(cond) do { if (!(cond)) { std::printf("heads driver: %s failed at line %d\n", #cond, __LINE__); return 1; } } while (0)

int main() {
  for (int dim : {64, 128, 256})
    for (int kv_heads : {1, 8, 1024})
      for (int64_t heads : {(int64_t)kv_heads, (int64_t)kv_heads * 7, (int64_t)1 << 20, (int64_t)1 << 23, (int64_t)1 << 25, (int64_t)1 << 30}) {
        const int group = (int)(heads / kv_heads);
        EXPECT(query_offset(0, group, 0, dim) == 0);
        EXPECT(query_offset(kv_heads - 1, group, group - 1, dim) == ((int64_t)kv_heads * group - 1) * dim);
        for (int head = 0; head < kv_heads; ++head) {
          EXPECT(query_offset(head, group, 0, dim) >= 0 && query_offset(head, group, 0, dim) == (int64_t)dim * group * head);
          EXPECT(query_offset(head, group, group - 1, dim) == query_offset(head, group, 0, dim) + (int64_t)(group - 1) * dim);
        }
      }
  std::printf("heads driver ok\n");
  return 0;
}
