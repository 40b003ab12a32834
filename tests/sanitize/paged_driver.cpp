// Checks on the host, over many sizes, what the attention kernels' addresses and work lists are made of
// (paper_2502_13652_amd/csrc/k_paged.h): every key tile of every row tile belongs to one part, records of parts do not overlap and stay in
// the workspace, the launch has an item for every part, and whatever lengths, counts and page numbers the device's arrays hold
// become tokens and pages that exist.
#include "../../paper_2502_13652_amd/csrc/k_paged.h"

#include <cstdio>
#include <random>
#include <set>
#include <vector>

using namespace c2t;

#define EXPECT(cond) do { if (!(cond)) { std::printf("paged driver: %s failed at line %d\n", #cond, __LINE__); return 1; } } while (0)

static CacheView cache(int batch, int pages, int max_pages, int shift, int heads, int dim) {
  CacheView c{};
  c.batch = batch; c.layers = 3; c.pages = pages; c.max_pages = max_pages; c.page_shift = shift; c.kv_heads = heads; c.head_dim = dim;
  return c;
}

int main() {
  std::mt19937 rng(7);
  auto pick = [&](int lo, int hi) { return (int)(lo + rng() % ((uint32_t)hi - (uint32_t)lo + 1u)); };
  const int odd[] = {-2147483647 - 1, -1, 0, 1, 15, 16, 17, 1 << 20, 1 << 30, 2147483647};
  for (int shift = 4; shift <= 8; ++shift) {
    const CacheView c = cache(2, 1000, 64, shift, 8, 128);
    for (int x : odd) {
      const int len = tokens_in_cache(c, x);
      EXPECT(len >= 0 && len <= capacity_of(c));
      for (int y : odd) for (int slots : {1, 7, 5000, 1 << 30}) {
        const int n = new_tokens(c, len, y, slots);
        EXPECT(n >= 0 && n <= slots && len + n <= capacity_of(c));
        EXPECT(n == 0 || ((len + n - 1) >> shift) < c.max_pages);
      }
      const int p = valid_page(c, x);
      EXPECT(p == -1 || (p >= 0 && p < c.pages && p == x));
    }
  }
  // quotients from reciprocals, also ones as imprecise as the device's instruction gives them
  for (int i = 0; i < 2000000; ++i) {
    const int d = i < 1000 ? i + 1 : pick(1, 1 << pick(0, 30)), top = (1 << 30) + (1 << 20);
    const int n = i % 7 == 0 ? (int)std::min<int64_t>((int64_t)d * pick(0, 1 << pick(0, 30)), top) - (i % 3 == 0) : pick(0, top);
    if (n < 0) continue;
    for (float off : {1.f, 1.f + 1.5e-7f, 1.f - 1.5e-7f}) {
      int q, r;
      split(n, d, off / (float)d, &q, &r);
      EXPECT(q == n / d && r == n % d);
    }
  }
  {   // the largest pool there may be: offsets in 64 bits
    const CacheView c = cache(1, (1 << 27) - 1, 1 << 22, 4, 1024, 256);
    const int64_t last = row_offset(c, 2, c.pages - 1, c.kv_heads - 1, 15) + c.head_dim;
    EXPECT(last == (int64_t)3 * c.pages * c.kv_heads * 16 * 256);
  }
  for (int round = 0; round < 3000; ++round) {
    const int batch = pick(1, round % 10 == 0 ? 200 : 9), shift = pick(4, 8), heads = pick(1, 4);
    const int max_pages = pick(1, 1 << pick(0, 10 - shift + 4));
    const CacheView c = cache(batch, 1 << 20, max_pages, shift, heads, 64);
    AttendShape a;
    a.slots = pick(1, 1 << pick(0, 9)); a.group = pick(1, 9);
    a.rows_shift = pick(4, 8); a.keys_shift = pick(5, 6);
    a.target_shift = pick(0, 8); a.min_per = pick(1, 16); a.max_parts = round % 3 ? 1024 : pick(2, 40); a.inv_group = 1.f / (float)a.group;
    const int64_t target = (int64_t)1 << a.target_shift;
    const int chain = pick(0, a.slots);
    std::vector<int> len(batch), n(batch);
    float all = 0.f;
    for (int b = 0; b < batch; ++b) {
      len[b] = tokens_in_cache(c, pick(-1, capacity_of(c) + 1));
      n[b] = new_tokens(c, len[b], pick(-1, a.slots + 1), a.slots);
      all += sequence_tiles(c, a, len[b], n[b]);
    }
    const int per = tiles_per_part(a, all);
    EXPECT(per >= a.min_per);
    const float inv_per = 1.f / (float)per;
    const int64_t units_max = (int64_t)batch * heads * div_up64((int64_t)a.slots * a.group, 1 << a.rows_shift);
    int64_t items = 0, records = 0, units = 0;
    for (int b = 0; b < batch; ++b) {
      const int parts = n[b] ? parts_of(a, per, inv_per, len[b], n[b]) : 0, tiles = row_tiles(a, n[b]);
      EXPECT(n[b] == 0 || parts == std::min(a.max_parts, std::max(1, div_up(key_tiles(a, len[b] + n[b]), per))));
      items += (int64_t)parts * tiles * heads;
      units += (int64_t)tiles * heads;
      if (parts > 1) records += (int64_t)parts * tiles * heads;
      for (int rt = 0; rt < tiles; ++rt) {
        const int seen = keys_seen(a, len[b], n[b], chain, rt), kt = key_tiles(a, seen);
        EXPECT(seen >= 1 && seen <= len[b] + n[b]);
        // the last row of the tile sees no key past `seen`
        const int64_t last = std::min<int64_t>((int64_t)(rt + 1) << a.rows_shift, (int64_t)n[b] * a.group) - 1;
        const int t = (int)(last / a.group);
        EXPECT(t < n[b] && seen == (t < chain ? len[b] + t + 1 : len[b] + n[b]));
        int next = 0;
        for (int p = 0; p < parts; ++p) {
          int first, end;
          part_range(kt, parts, p, &first, &end);
          EXPECT(first == next && first <= end && end <= kt && (end - first <= per || parts == a.max_parts));
          next = end;
        }
        EXPECT(next == kt);
      }
    }
    a.run = pick(1, 9);
    const int64_t groups = workgroups_for(a, items);
    EXPECT(groups >= items && groups < items + DIES * a.run + 1);
    if (groups < 20000) {
      std::vector<char> taken(groups, 0);
      for (int w = 0; w < groups; ++w) {
        const int item = item_of_workgroup(a, w);
        EXPECT(item >= 0 && item < groups && !taken[item]);
        taken[item] = 1;
      }
    }
    EXPECT(units <= units_max && items <= units_max + target && records <= 2 * target);
  }
  std::printf("paged driver ok\n");
  return 0;
}
