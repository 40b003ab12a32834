// What the paged K/V cache's kernels share: where a token of a sequence lies, and how attention's work is dealt to
// workgroups.  Every index that comes from device memory (lengths, counts, page numbers) passes through here on its way to
// an address.  Plain functions of numbers, for host and device, so that their bounds can be checked on the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace c2t {

#define C2T_HD __host__ __device__ __forceinline__

struct CacheView {
  char* k; char* v;                        // [layers][pages][kv_heads][page_size][head_dim], 2 bytes an element
  int32_t* table;                          // [batch][max_pages]
  int32_t* length;                         // [batch]
  int32_t* refcount;                       // [pages]
  uint32_t* status;                        // [batch]
  int32_t batch, layers, pages, max_pages, kv_heads, head_dim;
  int32_t page_shift;                      // page_size = 1 << page_shift
};

enum : uint32_t { CACHE_POOL_EMPTY = 1u, CACHE_ROW_FULL = 2u, CACHE_INVALID = 4u, CACHE_SHARED = 8u };     // C2T_CACHE_* of the C ABI
__device__ __forceinline__ void report(const CacheView& c, int b, uint32_t bit) { atomicOr(c.status + b, bit); }

C2T_HD int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
C2T_HD int div_up(int a, int b) { return (a + b - 1) / b; }
C2T_HD int64_t div_up64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// n = q d + r, 0 <= r < d, for 0 <= n <= 2^30 + 2^20 and 1 <= d <= 2^30: from the reciprocal, of which `inverse` holds 22 bits or more.  The first quotient is off by at most 2^10 (and
// 1), what is left over gives that within 1.  A fifth of an integer division's instructions, of which a workgroup's start had a dozen.
C2T_HD void split(int n, int d, float inverse, int* q, int* r) {
  int a = (int)((float)n * inverse);
  int b = (int)((uint32_t)n - (uint32_t)a * (uint32_t)d);     // (a d may pass 31 bits where a is one too large)
  const int more = (int)((float)b * inverse);
  a += more; b -= more * d;
  if (b < 0) { b += d; a -= 1; }
  if (b >= d) { b -= d; a += 1; }
  *q = a; *r = b;
}

// tokens that a sequence's row of the page table has room for (at most 2^30: checked by the host)
C2T_HD int capacity_of(const CacheView& c) { return c.max_pages << c.page_shift; }
C2T_HD int tokens_in_cache(const CacheView& c, int length) { return clamp_int(length, 0, capacity_of(c)); }
// new tokens behind `len` cached ones: at most `slots`, and no more than the row has room for
C2T_HD int new_tokens(const CacheView& c, int len, int n_new, int slots) {
  const int room = capacity_of(c) - len;
  return clamp_int(n_new, 0, slots < room ? slots : room);
}
// a page number as the table holds it; -1 if it is none of the pool's
C2T_HD int valid_page(const CacheView& c, int page) { return (uint32_t)page < (uint32_t)c.pages ? page : -1; }

// Offset, in elements, of a token's row of one head: `row` of page `page`.
C2T_HD int64_t row_offset(const CacheView& c, int layer, int page, int head, int row) {
  return ((((int64_t)layer * c.pages + page) * c.kv_heads + head) << c.page_shift) * c.head_dim + (int64_t)row * c.head_dim;
}

// Offset, in elements, of a query head in its token's row (of queries, and of outputs): head `g` of the `group` that share cached head `head`.  Heads may be
// as many as 2^30, so 31 bits do not hold it.
C2T_HD int64_t query_offset(int head, int group, int g, int head_dim) { return ((int64_t)head * group + g) * head_dim; }

// ---- Attention's work ----
// A unit is a tile of query rows of one cached head of one sequence; it goes over the sequence's keys tile by tile.  Units
// are split over their keys into parts so that the launch has about `target` parts of about the same length whatever
// the lengths of the sequences: with `per` = max(min_per, ceil(all tiles / target)), a
// sequence's units have ceil(its tiles / per) parts each, up to max_parts.  Parts of one unit leave records for the join; there are never more than
// 2 target of those: a unit of p >= 2 parts has more than per (p - 1) >= per p / 2 tiles.
struct AttendShape {
  int32_t slots;                           // new tokens a sequence at most
  int32_t group;                           // query heads per cached head
  int32_t rows_shift, keys_shift;          // tiles of 1 << rows_shift query rows and 1 << keys_shift keys
  int32_t target_shift, min_per;           // about 1 << target_shift parts, of min_per key tiles or more
  int32_t max_parts;                       // of a unit, 2 to 1024
  int32_t run;                             // items in a row for one die
  float inv_group;                         // 1 / group
};
// Workgroups go to the chip's eight dies in turn.  Neighbouring items, whose rows share keys, belong on one die and its L2; runs of
// items are dealt to the dies in turn, since items come longest first.
constexpr int DIES = 8;
C2T_HD int item_of_workgroup(const AttendShape& a, int workgroup) {
  const int i = workgroup / DIES;
  return (i / a.run * DIES + workgroup % DIES) * a.run + i % a.run;
}
C2T_HD int64_t workgroups_for(const AttendShape& a, int64_t items) { return div_up64(items, DIES * a.run) * DIES * a.run; }
// (rows: at most 2^30, checked by the host)
C2T_HD int row_tiles(const AttendShape& a, int n_new) { return (n_new * a.group + (1 << a.rows_shift) - 1) >> a.rows_shift; }
C2T_HD int key_tiles(const AttendShape& a, int keys) { return (keys + (1 << a.keys_shift) - 1) >> a.keys_shift; }
// key tiles of all units of a sequence; only their sum's size matters, in which 24 bits are plenty
C2T_HD float sequence_tiles(const CacheView& c, const AttendShape& a, int len, int n_new) {
  return (float)row_tiles(a, n_new) * (float)c.kv_heads * (float)key_tiles(a, len + n_new);
}
// (a thousandth more than the share: the sum's roundings do not make it less)
C2T_HD int tiles_per_part(const AttendShape& a, float all_tiles) {
  const float per = all_tiles * (1.001f / (float)(1 << a.target_shift)) + 1.f;
  return per < (float)a.min_per ? a.min_per : per > 1e9f ? 1000000000 : (int)per;
}
C2T_HD int parts_of(const AttendShape& a, int per, float inv_per, int len, int n_new) {
  const int t = key_tiles(a, len + n_new);
  if (t <= per) return 1;
  if ((int64_t)per * a.max_parts <= t) return a.max_parts;
  int q, r;
  split(t, per, inv_per, &q, &r);
  return q + (r > 0);
}
// keys that some row of a tile of query rows sees, from the first: rows of the sequence's n_new * group, `chain` causal slots ahead of the nodes
C2T_HD int keys_seen(const AttendShape& a, int len, int n_new, int chain, int row_tile) {
  const int last_row = ((row_tile + 1) << a.rows_shift) - 1, rows = n_new * a.group;
  int t, g;
  split(last_row < rows ? last_row : rows - 1, a.group, a.inv_group, &t, &g);
  return t < chain ? len + t + 1 : len + n_new;
}
// key tiles first .. end-1 of part `part` of `parts`; empty for the last parts of a row tile that sees few keys
C2T_HD void part_range(int tiles, int parts, int part, int* first, int* end) {
  int q, r;
  split(tiles, parts, 1.f / (float)parts, &q, &r);
  const int per = q + (r > 0), f = per * part;
  *first = f < tiles ? f : tiles;
  *end = f + per < tiles ? f + per : tiles;
}

}  // namespace c2t
