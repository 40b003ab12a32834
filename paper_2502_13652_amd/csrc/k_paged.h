// What the paged K/V cache's kernels share: where a token of a sequence lies, and how attention's work is dealt to
// workgroups.  Every index that comes from device memory (lengths, counts, page numbers) passes through here on its way to
// an address.  Plain functions of numbers, for host and device, so that their bounds can be checked on the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace c2t {

#define C2T_HD __host__ __device__ __forceinline__

constexpr int KEY_BLOCK = 16;              // keys that lie in one page together: page sizes are multiples of it, pages start at multiples of it

struct CacheView {
  char* k; char* v;                        // [layers][pages][kv_heads][page_size][head_dim], 2 bytes an element
  int32_t* table;                          // [batch][max_pages]
  int32_t* length;                         // [batch]
  int32_t* refcount;                       // [pages]
  uint32_t* status;                        // [batch]
  int32_t batch, layers, pages, max_pages, kv_heads, head_dim;
  int32_t page_shift;                      // page_size = 1 << page_shift
};

C2T_HD int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
C2T_HD int div_up(int a, int b) { return (a + b - 1) / b; }
C2T_HD int64_t div_up64(int64_t a, int64_t b) { return (a + b - 1) / b; }

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
  int32_t max_parts;                       // of a unit, 2 or more
  int32_t run;                             // items in a row for one die
};
// Workgroups go to the chip's eight dies in turn.  Neighbouring items, whose rows share keys, belong on one die and its L2; runs of
// items are dealt to the dies in turn, since items come longest first.
constexpr int DIES = 8;
C2T_HD int item_of_workgroup(const AttendShape& a, int workgroup) {
  const int i = workgroup / DIES;
  return (i / a.run * DIES + workgroup % DIES) * a.run + i % a.run;
}
C2T_HD int64_t workgroups_for(const AttendShape& a, int64_t items) { return div_up64(items, DIES * a.run) * DIES * a.run; }
C2T_HD int row_tiles(const AttendShape& a, int n_new) { return (int)(((int64_t)n_new * a.group + (1 << a.rows_shift) - 1) >> a.rows_shift); }
C2T_HD int key_tiles(const AttendShape& a, int keys) { return (keys + (1 << a.keys_shift) - 1) >> a.keys_shift; }
C2T_HD int64_t sequence_tiles(const CacheView& c, const AttendShape& a, int len, int n_new) {
  return (int64_t)row_tiles(a, n_new) * c.kv_heads * key_tiles(a, len + n_new);
}
C2T_HD int tiles_per_part(const AttendShape& a, int64_t all_tiles) {
  const int64_t per = (all_tiles + (1 << a.target_shift) - 1) >> a.target_shift;
  return per < a.min_per ? a.min_per : per > (1 << 30) ? 1 << 30 : (int)per;
}
C2T_HD int parts_of(const AttendShape& a, int per, int len, int n_new) {
  const int t = key_tiles(a, len + n_new);
  const int parts = t <= per ? 1 : div_up(t, per);
  return parts < a.max_parts ? parts : a.max_parts;
}
// parts of all units of a sequence
C2T_HD int sequence_parts(const CacheView& c, const AttendShape& a, int per, int len, int n_new) {
  return n_new == 0 ? 0 : row_tiles(a, n_new) * c.kv_heads * parts_of(a, per, len, n_new);
}
// keys that some row of a tile of query rows sees, from the first: rows row0 .. of the sequence's n_new * group, `chain` causal slots ahead of the nodes
C2T_HD int keys_seen(const AttendShape& a, int len, int n_new, int chain, int row_tile) {
  const int64_t last_row = ((int64_t)(row_tile + 1) << a.rows_shift) - 1, rows = (int64_t)n_new * a.group;
  const int t = (int)((last_row < rows ? last_row : rows - 1) / a.group);
  return t < chain ? len + t + 1 : len + n_new;
}
// key tiles first .. end-1 of part `part` of `parts`; empty for the last parts of a row tile that sees few keys
C2T_HD void part_range(int tiles, int parts, int part, int* first, int* end) {
  const int per = div_up(tiles, parts);
  const int64_t f = (int64_t)per * part, e = f + per;
  *first = f < tiles ? (int)f : tiles;
  *end = e < tiles ? (int)e : tiles;
}

}  // namespace c2t
