// The paged cache's bookkeeping and the movement of its tokens: reserve, write, commit, fork, truncate.
//
// A sequence holds the pages of its row of the page table (-1: none there); a page is free when nobody holds it (count 0).
// All of it lives on the device, so that a step whose lengths come from the step before needs no answer from it.
#pragma once
#include "k_common.h"
#include "k_paged.h"

namespace c2t {

constexpr int CACHE_NT = 256;
constexpr int RESERVE_NT = 1024;
constexpr int RESERVE_MAX_B = 4096;        // sequences; their counts are kept in LDS
constexpr int RESERVE_LANES = 16;          // lanes that look at a sequence's pages together
constexpr int MAX_PATH_TOKENS = 1025;             // tokens of an accepted path: the root and as many nodes as a tree may have

// one holder less; a count that is no one's is left alone
__device__ __forceinline__ bool let_go(int32_t* refcount) {
  if (atomicSub(refcount, 1) > 0) return true;
  atomicAdd(refcount, 1);
  return false;
}

// ---- write: K and V of the new tokens, one layer.  One 16-byte chunk of a token a thread.  Bound by the bytes: 64 sequences of 1024 tokens, 8 heads of
// 128, 93 us, 5.8 TB/s read and written; a prompt of 8 x 2048 16.7 us, 6.0 TB/s; a tree of 65 for 64 sequences 7.2 us, the call's own cost. ----
struct NewTokens {
  const char* k; const char* v;            // [batch][slots][kv_heads][head_dim]
  int64_t batch_stride, token_stride;      // of both, in bytes
  const int32_t* n_new;                    // [batch] or null: all slots
  int32_t slots;
};

__global__ __launch_bounds__(CACHE_NT) void k_cache_write(CacheView c, int layer, NewTokens x) {
  const int b = blockIdx.y, per_head = c.head_dim / 8, per_token = c.kv_heads * per_head;
  const int len = tokens_in_cache(c, c.length[b]);
  const int asked = x.n_new ? x.n_new[b] : x.slots, n = new_tokens(c, len, asked, x.slots);
  if (blockIdx.x == 0 && threadIdx.x == 0 && clamp_int(asked, 0, x.slots) > n) report(c, b, CACHE_ROW_FULL);
  const int64_t i = (int64_t)blockIdx.x * CACHE_NT + threadIdx.x;
  const int t = (int)(i / per_token), chunk = (int)(i % per_token);
  if (t >= n) return;
  const int at = len + t, head = chunk / per_head;
  const int page = valid_page(c, c.table[(int64_t)b * c.max_pages + (at >> c.page_shift)]);
  if (page < 0) { if (chunk == 0) report(c, b, CACHE_INVALID); return; }
  if (c.refcount[page] > 1) { if (chunk == 0) report(c, b, CACHE_SHARED); return; }
  const int64_t from = b * x.batch_stride + t * x.token_stride + (int64_t)chunk * 16;
  const int64_t to = (row_offset(c, layer, page, head, at & ((1 << c.page_shift) - 1)) + (chunk % per_head) * 8) * 2;
  *(uint4*)(c.k + to) = *(const uint4*)(x.k + from);
  *(uint4*)(c.v + to) = *(const uint4*)(x.v + from);
}

// ---- commit: the tokens in slots path[0] < path[1] < ... behind a sequence's length move to slots 0, 1, ..., all layers ----
struct Path { const int32_t* slot; const int32_t* n; int32_t stride; };

// Where token `at` of sequence b lies, page * page_size + row (below 2^31: checked by the host); -1 on no valid page.
__device__ __forceinline__ int token_place(const CacheView& c, int b, int64_t at, bool written, uint32_t* why) {
  if (at < 0 || at >= capacity_of(c)) { *why |= CACHE_INVALID; return -1; }
  const int page = valid_page(c, c.table[(int64_t)b * c.max_pages + (at >> c.page_shift)]);
  if (page < 0) { *why |= CACHE_INVALID; return -1; }
  if (written && c.refcount[page] > 1) { *why |= CACHE_SHARED; return -1; }
  return (page << c.page_shift) + (int)(at & ((1 << c.page_shift) - 1));
}
// Step i of a path: from where to where; nonzero `why`: the path is refused.
__device__ __forceinline__ int2 path_step(const CacheView& c, const Path& p, int b, int len, int i, uint32_t* why) {
  const int32_t* slot = p.slot + (int64_t)b * p.stride;
  const int s = slot[i];
  if (s < i || (i > 0 && slot[i - 1] >= s)) { *why |= CACHE_INVALID; return make_int2(-1, -1); }        // (rising from 0 or more: s >= i)
  return make_int2(token_place(c, b, (int64_t)len + s, false, why), token_place(c, b, (int64_t)len + i, s != i, why));
}

// Steps are taken in order, and path[i] >= i, so a row is read before a later step writes it.  Each thread moves one
// 16-byte column of one head for all steps, so that order holds without a barrier; batches of steps are loaded
// before they are stored: in a batch from step i on nothing is written below slot i, and nothing read there.  Bound by pieces of 256 bytes (a head's
// row of 128) whose places depend on the path: 64 sequences, 32 layers, paths of 8: 35 us, 3.4 TB/s read and written; paths of 32 173 us, 3.0;
// one sequence 6 us.
__global__ __launch_bounds__(CACHE_NT) void k_cache_commit(CacheView c, Path p) {
  constexpr int BATCH = 8;
  __shared__ int2 step[MAX_PATH_TOKENS];
  __shared__ uint32_t why_not;
  const int b = blockIdx.y, tid = threadIdx.x, per_head = c.head_dim / 8;
  const int len = tokens_in_cache(c, c.length[b]), n = clamp_int(p.n[b], 0, p.stride);
  if (tid == 0) why_not = 0u;
  __syncthreads();
  uint32_t why = 0u;
  for (int i = tid; i < n; i += CACHE_NT) step[i] = path_step(c, p, b, len, i, &why);
  if (why) atomicOr(&why_not, why);
  __syncthreads();
  if (why_not) return;
  const int64_t i = (int64_t)blockIdx.x * CACHE_NT + tid, columns = (int64_t)c.layers * 2 * c.kv_heads * per_head;
  if (i >= columns) return;
  const int column = (int)(i % per_head), head = (int)(i / per_head % c.kv_heads);
  const int64_t plane = i / per_head / c.kv_heads;                              // layer * 2 + (0: K, 1: V)
  char* base = ((plane & 1) ? c.v : c.k) + (row_offset(c, (int)(plane >> 1), 0, head, 0) + column * 8) * 2;
  const int mask = (1 << c.page_shift) - 1;
  auto row = [&](int place) -> uint4* {
    return (uint4*)(base + (((int64_t)(place >> c.page_shift) * c.kv_heads << c.page_shift) + (place & mask)) * c.head_dim * 2);
  };
  for (int s0 = 0; s0 < n; s0 += BATCH) {
    uint4 x[BATCH];
#pragma unroll
    for (int s = 0; s < BATCH; ++s) if (s0 + s < n && step[s0 + s].x != step[s0 + s].y) x[s] = *row(step[s0 + s].x);
#pragma unroll
    for (int s = 0; s < BATCH; ++s) if (s0 + s < n && step[s0 + s].x != step[s0 + s].y) *row(step[s0 + s].y) = x[s];
  }
}

// the sequences' lengths, once all tokens have moved; one wavefront a sequence
__global__ __launch_bounds__(CACHE_NT) void k_cache_commit_lengths(CacheView c, Path p) {
  const int b = blockIdx.x * (CACHE_NT / WAVE) + (threadIdx.x >> 6), lane = threadIdx.x & (WAVE - 1);
  if (b >= c.batch) return;
  const int len = tokens_in_cache(c, c.length[b]), n = clamp_int(p.n[b], 0, p.stride);
  uint32_t why = 0u;
  for (int i = lane; i < n; i += WAVE) (void)path_step(c, p, b, len, i, &why);
  const uint32_t all = wave_reduce_u32(why, 0u, [](uint32_t x, uint32_t y) { return x | y; });
  if (lane == 0) { if (all) report(c, b, all); else c.length[b] = len + n; }
}

// ---- truncate: shorter sequences; the pages past what they keep are let go ----
__global__ __launch_bounds__(CACHE_NT) void k_cache_truncate(CacheView c, const int32_t* new_length, int keep) {
  const int b = blockIdx.x;
  int len = tokens_in_cache(c, c.length[b]);
  if (new_length) len = min(len, max(new_length[b], 0));
  const int first = min((int)div_up64((int64_t)len + keep, 1 << c.page_shift), c.max_pages);
  __syncthreads();                                           // (every thread has read the length)
  if (threadIdx.x == 0) c.length[b] = len;
  int32_t* row = c.table + (int64_t)b * c.max_pages;
  bool bad = false;
  for (int i = first + threadIdx.x; i < c.max_pages; i += CACHE_NT) {
    const int page = row[i];
    if (page == -1) continue;
    row[i] = -1;
    if (valid_page(c, page) < 0 || !let_go(c.refcount + page)) bad = true;
  }
  if (bad) report(c, b, CACHE_INVALID);
}

// ---- fork: one workgroup an entry.  Entries that get in each other's way (a sequence that is made twice, or made and forked
// in the same call) are refused, all of them: whatever order they ran in would show. ----
__global__ __launch_bounds__(CACHE_NT) void k_cache_fork(CacheView c, const int32_t* src, const int32_t* dst, int n) {
  const int e = blockIdx.x, tid = threadIdx.x, s = src[e], d = dst[e];
  if (s < 0 || s >= c.batch || d < 0 || d >= c.batch || s == d) return;
  __shared__ int clash;
  if (tid == 0) clash = 0;
  __syncthreads();
  for (int i = tid; i < n; i += CACHE_NT) {
    if (i == e) continue;
    const int s2 = src[i], d2 = dst[i];
    if (s2 < 0 || s2 >= c.batch || d2 < 0 || d2 >= c.batch || s2 == d2) continue;
    if (d2 == d || s2 == d || d2 == s) clash = 1;
  }
  __syncthreads();
  if (clash) { if (tid == 0) report(c, d, CACHE_INVALID); return; }
  const int len = tokens_in_cache(c, c.length[s]), held = div_up(len, 1 << c.page_shift);
  const int32_t* from = c.table + (int64_t)s * c.max_pages;
  int32_t* to = c.table + (int64_t)d * c.max_pages;
  bool bad = false;
  for (int i = tid; i < c.max_pages; i += CACHE_NT) {
    const int old = to[i];
    int page = i < held ? from[i] : -1;
    if (i < held && valid_page(c, page) < 0) { page = -1; bad = true; }
    if (page >= 0) atomicAdd(c.refcount + page, 1);          // ahead of letting go: the two rows may hold the same page
    to[i] = page;
    if (old != -1 && (valid_page(c, old) < 0 || !let_go(c.refcount + old))) bad = true;
  }
  if (tid == 0) c.length[d] = len;
  if (bad) report(c, d, CACHE_INVALID);
}

// ---- reserve ----
// Entries first .. end-1 of a sequence's row have to be its own to write: no page there, or one that others hold as well,
// takes a fresh one.
struct Wanted { int first, end; uint32_t why; };
__device__ __forceinline__ Wanted wanted_pages(const CacheView& c, int len, int n_new) {
  Wanted w{0, 0, 0u};
  if (n_new <= 0) return w;
  if (n_new > capacity_of(c) - len) { w.why = CACHE_ROW_FULL; return w; }
  w.first = len >> c.page_shift;
  w.end = (int)div_up64((int64_t)len + n_new, 1 << c.page_shift);
  return w;
}

// Scratch: fresh [cap] page that the fresh place of each rank gets, given_up [cap] page that it replaces (-1: none, -2: not given
// out), cap = min(pages, batch * max_pages); copied [batch] page whose first tokens move to the sequence's fresh one (-1: none).
struct ReserveScratch { int32_t* fresh; int32_t* given_up; int32_t* copied; int32_t cap; };

// inclusive sum over the workgroup's threads of one number each, and the total
__device__ __forceinline__ int block_scan(int v, int* of_waves, int* total) {
  const int incl = wave_scan_incl(v), w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) of_waves[w] = incl;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < RESERVE_NT / WAVE; ++i) { const int x = of_waves[i]; before += i < w ? x : 0; all += x; }
  __syncthreads();
  *total = all;
  return before + incl;
}

// The same of numbers of up to 2^26 each.  4096 rows of so many places pass 31 bits (a rank that wrapped would be looked up far outside the list of pages), so
// the lanes' sums are made of halves of 16 bits and fewer.
__device__ __forceinline__ int64_t block_scan64(int v, int64_t* of_waves, int64_t* total) {
  const int64_t incl = ((int64_t)wave_scan_incl(v >> 16) << 16) + wave_scan_incl(v & 0xffff);
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) of_waves[w] = incl;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < RESERVE_NT / WAVE; ++i) { const int64_t x = of_waves[i]; before += i < w ? x : 0; all += x; }
  __syncthreads();
  *total = all;
  return before + incl;
}

// One workgroup: decisions of all sequences are made on the counts as they are at the start (a page that two of them hold is replaced
// for both), the lowest free pages go out in order of sequence and place.  Sequences are served in order until the pool runs out: one
// whose places do not all get a page gets none.  On a pool of some hundred pages latency bounds it, three or four trips to memory that wait for each
// other: 6 to 7 us for 2 or 80 sequences.  Pages in use come first, and are passed 4096 a round: 64 pages behind 18000 held ones take 11 us, behind 100000 39, behind 900000 300.
__global__ __launch_bounds__(RESERVE_NT) void k_cache_reserve(CacheView c, const int32_t* n_new, ReserveScratch x) {
  constexpr int GROUPS = RESERVE_NT / RESERVE_LANES;
  __shared__ int need[RESERVE_MAX_B];                        // places that need a page; then: those of the sequences before it
  __shared__ int of_waves[RESERVE_NT / WAVE];
  __shared__ int64_t places_of_waves[RESERVE_NT / WAVE];
  const int tid = threadIdx.x, group = tid / RESERVE_LANES, lane = tid % RESERVE_LANES;
  const uint64_t group_lanes = (0xffffull) << ((tid & 63) / RESERVE_LANES * RESERVE_LANES);
  auto needs_page = [&](int page) { return page < 0 || c.refcount[page] > 1; };        // (of a valid page or -1)

  for (int b = group; b < c.batch; b += GROUPS) {
    Wanted w = wanted_pages(c, tokens_in_cache(c, c.length[b]), n_new[b]);
    int count = 0;
    bool bad = false;
    for (int i0 = w.first; i0 < w.end; i0 += RESERVE_LANES) {
      const int i = i0 + lane;
      const int page = i < w.end ? c.table[(int64_t)b * c.max_pages + i] : 0;
      const bool broken = i < w.end && page != -1 && valid_page(c, page) < 0;
      const bool fresh = i < w.end && !broken && needs_page(page);
      bad = bad || (__ballot(broken) & group_lanes) != 0ull;
      count += __popcll(__ballot(fresh) & group_lanes);
    }
    if (bad) { w.why |= CACHE_INVALID; count = 0; }
    if (lane == 0) {
      need[b] = bad ? -1 : count;                            // -1: not served
      x.copied[b] = -1;
      if (w.why) report(c, b, w.why);
    }
  }
  __syncthreads();

  constexpr int64_t TOO_MANY = 1 << 30;                      // more than there may be pages; with a row's places it still fits 31 bits
  int64_t all = 0;                                           // of all sequences; need[b] becomes the count before b, sign: not served
  for (int b0 = 0; b0 < c.batch; b0 += RESERVE_NT) {
    const int b = b0 + tid, mine = b < c.batch ? need[b] : 0, v = max(mine, 0);
    int64_t total;
    const int64_t before = all + block_scan64(v, places_of_waves, &total) - v;
    if (b < c.batch) need[b] = mine < 0 ? -1 : (int)min(before, TOO_MANY);
    all += total;
  }
  __syncthreads();
  const int wanted = (int)min(all, (int64_t)x.cap);

  // the first `wanted` free pages, in order
  int found = 0;
  for (int p0 = 0; p0 < c.pages && found < wanted; p0 += RESERVE_NT * 4) {
    int free_of[4];
    int n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = p0 + tid * 4 + j;
      free_of[j] = p < c.pages && c.refcount[p] == 0;
      n += free_of[j];
    }
    int total;
    int rank = found + block_scan(n, of_waves, &total) - n;
#pragma unroll
    for (int j = 0; j < 4; ++j) if (free_of[j]) { if (rank < wanted) x.fresh[rank] = p0 + tid * 4 + j; rank += 1; }
    found += total;
  }
  const int given = min(found, wanted);
  __syncthreads();

  // tables; the counts still stand as they did
  for (int b = group; b < c.batch; b += GROUPS) {
    const int first_rank = need[b];
    if (first_rank < 0) continue;
    const int len = tokens_in_cache(c, c.length[b]);
    const Wanted w = wanted_pages(c, len, n_new[b]);
    int32_t* row = c.table + (int64_t)b * c.max_pages;
    int count = 0;
    for (int i0 = w.first; i0 < w.end; i0 += RESERVE_LANES) {        // how many: whether they all get one
      const int i = i0 + lane;
      count += __popcll(__ballot(i < w.end && needs_page(row[i])) & group_lanes);
    }
    const bool served = first_rank + count <= given;
    if (!served && count > 0 && lane == 0) report(c, b, CACHE_POOL_EMPTY);
    int rank0 = first_rank;
    for (int i0 = w.first; i0 < w.end; i0 += RESERVE_LANES) {
      const int i = i0 + lane;
      const int page = i < w.end ? row[i] : 0;
      const bool fresh = i < w.end && needs_page(page);
      const uint64_t here = __ballot(fresh) & group_lanes;
      if (fresh) {
        const int rank = rank0 + __popcll(here & ((1ull << (tid & 63)) - 1ull));
        if (rank < given) x.given_up[rank] = served ? page : -2;
        if (served) {
          row[i] = x.fresh[rank];
          if (i == w.first && page >= 0 && (len & ((1 << c.page_shift) - 1)) != 0) x.copied[b] = page;
        }
      }
      rank0 += __popcll(here);
    }
  }
  __syncthreads();
  for (int r = tid; r < given; r += RESERVE_NT) {
    const int old = x.given_up[r];
    if (old == -2) continue;
    c.refcount[x.fresh[r]] = 1;
    if (old >= 0) atomicSub(c.refcount + old, 1);
  }
}

// The tokens of a partial page that was shared, copied to the sequence's own, all layers.  One workgroup a head of a layer's K or V: 12 us for 48
// of 64 sequences, 16 layers of 8 heads of 128.
__global__ __launch_bounds__(CACHE_NT) void k_cache_copy_partial(CacheView c, ReserveScratch x) {
  const int b = blockIdx.y, from = x.copied[b];
  if (from < 0) return;
  const int len = tokens_in_cache(c, c.length[b]);
  const int to = valid_page(c, c.table[(int64_t)b * c.max_pages + (len >> c.page_shift)]);
  if (to < 0) return;
  const int head = blockIdx.x % c.kv_heads, plane = blockIdx.x / c.kv_heads;
  char* pool = (plane & 1) ? c.v : c.k;
  const uint4* s = (const uint4*)(pool + row_offset(c, plane >> 1, from, head, 0) * 2);
  uint4* d = (uint4*)(pool + row_offset(c, plane >> 1, to, head, 0) * 2);
  const int chunks = (len & ((1 << c.page_shift) - 1)) * c.head_dim / 8;
  for (int i = threadIdx.x; i < chunks; i += CACHE_NT) d[i] = s[i];
}

}  // namespace c2t
