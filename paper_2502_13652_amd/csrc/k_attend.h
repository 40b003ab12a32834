// Attention of new tokens (one token, a tree behind its root, a chunk of a prompt) over a paged K/V cache.
//
//   s_j = scale q.k_j over the keys j that the row sees,  p_j = e^(s_j - m),  m = max s,  out = sum p_j v_j / sum p_j
//
// One pass over the keys: a wavefront keeps, for every row it has, a reference m that follows the running maximum (of s log2 e), the sum l of p and
// sum p v, and multiplies the last two by 2^(m_old - m_new) where a tile raises m.  A row that sees no key has m = -inf, l = 0
// and is put out as zeros.  Where the second product takes weights rounded to 16 bits, l is their sum as rounded, so that a row of few or of sharp
// weights keeps a mean of its values: what one weight's rounding adds to the product it adds to the divisor.  If the log of the sum is asked for,
// the weights as they were are then summed too, for that alone.
//
// Rows: the query heads of one cached head share its keys, so rows are (slot, head of the group) with the head
// fastest.  Products are taken transposed: S^T = K Q^T leaves in a lane one row (lane & 15) and 4 neighbouring keys of each
// block of 16, which are just the operand that out^T = V^T P^T takes of two blocks: P never leaves its registers, and row
// statistics are one number a lane, reduced over 4 lanes.
//
// Two layouts.  A tile of 16 rows (single tokens, small trees): the keys' bytes bound it, so each of a workgroup's four wavefronts goes over key tiles of
// its own, K straight into the matrix operands, V through LDS for its transposition only.  64 single tokens of 300 to 8000 cached tokens, 32 heads
// over 8: 201 us for 1.09 GB of K and V, 5.4 TB/s; a kernel that only reads rows gets 6.4.  More rows: the matrix products and the weights' exponentials
// bound it, so the wavefronts share K and V tiles in LDS, two of them in turn, the next one's loads on their way while a tile is used.  Two
// chunks of 2048 behind 9000 and 31000 tokens, 64 wide, with the log of the sums: 465 to 488 us for 353 GFLOP, up to 0.76 PFLOP/s; vector instructions but the matrix unit's are issued for
// 55 % of that time and the matrix unit works for 38 %: the two hardly overlap.  64 trees of 65 behind 100 to 4000 tokens: 200 to 232 us for 116 GFLOP, up to 0.58 PFLOP/s; of 260 rows a
// head the last four take a third pass.  One token behind 701: 9.9 us, of which 8 are the launch, the item's search and the join of its parts.
#pragma once
#include "k_common.h"
#include "k_paged.h"

namespace c2t {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  typedef __bf16 T; typedef __bf16 T4 __attribute__((ext_vector_type(4))); typedef __bf16 T8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mfma(T8 a, T8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static constexpr uint32_t EXPONENT = 0x7f80u;
  static constexpr float TOP = 0.f, SLACK = 8.f;
};
struct F16 {
  typedef _Float16 T; typedef _Float16 T4 __attribute__((ext_vector_type(4))); typedef _Float16 T8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mfma(T8 a, T8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static constexpr uint32_t EXPONENT = 0x7c00u;
  static constexpr float TOP = 15.f, SLACK = 2.f;
};

struct AttendArgs {
  const char* q; char* out; float* lse;    // [batch][slots][heads][head_dim], strides in bytes; lse [batch][slots][heads] or null
  int64_t q_batch, q_token, out_batch, out_token;
  const int32_t* n_new;                    // [batch] or null: all slots
  const uint8_t* mask;                     // [batch][nodes][nodes] or null
  int32_t nodes, chain;                    // slots = chain + nodes
  int32_t layer;
  float scale_log2e;
  // records of parts: [records][rows of a tile][head_dim], and (m, l) of each row, with `lse` also the sum of its weights as they were.  Joined by the
  // unit's last part: tickets [records], parts of the unit with that first record that have left theirs, zero between launches.  Joined by a launch of
  // their own: what each record is of, and how many there are.
  float* part_o; float2* part_ml; float* part_e; int32_t* tickets;
  struct Unit* units; int32_t* n_records;
  AttendShape shape;
};

// What a workgroup, and the join of its unit, know of where they are.
struct Unit { int b, len, n_new, row_tile, head, part, parts, slot0; };   // slot0: record of the unit's first part

// Deals a workgroup its item.  Every wavefront computes it for itself, each lane summing a stretch of sequences: no barrier.  Where
// each lane has one sequence at most, the longest go first: workgroups start in about this order, and none that starts last is long.  It costs
// 8 to 12 us of a launch of 64 sequences; a launch of its own that left a list would cost a launch.  Past 64 a lane reads its sequences one after the other, twice, and items come
// in no order: 512 tokens behind 300 to 2000 take 438 us for bytes of 500, but 4096 behind 30 to 300 2.8 ms for 0.6, most of it the search (behind one token each 2.5 ms).
// False: there is no item for it.
__device__ __forceinline__ bool find_item(const CacheView& c, const AttendArgs& a, int workgroup, Unit* u) {
  const int lane = lane_id(), each = div_up(c.batch, WAVE), b0 = min(lane * each, c.batch), b1 = min(b0 + each, c.batch);
  const bool reports = workgroup == 0 && threadIdx.x < WAVE;
  auto load = [&](int b, int* n) {
    const int len = tokens_in_cache(c, c.length[b]), asked = a.n_new ? a.n_new[b] : a.shape.slots;
    *n = new_tokens(c, len, asked, a.shape.slots);
    if (reports && clamp_int(asked, 0, a.shape.slots) > *n) report(c, b, CACHE_ROW_FULL);
    return len;
  };
  // of a lane with one sequence: that one; of one with more: the first, and the one that is found
  int my_b = b0, my_n = 0, my_len = 0;
  if (b0 < b1) my_len = load(b0, &my_n);
  if (each == 1 && c.batch > 1) {
    // in steps of 32 keys, equal ones by lane: numbers of their own, one comparison each
    const uint32_t cost = b0 < b1 ? (uint32_t)((my_len + my_n) >> 5) << 6 | (uint32_t)(WAVE - 1 - lane) : 0u;
    int rank = 0;
    for (int j = 0; j < c.batch; ++j) rank += (uint32_t)__builtin_amdgcn_readlane((int)cost, j) > cost;
    if (b0 >= b1) rank = lane;
    my_b = __builtin_amdgcn_ds_permute(rank * 4, my_b);
    my_n = __builtin_amdgcn_ds_permute(rank * 4, my_n);
    my_len = __builtin_amdgcn_ds_permute(rank * 4, my_len);
  }
  const int tiles = row_tiles(a.shape, my_n);
  float mine = b0 < b1 ? sequence_tiles(c, a.shape, my_len, my_n) : 0.f;
#pragma unroll 1
  for (int b = b0 + 1; b < b1; ++b) { int n; const int len = load(b, &n); mine += sequence_tiles(c, a.shape, len, n); }
  const int per = tiles_per_part(a.shape, (float)wave_sum((double)mine));
  const float inv_per = __builtin_amdgcn_rcpf((float)per);
  int my_parts = parts_of(a.shape, per, inv_per, my_len, my_n);
  const int first_parts = b0 < b1 ? my_parts * tiles * c.kv_heads : 0;
  int items = first_parts, slots = my_parts > 1 ? first_parts : 0;
#pragma unroll 1
  for (int b = b0 + 1; b < b1; ++b) {
    int n; const int len = load(b, &n), p = parts_of(a.shape, per, inv_per, len, n), parts = p * row_tiles(a.shape, n) * c.kv_heads;
    items += parts;
    if (p > 1) slots += parts;
  }
  const int items_to = wave_scan_incl(items), slots_to = wave_scan_incl(slots);
  if (workgroup == 0 && threadIdx.x == WAVE - 1) *a.n_records = slots_to;
  const int w = item_of_workgroup(a.shape, workgroup);
  int item0 = items_to - items, slot0 = slots_to - slots;
  const bool here = w >= item0 && w < item0 + items;
  const uint64_t has = __ballot(here);
  if (has == 0ull) return false;
  if (each > 1 && here) {
    int parts = first_parts;
#pragma unroll 1
    for (int b = b0; w >= item0 + parts; ) {                 // (it ends: the lane has the item)
      item0 += parts;
      if (my_parts > 1) slot0 += parts;
      my_b = ++b;
      my_len = load(b, &my_n);
      my_parts = parts_of(a.shape, per, inv_per, my_len, my_n);
      parts = my_parts * row_tiles(a.shape, my_n) * c.kv_heads;
    }
  }
  const int from = __builtin_ctzll(has);
  u->b = __builtin_amdgcn_readlane(my_b, from);
  u->len = __builtin_amdgcn_readlane(my_len, from);
  u->n_new = __builtin_amdgcn_readlane(my_n, from);
  u->parts = __builtin_amdgcn_readlane(my_parts, from);
  const int rel = __builtin_amdgcn_readlane(w - item0, from), first_slot = __builtin_amdgcn_readlane(slot0, from);
  const int n_tiles = row_tiles(a.shape, u->n_new);
  // row tiles of the same keys next to each other: they run at the same time.  The last first: of a causal chunk they see the most keys
  int rest, tile, head, part;
  split(rel, n_tiles, __builtin_amdgcn_rcpf((float)n_tiles), &rest, &tile);
  split(rest, u->parts, __builtin_amdgcn_rcpf((float)u->parts), &head, &part);
  u->row_tile = uniform(n_tiles - 1 - tile);
  u->head = uniform(head); u->part = uniform(part);
  u->slot0 = first_slot + (u->head * n_tiles + u->row_tile) * u->parts;
  return true;
}

template <typename E, int D> struct TileLayout {
  // rows of a tile in LDS, bytes: the reads of 16 rows' fragments (K) and of four rows' 32 bytes (V, transposed) then fall on different banks
  static constexpr int K_ROW = D * 2 + 16, V_ROW = D * 2 + 32;
};

template <typename E> __device__ __forceinline__ uint32_t odd_halves(uint32_t w) {     // halves whose exponent is all ones, as a mask of them
  return ((w & E::EXPONENT) == E::EXPONENT ? 0xffffu : 0u) | (((w >> 16) & E::EXPONENT) == E::EXPONENT ? 0xffff0000u : 0u);
}

// four neighbouring elements of a row's output, and with the first of them its log of the sum
template <typename E, int D>
__device__ __forceinline__ void put_row(const CacheView& c, const AttendArgs& a, const Unit& u, int t, int g, int dim, f32x4 x, float m, float l, float e) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  typename E::T4 y;
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = (typename E::T)(x[r] * inv);
  *(typename E::T4*)(a.out + u.b * a.out_batch + t * a.out_token + (query_offset(u.head, a.shape.group, g, D) + dim) * 2) = y;
  if (dim == 0 && a.lse) {
    // of a sum as if the reference were the largest score: the log's own rounding is then of its size, not of the distance between the two
    constexpr float BELOW = E::TOP - E::SLACK;
    constexpr float UNIT = BELOW < 0.f ? (float)(1 << (int)-BELOW) : 1.f / (float)(1 << (int)BELOW);     // 2^-BELOW
    a.lse[((int64_t)u.b * a.shape.slots + t) * c.kv_heads * a.shape.group + query_offset(u.head, a.shape.group, g, 1)] = l == 0.f ? -INFINITY : ((m + BELOW) + __builtin_amdgcn_logf(e * UNIT)) * 0.69314718055994531f;
  }
}
// running join of parts
struct Joined {
  float m = -INFINITY, l = 0.f, e = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(float2 ml, float of_e, f32x4 x) {
    const float m_new = fmaxf(m, ml.x), ref = m_new == -INFINITY ? 0.f : m_new;
    const float back = __builtin_amdgcn_exp2f(m - ref), f = __builtin_amdgcn_exp2f(ml.x - ref);
    l = l * back + ml.y * f;
    e = e * back + of_e * f;
    o = o * back + x * f;
    m = m_new;
  }
};

// A product's result may be read only some issue slots after the product, which the compiler counts.  An earlier form of the loop below, which read its scores in a later
// block than the products', was compiled to read them too early, so scores are put into ordinary registers in the block that makes them.  Outputs are
// read behind the next tile's products or after the loop, both far enough.  tests/test_matrix_waits.py looks at every path of the builds as compiled.
template <typename X> __device__ __forceinline__ void settle(X& x) { asm volatile("" : "+v"(x)); }

// x scale - ref, the product rounded
__device__ __forceinline__ float rounded_difference(float x, float scale, float ref) {
#pragma clang fp contract(off)
  const float y = x * scale;
  return y - ref;
}

// pairs of numbers that one workgroup writes and another reads in the same launch
__device__ __forceinline__ void st_dev64(uint64_t* p, float x, float y) {
  __hip_atomic_store(p, (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 ld_dev64(const uint64_t* p) {
  const uint64_t v = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// MT tiles of 16 rows a wavefront; RW wavefronts share the key tiles and have rows of their own, or (RW = 1) KW wavefronts have the same rows
// and key tiles of their own, joined at the end.  KB blocks of 16 keys a tile.  OCC workgroups a CU.  NODES: some slots
// are nodes with a mask; the code for it, where it is never used, costs a chunk of 2048 tokens 560 us for 505.
template <typename E, int D, int MT, int RW, int KW, int KB, int OCC, bool NODES>
__global__ __launch_bounds__(64 * RW * KW, OCC) void k_attend(CacheView c, AttendArgs a) {
  static_assert(RW == 1 || KW == 1, "rows or keys");
  typedef typename E::T T; typedef typename E::T4 T4; typedef typename E::T8 T8;
  typedef TileLayout<E, D> L;
  constexpr int NT = 64 * RW * KW, KT = 16 * KB, CH = D / 8 /* 16-byte chunks of a row */, DB = D / 16, DK = D / 32;
  constexpr int SHARERS = 64 * RW;                          // threads that load a tile together
  constexpr int LOADS = KT * CH / SHARERS;                  // chunks each of K and V a thread
  constexpr int ROWS_A_LOAD = SHARERS / CH;
  static_assert(ROWS_A_LOAD <= 16 ? 16 % ROWS_A_LOAD == 0 : ROWS_A_LOAD % 16 == 0, "");
  constexpr bool K_LDS = RW > 1;
  // A weight as the second product takes it: one number of 16 bits, off by 2^-8 of it at most (2^-11 for halves that are not subnormal), or a second one for what the first leaves,
  // off by 2^-16 (2^-22).  Where the keys' bytes bound the kernel the second costs next to nothing (64 tokens 200 us with and without, one 9.9 and 9.7) and the output is as exact as its type; elsewhere it
  // costs the 64 trees 261 us for 200, the two chunks 640 for 472 and tiles of 64 rows 1 to 12 %, and is left out: of Gaussian keys and values outputs are then off by 0.0022 of their size
  // (rms, of bf16; 0.0017 of it are their own rounding, of halves 0.00027 and 0.00021).
  constexpr bool PAIRS = KW > 1;
  constexpr int TILE_BYTES = KT * L::V_ROW + (K_LDS ? KT * L::K_ROW : 0);
  constexpr int JOIN_BYTES = KW > 1 ? KW * 16 * (D + 3) * 4 : 0;
  constexpr int BUFFERS = RW > 1 ? 2 : KW;                  // of the tile: the next one's while this one is used, or one a wavefront
  constexpr int LDS_BYTES = BUFFERS * TILE_BYTES > JOIN_BYTES ? BUFFERS * TILE_BYTES : JOIN_BYTES;
  // A row's reference is only raised where a weight would pass 2^TOP, and then to where the largest is 2^(TOP - SLACK).  Of bf16, whose values may be as large as an fp32
  // number, no weight is above 1: the products then overflow only where their sum does.  Halves have 2^-14 for their least number of
  // all bits and 2^-24 for their least: at the top of their range, weights of 2^-27 of a row's largest keep all bits, and what the others lose is 2^-38
  // of the largest at most (keys of small weights are many, and all there is where a sharp key's value is 0).  A slack of 8 saves the two chunks 0.4 %.
  constexpr float TOP = E::TOP, SLACK = E::SLACK;
  // Weights are 2^(s log2 e - m), with one rounding, but m was rounded from such a product itself, and where it is this large the two are a fourth and more apart, in the end by
  // more than exponents hold.  From there on the scores' products are rounded first, as the references' were (for all tiles so, one multiplication a weight more).  Rows of such scores are as
  // sharp as rows get: it is for them to be the value of their largest score, and not zeros or NaN.
  constexpr float BIG = 0x1p22f;
  int big = 0;
  float factor = a.scale_log2e;                              // of the scores, which from there on are multiplied already: 1
  __shared__ __align__(16) char lds[LDS_BYTES];
  __shared__ int odd_value;                                  // a tile held a value that is not finite

  Unit u;
  if (!find_item(c, a, blockIdx.x, &u)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 15, quad = lane >> 4;
  const int rw = RW > 1 ? wave : 0, kw = KW > 1 ? wave : 0;
  const int rows = u.n_new * a.shape.group, G = a.shape.group;
  const int wave_row0 = (u.row_tile << a.shape.rows_shift) + rw * 16 * MT;

  const int seen = keys_seen(a.shape, u.len, u.n_new, a.chain, u.row_tile);
  int tile, tile_end;
  part_range(key_tiles(a.shape, seen), u.parts, u.part, &tile, &tile_end);
  // keys below this are seen by every row of the wavefront
  int first_slot, first_g;
  split(wave_row0 < rows ? wave_row0 : 0, G, a.shape.inv_group, &first_slot, &first_g);
  const int all_see = uniform(u.len + min(first_slot + 1, a.chain));
  const bool idle = wave_row0 >= rows;                       // no row of the wavefront's: it only helps to load
  const int32_t* const table = c.table + (int64_t)u.b * c.max_pages;
  const uint8_t* const mask = a.mask ? a.mask + (int64_t)u.b * a.nodes * a.nodes : nullptr;
  auto sees = [&](int t, int key) {                          // slot t, key below `seen`
    const int s = key - u.len;
    bool yes = s < a.chain && (t >= a.chain || s <= t);
    if (NODES && t >= a.chain && s >= a.chain) yes = mask[(t - a.chain) * a.nodes + (s - a.chain)] != 0;      // (nodes^2: at most 2^20)
    return yes;
  };
  // the page that a block of 16 keys lies in, -1 behind the last key or if the table has none
  auto page_of = [&](int key) { return key < seen ? valid_page(c, table[key >> c.page_shift]) : -1; };
  const int in_page = (1 << c.page_shift) - 1;
  const int64_t head_offset = row_offset(c, a.layer, 0, u.head, 0) * 2;
  const uint32_t page_bytes = (uint32_t)(c.kv_heads << c.page_shift) * (D * 2);      // at most 2^27: 1024 heads, 256 tokens, 256 wide
  const char* const k_head = c.k + head_offset;
  const char* const v_head = c.v + head_offset;

  // this lane's rows and their queries
  int slot[MT];
  T8 q[MT][DK];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int r = wave_row0 + m * 16 + col;
    int g;
    split(r, G, a.shape.inv_group, &slot[m], &g);
    if (r >= rows) slot[m] = -1;
#pragma unroll
    for (int kk = 0; kk < DK; ++kk) {
      if (slot[m] >= 0) q[m][kk] = *(const T8*)(a.q + u.b * a.q_batch + slot[m] * a.q_token + (query_offset(u.head, G, g, D) + kk * 32 + quad * 8) * 2);
      else q[m][kk] = T8{};
    }
  }

  f32x4 o[MT][DB];
  float m_run[MT], l_run[MT], e_run[MT];                     // sums of weights: rounded ones of the row, and this lane's keys' as they were (with PAIRS or `lse`)
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    m_run[m] = -INFINITY; l_run[m] = 0.f; e_run[m] = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[m][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  u32x4 vr[LOADS];
  u32x4 kr[K_LDS ? LOADS : KB * DK];
  const int lt = RW > 1 ? tid : lane;                        // this thread among those that load the tile
  uint32_t there = 0u; bool full = false;                    // blocks of the requested tile that lie on a page; all do, and no key is past the last
  // The pages of a tile's blocks, one a lane: asked for a tile ahead of the keys, which cannot be asked for without them.  Without a condition (blocks
  // behind the last key take its page): with one, the register that some lanes leave alone is waited for, and every load before it.
  auto pages_of = [&](int t) { return table[min(t * KT + (lane % KB) * 16, seen - 1) >> c.page_shift]; };
  // Every lane loads, without a condition that would make each load wait for itself: a block that is on no page comes from the pool's first page, and
  // rows behind the last key lie on its page; both are taken out before they are used.
  auto request = [&](int t, int pages) {
    const int key0 = t * KT;
    constexpr int BLOCKS_A_LOAD = ROWS_A_LOAD > 16 ? ROWS_A_LOAD / 16 : 1, LOADS_A_BLOCK = ROWS_A_LOAD > 16 ? 1 : 16 / ROWS_A_LOAD;
    const int in = lt / CH % 16 * (D * 2) + lt % CH * 16;
    static_assert(64 / CH <= 16, "a wavefront's rows lie in one block");
    const int block = uniform(lt / CH / 16);
    uint64_t mine = 0;
    there = 0u;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      // scalar, and few: a quarter of what a tile's instructions were went into this
      const int key = key0 + kb * 16;
      const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(pages, kb);
      const bool ok = page < (uint32_t)c.pages && key < seen;
      there |= ok ? 1u << kb : 0u;
      const uint64_t off = (uint64_t)(ok ? page : 0u) * page_bytes + (uint32_t)((key & in_page) * (D * 2));
      if (BLOCKS_A_LOAD == 1) {
#pragma unroll
        for (int x = 0; x < LOADS_A_BLOCK; ++x) {
          const int j = kb * LOADS_A_BLOCK + x;
          vr[j] = *(const u32x4*)(v_head + off + in + x * ROWS_A_LOAD * (D * 2));
          if (K_LDS) kr[j] = *(const u32x4*)(k_head + off + in + x * ROWS_A_LOAD * (D * 2));
        }
      } else {
        if (kb % BLOCKS_A_LOAD == 0 || block == kb % BLOCKS_A_LOAD) mine = off;
        if (kb % BLOCKS_A_LOAD == BLOCKS_A_LOAD - 1) {
          vr[kb / BLOCKS_A_LOAD] = *(const u32x4*)(v_head + mine + in);
          if (K_LDS) kr[kb / BLOCKS_A_LOAD] = *(const u32x4*)(k_head + mine + in);
        }
      }
      if (!K_LDS) {
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) kr[kb * DK + kk] = *(const u32x4*)(k_head + off + col * (D * 2) + quad * 16 + kk * 64);
      }
    }
    full = key0 + KT <= seen && there == (1u << KB) - 1u;
  };

  // the requested tile into LDS
  auto stage = [&](int t, char* v_lds) {
    const int key0 = t * KT;
    if (!full) {
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const int row = j * ROWS_A_LOAD + lt / CH;
        const bool ok = key0 + row < seen && (there >> (row / 16) & 1u);
        vr[j] = ok ? vr[j] : u32x4{0u, 0u, 0u, 0u};
      }
    }
    bool odd = false;
    if (key0 + KT > u.len) {                                 // holds new tokens: some rows may see a value that others do not
      // 0 x infinity is not 0: a value that is not finite is left out of the product and added for the rows that see it
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const uint32_t x = odd_halves<E>(vr[j].x), y = odd_halves<E>(vr[j].y), z = odd_halves<E>(vr[j].z), w = odd_halves<E>(vr[j].w);
        odd = odd || (x | y | z | w) != 0u;
        vr[j].x &= ~x; vr[j].y &= ~y; vr[j].z &= ~z; vr[j].w &= ~w;
      }
      odd = __any(odd);
    }
    char* const k_lds = v_lds + KT * L::V_ROW;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = j * ROWS_A_LOAD + lt / CH;
      *(u32x4*)(v_lds + row * L::V_ROW + lt % CH * 16) = vr[j];
      if (K_LDS) *(u32x4*)(k_lds + row * L::K_ROW + lt % CH * 16) = kr[j];
    }
    return odd;
  };

  const int step = KW, first_key = tile * KT;
  tile += kw;
  const int first_tile = tile;
  int pages = pages_of(tile), buffer = 0;
  uint32_t on_page = 0u;                                     // of the tile in LDS
  bool all_there = false, odd = false;
  if (tile < tile_end) request(tile, pages);
  pages = pages_of(tile + step);
  // Keys on no page are left out, and the status says so: looked for by one head's last row tile, which sees all keys, while the first tile is on
  // its way (noted tile by tile in the loop, 230 us became 232 for the 64 trees and 478 became 483 for the chunks; so, 231 and 480).
  if (u.head == 0 && wave == 0 && (u.row_tile + 1) << a.shape.rows_shift >= rows) {
    bool none = false;
    for (int i = (first_key >> c.page_shift) + lane; i << c.page_shift < min(tile_end * KT, seen); i += WAVE) none = none || valid_page(c, table[i]) < 0;
    if (__any(none) && lane == 0) report(c, u.b, CACHE_INVALID);
  }
  // The queries are here before the loop: loads that were still on their way when it starts would be waited for in each of its rounds, and the next
  // tile's, which are younger, with them.
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int kk = 0; kk < DK; ++kk) { u32x4 x = __builtin_bit_cast(u32x4, q[m][kk]); settle(x); q[m][kk] = __builtin_bit_cast(T8, x); }
  if (RW > 1) {                                              // (the loop is the same for all wavefronts, which meet in it)
    if (tid == 0) odd_value = 0;
    __syncthreads();
    if (tile < tile_end) {
      if (stage(tile, lds) && lane == 0) odd_value = 1;
      on_page = there; all_there = full;
      if (tile + 1 < tile_end) request(tile + 1, pages);
      pages = pages_of(tile + 2);
    }
    __syncthreads();
  }
  for (; tile < tile_end; tile += step) {
    const int key0 = tile * KT;
    char* const v_lds = lds + (RW > 1 ? buffer : kw) * TILE_BYTES;
    char* const k_lds = v_lds + KT * L::V_ROW;
    T8 kf[K_LDS ? 1 : KB][K_LDS ? 1 : DK];
    if (RW == 1) {
      if (stage(tile, v_lds)) odd = true;
      on_page = there; all_there = full;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) kf[K_LDS ? 0 : kb][K_LDS ? 0 : kk] = __builtin_bit_cast(T8, kr[K_LDS ? 0 : kb * DK + kk]);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront"); __builtin_amdgcn_wave_barrier(); __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      if (tile + step < tile_end) request(tile + step, pages);
      pages = pages_of(tile + 2 * step);
    }
    const bool whole = all_there && key0 + KT <= all_see;    // every row sees every key of the tile
    const uint32_t blocks = on_page;

    f32x4 s[MT][KB];
    if (!idle) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int m = 0; m < MT; ++m) s[m][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) {
          const T8 k = K_LDS ? *(const T8*)(k_lds + (kb * 16 + col) * L::K_ROW + kk * 64 + quad * 16) : kf[K_LDS ? 0 : kb][K_LDS ? 0 : kk];
#pragma unroll
          for (int m = 0; m < MT; ++m) s[m][kb] = E::mfma(k, q[m][kk], s[m][kb]);
        }
      }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) settle(s[m][kb]);
      if (!whole) {
        // of nodes, mask bytes: a word of the lane's keys, asked for together and without a condition, from the nearest place that there is
        uint32_t open[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) open[m] = 0u;
        if (NODES && key0 + KT > u.len + a.chain) {
          const int s0 = key0 + quad * 4 - u.len - a.chain;    // node that the lane's first key is
          uint8_t byte[MT][KB][4];
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int r = 0; r < 4; ++r) byte[m][kb][r] = mask[max(slot[m] - a.chain, 0) * a.nodes + max(0, min(s0 + kb * 16 + r, a.nodes - 1))];
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int r = 0; r < 4; ++r) open[m] |= byte[m][kb][r] != 0 && slot[m] >= a.chain ? 1u << (kb * 4 + r) : 0u;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          // keys that the row sees without a mask
          const int below = min(seen, slot[m] < 0 ? 0 : u.len + min(slot[m] + 1, a.chain)), k = key0 + quad * 4;
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool yes = (blocks >> kb & 1u) && (k + kb * 16 + r < below || (NODES && k + kb * 16 + r < seen && (open[m] >> (kb * 4 + r) & 1u)));
              s[m][kb][r] = yes ? s[m][kb][r] : -INFINITY;
            }
        }
      }

      if (big != 0) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) s[m][kb] *= a.scale_log2e;
      }

      T8 p[MT][KB / 2], rest[PAIRS ? MT : 1][PAIRS ? KB / 2 : 1];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        float top = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, s[m][kb][r]);
        top *= factor;
        if (__any(top - m_run[m] > TOP)) {                 // (uniform) of all four lanes of a row, then
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          float m_new = fmaxf(m_run[m], top - (TOP - SLACK));
          if (top - m_new > TOP) m_new = top;                // (it was rounded further down)
          if (big == 0 && __any(__builtin_fabsf(m_new) >= BIG && m_new != -INFINITY)) {
            big = 1; factor = 1.f;
#pragma unroll
            for (int n = m; n < MT; ++n)
#pragma unroll
              for (int kb = 0; kb < KB; ++kb) s[n][kb] *= a.scale_log2e;
          }
          const float back = __builtin_amdgcn_exp2f(m_run[m] - (m_new == -INFINITY ? 0.f : m_new));
          m_run[m] = m_new;
          l_run[m] *= back; e_run[m] *= back;
#pragma unroll
          for (int d = 0; d < DB; ++d) o[m][d] *= back;
        }
        const float ref = m_run[m] == -INFINITY ? 0.f : m_run[m];
#pragma unroll
        for (int h = 0; h < KB / 2; ++h) {
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][h * 2 + r / 4][r % 4], factor, -ref));
            s[m][h * 2 + r / 4][r % 4] = w;
            p[m][h][r] = (T)w;
            if (PAIRS) rest[PAIRS ? m : 0][PAIRS ? h : 0][r] = (T)(w - (float)p[m][h][r]);
          }
        }
        if (PAIRS || a.lse) {
          f32x4 all = s[m][0];
#pragma unroll
          for (int kb = 1; kb < KB; ++kb) all += s[m][kb];
          e_run[m] += (all[0] + all[1]) + (all[2] + all[3]);
        }
      }
      // The rounded weights' sum is a product with ones: the matrix unit has time for it.  The two chunks, with `lse`, 479 us, with additions of pairs 484, with the
      // sum of the weights as they were for divisor 468; the 64 trees 232, 235 and 237.
      f32x4 sum[MT];
      if constexpr (!PAIRS) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          T8 ones;
#pragma unroll
          for (int r = 0; r < 8; ++r) ones[r] = (T)1.f;
          sum[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int h = 0; h < KB / 2; ++h) sum[m] = E::mfma(ones, p[m][h], sum[m]);
        }
      }
#pragma unroll
      for (int h = 0; h < KB / 2; ++h) {
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          // keys 4 quad + r of two blocks, as P holds them
          const char* at = v_lds + (h * 32 + quad * 4 + col / 4) * L::V_ROW + d * 32 + col % 4 * 8;
          typedef __attribute__((address_space(3))) s16x4* lds4;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 16 * L::V_ROW));
          struct { s16x4 a, b; } pair{lo, hi};
          const T8 v = __builtin_bit_cast(T8, pair);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            o[m][d] = E::mfma(v, p[m][h], o[m][d]);
            if (PAIRS) o[m][d] = E::mfma(v, rest[PAIRS ? m : 0][PAIRS ? h : 0], o[m][d]);
          }
        }
      }
      if constexpr (!PAIRS) {
#pragma unroll
        for (int m = 0; m < MT; ++m) l_run[m] += sum[m][0];
      }
    }
    if (RW > 1) {
      if (tile + 1 < tile_end) {
        if (stage(tile + 1, lds + (buffer ^ 1) * TILE_BYTES) && lane == 0) odd_value = 1;
        on_page = there; all_there = full;
        if (tile + 2 < tile_end) request(tile + 2, pages);
        pages = pages_of(tile + 3);
      }
      __syncthreads();
      buffer ^= 1;
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    e_run[m] += __shfl_xor(e_run[m], 16); e_run[m] += __shfl_xor(e_run[m], 32);
    if (PAIRS) l_run[m] = e_run[m];
#pragma unroll
    for (int d = 0; d < DB; ++d) settle(o[m][d]);
  }

  // Values that are not finite were left out of the products; rows that see their keys get them here.  A weight is made again from its key.
  if (RW > 1 ? odd_value != 0 : odd) {
    for (int key = first_key; key < tile_end * KT; ++key) {
      if (key + KT - key % KT <= u.len || (KW > 1 && key / KT % KW != first_tile % KW) || key >= seen || idle) continue;
      const int page = uniform(page_of(key));
      if (page < 0) continue;
      const uint64_t at = (uint64_t)(uint32_t)page * page_bytes + (uint32_t)((key & in_page) * (D * 2));
      T4 v[DB];
      bool any = false;
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        v[d] = *(const T4*)(v_head + at + (d * 16 + quad * 4) * 2);
#pragma unroll
        for (int r = 0; r < 4; ++r) any = any || !(__builtin_fabsf((float)v[d][r]) < INFINITY);
      }
      if (!__any(any)) continue;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        float x = 0.f;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) {
          const T8 k = *(const T8*)(k_head + at + quad * 16 + kk * 64);
#pragma unroll
          for (int r = 0; r < 8; ++r) x = __builtin_fmaf((float)k[r], (float)q[m][kk][r], x);
        }
        x += __shfl_xor(x, 16); x += __shfl_xor(x, 32);
        const float w = __builtin_amdgcn_exp2f(rounded_difference(x, a.scale_log2e, m_run[m] == -INFINITY ? 0.f : m_run[m]));
        if (slot[m] < 0 || !sees(slot[m], key)) continue;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) { const float y = (float)v[d][r]; if (!(__builtin_fabsf(y) < INFINITY)) o[m][d][r] += w * y; }
      }
    }
  }

  // what this workgroup has of a row: to the record of its part, or out
  const auto put = [&](int row_in_tile, int t, int g, int dim, f32x4 x, float m, float l, float e) {
    if (u.parts == 1) { put_row<E, D>(c, a, u, t, g, dim, x, m, l, e); return; }
    const int64_t rec = ((int64_t)(u.slot0 + u.part) << a.shape.rows_shift) + row_in_tile;
    float* to = a.part_o + rec * D + dim;
    if (KW > 1) {
      st_dev64((uint64_t*)to, x[0], x[1]); st_dev64((uint64_t*)to + 1, x[2], x[3]);
      if (dim == 0) { st_dev64((uint64_t*)(a.part_ml + rec), m, l); if (a.lse) st_dev(a.part_e + rec, e); }
    } else {
      *(f32x4*)to = x;
      if (dim == 0) { a.part_ml[rec] = make_float2(m, l); if (a.lse) a.part_e[rec] = e; }
    }
  };
  if (KW == 1) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int r = wave_row0 + m * 16 + col;
      if (slot[m] < 0) continue;
#pragma unroll
      for (int d = 0; d < DB; ++d) put(rw * 16 * MT + m * 16 + col, slot[m], r - slot[m] * G, d * 16 + quad * 4, o[m][d], m_run[m], l_run[m], e_run[m]);
    }
  } else {
    // the wavefronts' results of 16 rows at a time through LDS
    float* const jo = (float*)lds;                           // [KW][16][D]
    float* const jm = jo + KW * 16 * D; float* const jl = jm + KW * 16; float* const je = jl + KW * 16;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      __syncthreads();
#pragma unroll
      for (int d = 0; d < DB; ++d) *(f32x4*)(jo + (kw * 16 + col) * D + d * 16 + quad * 4) = o[m][d];
      if (quad == 0) { jm[kw * 16 + col] = m_run[m]; jl[kw * 16 + col] = l_run[m]; je[kw * 16 + col] = e_run[m]; }
      __syncthreads();
      for (int i = tid; i < 16 * D / 4; i += NT) {
        const int row = i / (D / 4), dim = i % (D / 4) * 4, r = wave_row0 + m * 16 + row;
        if (r >= rows) continue;
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < KW; ++w) mm = fmaxf(mm, jm[w * 16 + row]);
        const float ref = mm == -INFINITY ? 0.f : mm;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f, e = 0.f;
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          const float f = __builtin_amdgcn_exp2f(jm[w * 16 + row] - ref);
          l += f * jl[w * 16 + row];
          e += f * je[w * 16 + row];
          x += f * *(const f32x4*)(jo + (w * 16 + row) * D + dim);
        }
        int t, g;
        split(r, G, a.shape.inv_group, &t, &g);
        put(m * 16 + row, t, g, dim, x, mm, l, e);
      }
    }
  }
  if (u.parts == 1) return;
  if (KW == 1) { if (tid == 0) a.units[u.slot0 + u.part] = u; return; }      // joined by the next launch

  // Few rows: the unit's last part to get here joins them, in their order whichever it is.  Each load is waited for some microseconds, so
  // those of several parts are asked for at once.
  __shared__ int last;
  wait_vector_memory();
  __syncthreads();
  if (tid == 0) last = __hip_atomic_fetch_add(a.tickets + u.slot0, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == u.parts - 1;
  __syncthreads();
  if (!last) return;
  if (tid == 0) st_dev(a.tickets + u.slot0, 0);
  constexpr int AT_ONCE = 8;
  const int row0 = u.row_tile << a.shape.rows_shift, n_rows = min(rows - row0, 1 << a.shape.rows_shift);
  for (int i = tid; i < n_rows * (D / 4); i += NT) {
    const int row = i / (D / 4), dim = i % (D / 4) * 4;
    const int64_t rec0 = ((int64_t)u.slot0 << a.shape.rows_shift) + row;
    Joined x;
    for (int p0 = 0; p0 < u.parts; p0 += AT_ONCE) {
      float2 ml[AT_ONCE], lo[AT_ONCE], hi[AT_ONCE];
      float e[AT_ONCE];
#pragma unroll
      for (int p = 0; p < AT_ONCE; ++p) {
        const int64_t rec = rec0 + ((int64_t)min(p0 + p, u.parts - 1) << a.shape.rows_shift);
        const uint64_t* from = (const uint64_t*)(a.part_o + rec * D + dim);
        e[p] = a.lse ? ld_dev(a.part_e + rec) : 0.f;
        ml[p] = ld_dev64((const uint64_t*)(a.part_ml + rec)); lo[p] = ld_dev64(from); hi[p] = ld_dev64(from + 1);
      }
#pragma unroll
      for (int p = 0; p < AT_ONCE; ++p) if (p0 + p < u.parts) x.add(ml[p], e[p], f32x4{lo[p].x, lo[p].y, hi[p].x, hi[p].y});
    }
    int t, g;
    split(row0 + row, G, a.shape.inv_group, &t, &g);
    put_row<E, D>(c, a, u, t, g, dim, x.o, x.m, x.l, x.e);
  }
}

// The parts of units of many rows, joined: a workgroup a record, which takes its share of its unit's rows.  Bound by the records' bytes, which are in the
// L2 for the most part: 7 us after the two chunks of 2048 (8.7 MB from memory), 5 after the 64 trees.
constexpr int JOIN_NT = 256;
template <typename E, int D>
__global__ __launch_bounds__(JOIN_NT) void k_attend_join(CacheView c, AttendArgs a) {
  if ((int)blockIdx.x >= *a.n_records) return;
  const Unit u = a.units[blockIdx.x];
  const int G = a.shape.group, row0 = u.row_tile << a.shape.rows_shift, n_rows = min(u.n_new * G - row0, 1 << a.shape.rows_shift);
  const int each = div_up(n_rows, u.parts), first = min(u.part * each, n_rows), end = min(first + each, n_rows);
  for (int i = threadIdx.x; i < (end - first) * (D / 4); i += JOIN_NT) {
    const int row = first + i / (D / 4), dim = i % (D / 4) * 4;
    const int64_t rec0 = ((int64_t)u.slot0 << a.shape.rows_shift) + row;
    Joined x;
#pragma unroll 4
    for (int p = 0; p < u.parts; ++p) {
      const int64_t rec = rec0 + ((int64_t)p << a.shape.rows_shift);
      x.add(a.part_ml[rec], a.lse ? a.part_e[rec] : 0.f, *(const f32x4*)(a.part_o + rec * D + dim));
    }
    int t, g;
    split(row0 + row, G, a.shape.inv_group, &t, &g);
    put_row<E, D>(c, a, u, t, g, dim, x.o, x.m, x.l, x.e);
  }
}

}  // namespace c2t
