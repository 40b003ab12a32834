// Host side of the cache, attention and logits entry points: argument checks, scratch, launch shapes.
#pragma once
#include "../../include/c2t.h"
#include "k_adjust.h"
#include "k_attend.h"
#include "k_cache.h"

namespace c2t {

static_assert(C2T_MAX_CACHE_BATCH == RESERVE_MAX_B && C2T_MAX_PATH == MAX_PATH_TOKENS && C2T_MAX_BIAS == ADJUST_MAX_BIAS && C2T_MAX_BUDGET == ADJUST_MAX_NODES &&
              C2T_CACHE_POOL_EMPTY == CACHE_POOL_EMPTY && C2T_CACHE_ROW_FULL == CACHE_ROW_FULL && C2T_CACHE_INVALID == CACHE_INVALID && C2T_CACHE_SHARED == CACHE_SHARED,
              "limits of the C ABI and of the kernels must agree");

constexpr int64_t MAX_STRIDE = (int64_t)1 << 40;             // elements: products of strides and indices then stay in 64 bits

constexpr int64_t MAX_BLOCKS = (1 << 24) - 1;                // workgroups of 256 threads of a launch: fewer than 2^32 threads

inline bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }
inline int hip_status() { return hipGetLastError() == hipSuccess ? C2T_OK : C2T_ERR_HIP; }

inline int check_cache(const c2t_cache* c) {
  if (!c || !c->k || !c->v || !c->page_table || !c->length || !c->refcount || !c->status) return C2T_ERR_INVALID_ARG;
  if (c->batch <= 0 || c->layers <= 0 || c->pages <= 0 || c->kv_heads <= 0 || c->max_pages <= 0) return C2T_ERR_INVALID_ARG;
  if (c->dtype != C2T_BF16 && c->dtype != C2T_F16) return c->dtype == C2T_F32 ? C2T_ERR_UNSUPPORTED : C2T_ERR_INVALID_ARG;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256) return C2T_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return C2T_ERR_UNSUPPORTED;
  if (c->batch > C2T_MAX_CACHE_BATCH || c->kv_heads > 1024 || c->layers > 4096) return C2T_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_size > (1 << 30) || (int64_t)c->pages * c->page_size > INT32_MAX) return C2T_ERR_UNSUPPORTED;
  if (!aligned16(c->k) || !aligned16(c->v)) return C2T_ERR_UNSUPPORTED;
  return C2T_OK;
}

inline CacheView view_of(const c2t_cache& c) {
  CacheView v;
  v.k = (char*)c.k; v.v = (char*)c.v; v.table = c.page_table; v.length = c.length; v.refcount = c.refcount; v.status = c.status;
  v.batch = c.batch; v.layers = c.layers; v.pages = c.pages; v.max_pages = c.max_pages; v.kv_heads = c.kv_heads; v.head_dim = c.head_dim;
  v.page_shift = __builtin_ctz((unsigned)c.page_size);
  return v;
}

inline int reserve_cap(const c2t_cache& c) { return (int)std::min<int64_t>(c.pages, (int64_t)c.batch * c.max_pages); }
inline size_t reserve_bytes(const c2t_cache& c) { return ((size_t)2 * reserve_cap(c) + c.batch) * 4; }

// ---- attention ----
// Which kernel a launch of that many rows a cached head takes, 16 << build of them a tile: wavefronts that share rows and divide keys (16), or that divide rows.
//   width 64 and 128, up to 16 rows: 16 (one token behind 700 tokens 10.0 us, with 64 12.4; 64 of 300 to 8000 200 and 211; it loses where lengths are alike and
//   many: 64 trees of 4 behind 500 43 and 33).  Up to 32 rows, two tiles of 16 where there are few sequences (a tree of 8 behind 500 tokens 12.4 us, with 64 15.4),
//   64 otherwise (64 such trees 43 and 35).  Width 256: never 16 (19 trees of 9 behind up to 3038 tokens 46 us, with 64 30; 5 tokens 14.7 and 14.1).
//   Up to 64 rows: 64 (64 trees of 16 behind 2000 109 us, with 128 108; width 256, 4 of them behind 4000, 38 and 53); more: 128 (64 trees of 32 158 and 121).
enum { AB_ROWS_16 = 0, AB_ROWS_64 = 2, AB_ROWS_128 = 3 };
inline int attend_build(int64_t rows, int head_dim, int64_t heads) {       // heads: cached heads of all sequences
  if (head_dim <= 128 && (rows <= 16 || (rows <= 32 && heads < 256))) return AB_ROWS_16;
  return rows <= 64 ? AB_ROWS_64 : AB_ROWS_128;
}
typedef void (*AttendKernel)(CacheView, AttendArgs);
template <typename E, int D, bool NODES> AttendKernel attend_kernel(int build) {
  constexpr int KB = D > 128 ? 2 : 4;
  if constexpr (D <= 128) if (build == AB_ROWS_16) return k_attend<E, D, 1, 1, 4, 2, 2, NODES>;
  return build == AB_ROWS_64 ? k_attend<E, D, 1, 4, 1, KB, 2, NODES> : k_attend<E, D, 2, 4, 1, KB, (D > 128 ? 1 : 2), NODES>;
}
template <typename E, bool NODES> AttendKernel attend_kernel(int build, int head_dim) {
  return head_dim == 64 ? attend_kernel<E, 64, NODES>(build) : head_dim == 128 ? attend_kernel<E, 128, NODES>(build) : attend_kernel<E, 256, NODES>(build);
}
template <typename E> AttendKernel attend_kernel(int build, int head_dim, bool nodes) {
  return nodes ? attend_kernel<E, true>(build, head_dim) : attend_kernel<E, false>(build, head_dim);
}
template <typename E> AttendKernel join_kernel(int head_dim) {
  return head_dim == 64 ? k_attend_join<E, 64> : head_dim == 128 ? k_attend_join<E, 128> : k_attend_join<E, 256>;
}
constexpr int MAX_RUN = 8;                                   // a chunk of 2048 463 us, in runs of one 472; 64 trees of 65 214 and 227
constexpr int MAX_TARGET_SHIFT = 10, MAX_PARTS_ROWS = 64;
// 32 rows a cached head of one sequence behind 32000 tokens 31 us, with 256 KiB 39, with 64 45; of 16 rows 30, 33, 45; of 16 rows of a single cached head 28, 24, 41.
constexpr int64_t JOIN_BYTES = 128 << 10;
struct AttendPlan { AttendShape shape; int build, records; int64_t units, items; size_t n_records, units_at, part_o, part_ml, part_e, total; };

// Sizes of a call alone: the workspace must not depend on what is on the device.
inline int attend_plan(const c2t_cache& c, const c2t_attention& a, AttendPlan* p) {
  if (a.tokens <= 0 || a.q_heads <= 0 || a.nodes < 0 || a.nodes > a.tokens) return C2T_ERR_INVALID_ARG;
  if (a.q_heads % c.kv_heads != 0) return C2T_ERR_INVALID_ARG;
  if (a.nodes > C2T_MAX_BUDGET || (int64_t)a.tokens * a.q_heads > (1 << 30)) return C2T_ERR_UNSUPPORTED;
  const int group = a.q_heads / c.kv_heads;
  const int64_t rows = (int64_t)a.tokens * group;
  p->build = attend_build(rows, c.head_dim, (int64_t)c.batch * c.kv_heads);
  p->shape.slots = a.tokens; p->shape.group = group; p->shape.inv_group = 1.f / (float)group;
  const bool by_keys = p->build == AB_ROWS_16;
  p->shape.rows_shift = 4 + p->build;
  p->shape.keys_shift = by_keys || c.head_dim > 128 ? 5 : 6;
  p->units = (int64_t)c.batch * c.kv_heads * row_tiles(p->shape, a.tokens);
  // Parts: enough for two workgroups a CU (as many are resident of the builds of width 128; of width 64 two to four, of width 256 one or two: one number serves
  // them all), since parts and their records cost more than what an even end saves: a chunk of 2048 466 us,
  // with twice the parts 514; 64 trees of 65 205 and 244; one token behind 32000 32 and 43.  Many units of few rows go twice round: 64 tokens of 300
  // to 8000 keys 202 us, with half of the parts 223; 32 tokens behind 4000 the other way, 105 and 100.
  p->shape.target_shift = by_keys && p->units >= 512 ? MAX_TARGET_SHIFT : MAX_TARGET_SHIFT - 1;
  // The shortest part: of many rows the longer, the more units share the chip without parts, since a join is a launch and a trip of all rows
  // through memory.  256 units of 5 tiles 24 us unsplit, 35 in parts of 4; 5 units of up to 59 tiles 19 us in parts of 4 and 37 in parts of 16.
  p->shape.min_per = by_keys ? 8 : (int)std::min<int64_t>(std::max<int64_t>(p->units / 16, 4), 16);
  p->shape.run = std::min(row_tiles(p->shape, a.tokens), MAX_RUN);
  p->items = workgroups_for(p->shape, p->units + (1 << p->shape.target_shift));
  if (p->items > MAX_BLOCKS) return C2T_ERR_UNSUPPORTED;
  // records of a unit: as many as its join reads in a few microseconds, by one workgroup where it has few rows, by one a record where it has more
  const int64_t record = std::min(rows, (int64_t)1 << p->shape.rows_shift) * c.head_dim * 4;
  p->shape.max_parts = by_keys ? (int)std::min<int64_t>(std::max<int64_t>(JOIN_BYTES / record, 2), 1024) : MAX_PARTS_ROWS;
  const size_t records = (size_t)2 << p->shape.target_shift, rows_of_them = records << p->shape.rows_shift;
  static_assert((2 << MAX_TARGET_SHIFT) * 4 == C2T_ATTENTION_COUNTERS, "one a record");
  p->n_records = C2T_ATTENTION_COUNTERS;                     // behind the counters, whose place is the same whatever the call's sizes
  p->units_at = p->n_records + 256;
  p->part_o = p->units_at + (sizeof(Unit) << (MAX_TARGET_SHIFT + 1));
  p->records = (int)records;
  p->part_ml = p->part_o + rows_of_them * c.head_dim * 4;
  p->part_e = p->part_ml + rows_of_them * 8;
  p->total = p->part_e + rows_of_them * 4;
  return C2T_OK;
}

// The checks that both entry points share; row and batch strides in elements become bytes.
inline int check_adjust(AdjustArgs& a, int dtype, int64_t in_stride, int64_t out_stride) {
  const int esz = dtype == C2T_BF16 ? 2 : 4;
  if (!a.in || !a.out || a.batch <= 0 || a.rows <= 0 || a.vocab <= 0 || !a.n_rows) return C2T_ERR_INVALID_ARG;
  if (dtype != C2T_F32 && dtype != C2T_BF16) return dtype == C2T_F16 ? C2T_ERR_UNSUPPORTED : C2T_ERR_INVALID_ARG;
  if (in_stride < a.vocab || out_stride < a.vocab) return C2T_ERR_INVALID_ARG;
  if (a.in == a.out && in_stride != out_stride) return C2T_ERR_INVALID_ARG;
  if (in_stride > MAX_STRIDE || out_stride > MAX_STRIDE) return C2T_ERR_UNSUPPORTED;
  a.in_row = in_stride * esz; a.out_row = out_stride * esz;
  a.in_batch = a.in_row * a.rows; a.out_batch = a.out_row * a.rows;
  if (!aligned16(a.in) || !aligned16(a.out) || a.in_row % 16 || a.out_row % 16) return C2T_ERR_UNSUPPORTED;
  if (a.batch > 65535 || a.rows > 65535 || a.vocab > (1 << 30)) return C2T_ERR_UNSUPPORTED;
  return C2T_OK;
}

// One round of two a CU: each workgroup makes its sequence's lists anew.  4 sequences of 65 rows of 128256: 25 us, with 1024 28, with 256 28, with 4096
// 36; one sequence of 32000 15 whatever it is; 64 of 128253, more than either in any case, 372, in four times as many 364.
constexpr int ADJUST_WORKGROUPS = 512;
inline int fill_adjust(AdjustArgs& a, const c2t_adjustments* t) {
  if (!t) return C2T_ERR_INVALID_ARG;
  if (t->tokens && (!t->n_tokens || t->token_stride <= 0)) return C2T_ERR_INVALID_ARG;
  if ((t->bias != nullptr) != (t->bias_tokens != nullptr) || (t->bias && t->bias_stride <= 0)) return C2T_ERR_INVALID_ARG;
  if (t->allowed && (t->allowed_row_stride < 0 || t->allowed_batch_stride < 0)) return C2T_ERR_INVALID_ARG;
  if (t->allowed_row_stride > MAX_STRIDE || t->allowed_batch_stride > MAX_STRIDE) return C2T_ERR_UNSUPPORTED;
  if (t->token_stride > ADJUST_MAX_CONTEXT || (t->bias && t->bias_stride > C2T_MAX_BIAS)) return C2T_ERR_UNSUPPORTED;
  a.tokens = t->tokens; a.token_stride = t->token_stride; a.n_tokens = t->n_tokens; a.n_prompt = t->n_prompt;
  a.repetition = t->repetition; a.frequency = t->frequency; a.presence = t->presence;
  a.bias_token = t->bias_tokens; a.bias = t->bias; a.n_bias = t->n_bias; a.bias_stride = t->bias_stride;
  a.allowed = t->allowed; a.allowed_row = t->allowed_row_stride; a.allowed_batch = t->allowed_batch_stride;
  return C2T_OK;
}

inline int launch_adjust(AdjustArgs a, int dtype, hipStream_t s) {
  const int stretches = div_up(a.vocab, ADJUST_STRETCH), batch = dtype == C2T_BF16 ? ADJUST_ROWS<__bf16> : ADJUST_ROWS<float>;
  const int64_t groups = div_up64(ADJUST_WORKGROUPS, (int64_t)stretches * a.batch);    // of rows
  a.rows_each = div_up(div_up(a.rows, (int)std::min<int64_t>(groups, a.rows)), batch) * batch;
  a.sparse = a.in == a.out && !a.allowed;
  const dim3 grid((unsigned)stretches, (unsigned)div_up(a.rows, a.rows_each), (unsigned)a.batch);
  if (dtype == C2T_BF16) hipLaunchKernelGGL(k_adjust<__bf16>, grid, dim3(ADJUST_NT), 0, s, a);
  else hipLaunchKernelGGL(k_adjust<float>, grid, dim3(ADJUST_NT), 0, s, a);
  return hip_status();
}

}  // namespace c2t

using namespace c2t;

extern "C" {

int c2t_cache_workspace_bytes(const c2t_cache* c, size_t* out) {
  if (!out) return C2T_ERR_INVALID_ARG;
  const int rc = check_cache(c);
  if (rc) return rc;
  *out = reserve_bytes(*c);
  return C2T_OK;
}

int c2t_cache_reserve(const c2t_cache* c, const int32_t* n_new, void* ws, size_t bytes, void* stream) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (!n_new) return C2T_ERR_INVALID_ARG;
  if (!ws || (uintptr_t)ws % 256 != 0 || bytes < reserve_bytes(*c)) return C2T_ERR_WORKSPACE;
  const CacheView v = view_of(*c);
  ReserveScratch x;
  x.cap = reserve_cap(*c);
  x.fresh = (int32_t*)ws; x.given_up = x.fresh + x.cap; x.copied = x.given_up + x.cap;
  hipLaunchKernelGGL(k_cache_reserve, dim3(1), dim3(RESERVE_NT), 0, (hipStream_t)stream, v, n_new, x);
  hipLaunchKernelGGL(k_cache_copy_partial, dim3((unsigned)(c->layers * 2 * c->kv_heads), (unsigned)c->batch), dim3(CACHE_NT), 0, (hipStream_t)stream, v, x);
  return hip_status();
}

int c2t_cache_write(const c2t_cache* c, int32_t layer, const void* k, const void* v, int64_t batch_stride, int64_t token_stride, int32_t tokens,
                    const int32_t* n_new, void* stream) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (!k || !v || layer < 0 || layer >= c->layers || tokens <= 0) return C2T_ERR_INVALID_ARG;
  const int64_t row = (int64_t)c->kv_heads * c->head_dim;
  if (token_stride < row || batch_stride < 0) return C2T_ERR_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v) || batch_stride % 8 || token_stride % 8 || tokens > (1 << 24) || batch_stride > MAX_STRIDE || token_stride > MAX_STRIDE) return C2T_ERR_UNSUPPORTED;
  const NewTokens x{(const char*)k, (const char*)v, batch_stride * 2, token_stride * 2, n_new, tokens};
  const int64_t blocks = div_up64((int64_t)tokens * (row / 8), CACHE_NT);
  if (blocks > MAX_BLOCKS) return C2T_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(k_cache_write, dim3((unsigned)blocks, (unsigned)c->batch), dim3(CACHE_NT), 0, (hipStream_t)stream, view_of(*c), layer, x);
  return hip_status();
}

int c2t_cache_commit(const c2t_cache* c, const int32_t* path, int32_t path_stride, const int32_t* n_path, void* stream) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (!path || !n_path || path_stride <= 0) return C2T_ERR_INVALID_ARG;
  if (path_stride > C2T_MAX_PATH) return C2T_ERR_UNSUPPORTED;
  const CacheView v = view_of(*c);
  const Path p{path, n_path, path_stride};
  const int64_t columns = (int64_t)c->layers * 2 * c->kv_heads * (c->head_dim / 8);
  hipLaunchKernelGGL(k_cache_commit, dim3((unsigned)div_up64(columns, CACHE_NT), (unsigned)c->batch), dim3(CACHE_NT), 0, (hipStream_t)stream, v, p);
  hipLaunchKernelGGL(k_cache_commit_lengths, dim3((unsigned)div_up(c->batch, CACHE_NT / WAVE)), dim3(CACHE_NT), 0, (hipStream_t)stream, v, p);
  return hip_status();
}

int c2t_cache_truncate(const c2t_cache* c, const int32_t* new_length, int32_t keep, void* stream) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (keep < 0) return C2T_ERR_INVALID_ARG;
  hipLaunchKernelGGL(k_cache_truncate, dim3((unsigned)c->batch), dim3(CACHE_NT), 0, (hipStream_t)stream, view_of(*c), new_length, keep);
  return hip_status();
}

int c2t_cache_fork(const c2t_cache* c, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (!src || !dst || n <= 0) return C2T_ERR_INVALID_ARG;
  if (n > C2T_MAX_CACHE_BATCH) return C2T_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(k_cache_fork, dim3((unsigned)n), dim3(CACHE_NT), 0, (hipStream_t)stream, view_of(*c), src, dst, n);
  return hip_status();
}

int c2t_attention_workspace_bytes(const c2t_cache* c, const c2t_attention* a, size_t* out) {
  if (!a || !out) return C2T_ERR_INVALID_ARG;
  int rc = check_cache(c);
  AttendPlan p;
  if (!rc) rc = attend_plan(*c, *a, &p);
  if (rc) return rc;
  *out = p.total;
  return C2T_OK;
}

int c2t_cache_attention(const c2t_cache* c, const c2t_attention* a, void* ws, size_t bytes, void* stream) {
  if (!a) return C2T_ERR_INVALID_ARG;
  int rc = check_cache(c);
  AttendPlan p;
  if (!rc) rc = attend_plan(*c, *a, &p);
  if (rc) return rc;
  const int64_t row = (int64_t)a->q_heads * c->head_dim;
  if (!a->q || !a->out || a->layer < 0 || a->layer >= c->layers || (a->nodes > 0) != (a->mask != nullptr)) return C2T_ERR_INVALID_ARG;
  if (a->q_token_stride < row || a->out_token_stride < row || a->q_batch_stride < 0 || a->out_batch_stride < 0) return C2T_ERR_INVALID_ARG;
  if (!(a->scale >= 0.f) || a->scale > 1e30f) return C2T_ERR_INVALID_ARG;
  for (int64_t stride : {a->q_token_stride, a->q_batch_stride, a->out_token_stride, a->out_batch_stride}) if (stride > MAX_STRIDE) return C2T_ERR_UNSUPPORTED;
  if (!aligned16(a->q) || !aligned16(a->out) || a->q_batch_stride % 8 || a->q_token_stride % 8 || a->out_batch_stride % 8 || a->out_token_stride % 8)
    return C2T_ERR_UNSUPPORTED;
  if (c->batch > 1 && a->out_batch_stride < row) return C2T_ERR_INVALID_ARG;       // one row in the place of several
  if (!ws || (uintptr_t)ws % 256 != 0 || bytes < p.total) return C2T_ERR_WORKSPACE;
  AttendArgs g;
  g.q = (const char*)a->q; g.out = (char*)a->out; g.lse = a->lse;
  g.q_batch = a->q_batch_stride * 2; g.q_token = a->q_token_stride * 2; g.out_batch = a->out_batch_stride * 2; g.out_token = a->out_token_stride * 2;
  g.n_new = a->n_new; g.mask = a->mask; g.nodes = a->nodes; g.chain = a->tokens - a->nodes; g.layer = a->layer;
  g.scale_log2e = std::max(a->scale, 1e-30f) * 1.44269504088896341f;       // (a masked score is -infinity times it: not 0)
  g.tickets = (int32_t*)ws; g.n_records = (int32_t*)((char*)ws + p.n_records); g.units = (Unit*)((char*)ws + p.units_at);
  g.part_o = (float*)((char*)ws + p.part_o); g.part_ml = (float2*)((char*)ws + p.part_ml); g.part_e = (float*)((char*)ws + p.part_e);
  g.shape = p.shape;
  const CacheView v = view_of(*c);
  const bool bf16 = c->dtype == C2T_BF16;
  const AttendKernel fn = bf16 ? attend_kernel<Bf16>(p.build, c->head_dim, a->nodes > 0) : attend_kernel<F16>(p.build, c->head_dim, a->nodes > 0);
  hipLaunchKernelGGL(fn, dim3((unsigned)p.items), dim3(256), 0, (hipStream_t)stream, v, g);
  if (p.build >= AB_ROWS_64)
    hipLaunchKernelGGL(bf16 ? join_kernel<Bf16>(c->head_dim) : join_kernel<F16>(c->head_dim), dim3((unsigned)p.records), dim3(JOIN_NT), 0, (hipStream_t)stream, v, g);
  return hip_status();
}

int c2t_stream_capture_id(void* stream, uint64_t* out) {
  if (!out) return C2T_ERR_INVALID_ARG;
  *out = 0;
  if (!stream) return C2T_OK;                                // (the default stream cannot be captured)
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  unsigned long long id = 0;
  if (hipStreamGetCaptureInfo((hipStream_t)stream, &status, &id) != hipSuccess) { (void)hipGetLastError(); return C2T_ERR_HIP; }
  if (status == hipStreamCaptureStatusActive) *out = id;
  return C2T_OK;
}

int c2t_adjust_tree_logits(const c2t_adjustments* t, int32_t batch, int32_t vocab, int32_t nodes, int32_t dtype, const int32_t* tree_tokens,
                           const int32_t* tree_parent, const int32_t* n_nodes, const void* logits, int64_t row_stride, void* out, int64_t out_row_stride,
                           void* stream) {
  AdjustArgs a{};
  const int rc = fill_adjust(a, t);
  if (rc) return rc;
  if (nodes < 0 || !n_nodes || (nodes > 0 && (!tree_tokens || !tree_parent))) return C2T_ERR_INVALID_ARG;
  if (nodes > C2T_MAX_BUDGET) return C2T_ERR_UNSUPPORTED;
  a.in = (const char*)logits; a.out = (char*)out;
  a.batch = batch; a.rows = 1 + nodes; a.vocab = vocab;
  a.n_rows = n_nodes; a.more_rows = 1;
  a.node_token = nodes > 0 ? tree_tokens : nullptr; a.node_parent = tree_parent; a.nodes = nodes; a.n_nodes = n_nodes;
  const int bad = check_adjust(a, dtype, row_stride, out_row_stride);
  return bad ? bad : launch_adjust(a, dtype, (hipStream_t)stream);
}

}  // extern "C"
