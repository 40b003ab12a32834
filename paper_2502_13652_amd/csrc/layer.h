// Host side of a layer's other entry points: norm, rotation on the way into the cache, attention over prompts.
#pragma once
#include "verify.h"
#include "k_append.h"
#include "k_norm.h"
#include "k_prompt.h"

namespace c2t {

inline int size_of(int dtype) { return dtype == C2T_F32 ? 4 : dtype == C2T_E4M3 ? 1 : 2; }
inline bool is_real(int dtype) { return dtype == C2T_F32 || dtype == C2T_BF16 || dtype == C2T_F16; }

// ---- norm ----
// A wavefront a row up to 1024 elements, a workgroup above, of as many threads as leave 8 or 16 elements each up to 16384 (4160 rows of 4096 27 us, with 256
// threads 28; 16384 rows of 8192 260 us, with 256 threads 270, with a wavefront 331).
typedef void (*NormKernel)(NormArgs);
struct NormShape { NormKernel fn; int threads, rows; };      // of a workgroup
template <typename T, bool E4, bool WHOLE> NormShape norm_kernel(int width) {
  if (width <= 512) return {k_rms_norm<T, E4, 64, 1, WHOLE>, 256, 4};
  if (width <= 1024) return {k_rms_norm<T, E4, 64, 2, WHOLE>, 256, 4};
  if (width <= 2048) return {k_rms_norm<T, E4, 256, 1, WHOLE>, 256, 1};
  if (width <= 4096) return {k_rms_norm<T, E4, 512, 1, WHOLE>, 512, 1};
  if (width <= 8192) return {k_rms_norm<T, E4, 512, 2, WHOLE>, 512, 1};
  if (width <= 16384) return {k_rms_norm<T, E4, 1024, 2, WHOLE>, 1024, 1};
  if (width <= 32768) return {k_rms_norm<T, E4, 1024, 4, WHOLE>, 1024, 1};
  return {k_rms_norm<T, E4, 1024, 8, WHOLE>, 1024, 1};
}
template <typename T> NormShape norm_kernel(int width, bool e4, bool whole) {
  return e4 ? (whole ? norm_kernel<T, true, true>(width) : norm_kernel<T, true, false>(width)) : whole ? norm_kernel<T, false, true>(width) : norm_kernel<T, false, false>(width);
}

// ---- append ----
inline bool pieces(int64_t stride) { return stride % 8 == 0; }
// Wavefronts that share a token: of calls of few tokens one for each pass over its heads, of others one for two passes, so that a pass's elements are on their way while another's
// are turned (8 prompts of 1000 to 2011, 48 heads of 128: 62 us, with one a token 66, with one a pass 79; 64 trees of 65 19, 23 and 25).
constexpr int APPEND_FEW_TOKENS = 256;
inline int append_parts(int64_t tokens, int passes) { return tokens < APPEND_FEW_TOKENS ? passes : std::max(passes / 2, 1); }

// ---- prompt ----
// Which kernel a call takes.  Tiles of 128 rows of a workgroup, whose wavefronts share the keys; or, where there are few of those and the prompts are long, tiles of 32 rows whose four
// wavefronts divide the keys: four times the workgroups, each a quarter of the way.  Both are known but for the lengths, of which the mean stands for all.  Width 128, shared and divided: one prompt of
// 2000 tokens, 4 heads over one, 37.6 and 21.2 us; of 8192, one head, 135 and 65, 4 over one 137 and 143; 4 of 500, 8 over one, 13.6 and 16.3; one of 200, 32 over 8, 8.5 and 7.9, of 350 11.5 and 13.2.
// Width 64, of which two workgroups that divide fit a CU: 32 and 14; 116 and 42, 119 and 72; 11.9 and 7.6; 7.5 and 5.7, 10.0 and 6.9, of 1000 19.7 and 17.2, of 1500 27.1 and 26.8, of 2000 35 and 41.
// Of width 256, whose tiles hardly fit in LDS four times, the keys are never divided.
typedef void (*PromptKernel)(const int32_t*, int32_t, int32_t, int32_t, int32_t, float, float, PromptArgs);
enum { PROMPT_MANY, PROMPT_SOME, PROMPT_DIVIDED };
constexpr int PROMPT_KEYS = 4;                               // wavefronts that divide the keys
inline int prompt_build(int64_t tiles, int64_t rows, int64_t sequences, int head_dim) {        // tiles: of 128 rows, of all heads
  const int64_t length = rows / sequences;
  if (head_dim <= 128 && tiles <= 4096 && tiles * tiles <= (head_dim == 64 ? 72 : 20) * length) return PROMPT_DIVIDED;
  // Width 128, up to as many tiles as workgroups fit the card by three: two a CU with tiles of 64 keys (one prompt of 3000 tokens, 32 heads over 8, 78 us, by three with tiles of 32 88; of
  // 1000 22.8 and 26.4); with more tiles three hide each other's start and end (64 prompts of up to 2000 856 and 806).
  return head_dim == 128 && tiles <= 3 * 256 ? PROMPT_SOME : PROMPT_MANY;
}
template <typename E, bool LSE> PromptKernel prompt_kernel(int head_dim, int build) {
  if (build == PROMPT_DIVIDED) return head_dim == 64 ? k_prompt<E, 64, 64, 1, PROMPT_KEYS, 2, LSE> : k_prompt<E, 128, 128, 1, PROMPT_KEYS, 1, LSE>;
  if (build == PROMPT_SOME) return k_prompt<E, 128, 128, 2, 1, 2, LSE>;
  return head_dim == 64 ? k_prompt<E, 64, 64, 2, 1, 4, LSE> : head_dim == 128 ? k_prompt<E, 128, 128, 1, 1, 3, LSE> : k_prompt<E, 256, 128, 2, 1, 2, LSE>;
}
template <typename E> PromptKernel prompt_kernel(int head_dim, int build, bool lse) { return lse ? prompt_kernel<E, true>(head_dim, build) : prompt_kernel<E, false>(head_dim, build); }
constexpr int64_t MAX_PROMPT_STRIDE = 1 << 24;

}  // namespace c2t

extern "C" {

int c2t_rms_norm(const c2t_norm* n, void* stream) {
  if (!n || n->rows < 0 || n->width <= 0) return C2T_ERR_INVALID_ARG;
  if (!is_real(n->dtype) || (n->weight_dtype != n->dtype && n->weight_dtype != C2T_F32) || (n->out_dtype != n->dtype && n->out_dtype != C2T_E4M3))
    return C2T_ERR_INVALID_ARG;
  const bool e4 = n->out_dtype == C2T_E4M3;
  if (!n->x || !n->weight || !n->out || (n->residual != nullptr) != (n->residual_out != nullptr) || e4 != (n->scales != nullptr)) return C2T_ERR_INVALID_ARG;
  if (n->residual && n->residual_dtype != n->dtype && n->residual_dtype != C2T_F32) return C2T_ERR_INVALID_ARG;
  if (!(n->eps > 0.f) || n->eps > 1e30f) return C2T_ERR_INVALID_ARG;
  if (n->width > C2T_MAX_NORM_WIDTH) return C2T_ERR_UNSUPPORTED;
  const bool whole = n->scale_block == n->width;
  if (e4 ? !whole && n->scale_block != 32 && n->scale_block != 64 && n->scale_block != 128 : n->scale_block != 0) return e4 && n->scale_block > 0 ? C2T_ERR_UNSUPPORTED : C2T_ERR_INVALID_ARG;
  const int es = size_of(n->dtype), rs = n->residual ? size_of(n->residual_dtype) : es, os = size_of(n->out_dtype), ws = size_of(n->weight_dtype);
  struct { const void* p; int64_t stride; int size; bool used; } of[] = {
      {n->x, n->x_stride, es, true}, {n->residual, n->residual_stride, rs, n->residual != nullptr}, {n->residual_out, n->residual_out_stride, rs, n->residual != nullptr},
      {n->out, n->out_stride, os, true}, {n->weight, n->width, ws, true}};
  bool aligned = n->width % 8 == 0;
  for (const auto& o : of) {
    if (!o.used) continue;
    if (o.stride < n->width) return C2T_ERR_INVALID_ARG;
    if (o.stride > MAX_STRIDE || (uintptr_t)o.p % o.size) return C2T_ERR_UNSUPPORTED;
    const int piece = o.size == 1 ? 8 : 16;
    aligned = aligned && (uintptr_t)o.p % piece == 0 && o.stride * o.size % piece == 0;
  }
  if (e4 && n->scales_stride < div_up(n->width, n->scale_block)) return C2T_ERR_INVALID_ARG;
  if (e4 && (n->scales_stride > MAX_STRIDE || (uintptr_t)n->scales % 4)) return C2T_ERR_UNSUPPORTED;
  if ((n->residual == n->residual_out && n->residual && n->residual_stride != n->residual_out_stride) ||
      (n->out == n->x && (n->out_stride != n->x_stride || os != es)) || (n->residual_out == n->x && (n->residual_out_stride != n->x_stride || rs != es)) ||
      n->out == n->residual_out)
    return C2T_ERR_INVALID_ARG;
  if (n->rows == 0) return C2T_OK;
  NormArgs a;
  a.x = (const char*)n->x; a.weight = (const char*)n->weight; a.residual = (const char*)n->residual; a.residual_out = (char*)n->residual_out; a.out = (char*)n->out;
  a.scales = n->scales;
  a.x_row = n->x_stride * es; a.residual_row = n->residual_stride * rs; a.residual_out_row = n->residual_out_stride * rs; a.out_row = n->out_stride * os;
  a.scales_row = n->scales_stride;
  a.rows = n->rows; a.width = n->width; a.block = whole ? 0 : n->scale_block;
  a.weight_f32 = n->weight_dtype == C2T_F32; a.residual_f32 = n->residual && n->residual_dtype == C2T_F32;
  a.eps = n->eps;
  const NormShape s = n->dtype == C2T_F32 ? norm_kernel<float>(n->width, e4, aligned) : n->dtype == C2T_BF16 ? norm_kernel<__bf16>(n->width, e4, aligned) : norm_kernel<_Float16>(n->width, e4, aligned);
  const int64_t blocks = div_up64(n->rows, s.rows);
  if (blocks * s.threads > MAX_BLOCKS * 256) return C2T_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(s.fn, dim3((unsigned)blocks), dim3((unsigned)s.threads), 0, (hipStream_t)stream, a);
  return hip_status();
}

int c2t_cache_append(const c2t_cache* c, const c2t_append* x, void* stream) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (!x || x->tokens < 0 || x->q_heads <= 0 || x->layer < 0 || x->layer >= c->layers || x->nodes < 0 || x->nodes > x->tokens) return C2T_ERR_INVALID_ARG;
  if (!x->q || !x->k || !x->v || !x->q_out || !x->turns || (x->nodes > 0) != (x->position != nullptr)) return C2T_ERR_INVALID_ARG;
  if (x->starts && (x->nodes > 0 || x->n_new)) return C2T_ERR_INVALID_ARG;
  if (x->q_heads % c->kv_heads != 0 || x->pairs <= 0 || x->pairs % 8 || x->pairs > c->head_dim / 2 || (x->neighbours != 0 && x->neighbours != 1)) return C2T_ERR_INVALID_ARG;
  if (!(x->magnitude > -1e30f && x->magnitude < 1e30f)) return C2T_ERR_INVALID_ARG;
  const int64_t q_row = (int64_t)x->q_heads * c->head_dim, k_row = (int64_t)c->kv_heads * c->head_dim;
  if (x->q_token_stride < q_row || x->q_out_token_stride < q_row || x->kv_token_stride < k_row || (x->k_out && x->k_out_token_stride < k_row)) return C2T_ERR_INVALID_ARG;
  const bool batches = !x->starts;
  if (batches && (x->q_batch_stride < 0 || x->kv_batch_stride < 0)) return C2T_ERR_INVALID_ARG;
  if (batches && c->batch > 1 && (x->q_out_batch_stride < q_row || (x->k_out && x->k_out_batch_stride < k_row))) return C2T_ERR_INVALID_ARG;   // one row in the place of several
  if ((x->q_out == x->q && (x->q_out_token_stride != x->q_token_stride || (batches && x->q_out_batch_stride != x->q_batch_stride))) ||
      (x->k_out == x->k && (x->k_out_token_stride != x->kv_token_stride || (batches && x->k_out_batch_stride != x->kv_batch_stride))))
    return C2T_ERR_INVALID_ARG;
  for (int64_t s : {x->q_token_stride, x->kv_token_stride, x->q_out_token_stride, x->k_out ? x->k_out_token_stride : 0, batches ? x->q_batch_stride : 0,
                    batches ? x->kv_batch_stride : 0, batches ? x->q_out_batch_stride : 0, batches && x->k_out ? x->k_out_batch_stride : 0})
    if (s > MAX_STRIDE || s < -MAX_STRIDE || !pieces(s)) return C2T_ERR_UNSUPPORTED;
  if (!aligned16(x->q) || !aligned16(x->k) || !aligned16(x->v) || !aligned16(x->q_out) || !aligned16(x->k_out) || (uintptr_t)x->turns % 8) return C2T_ERR_UNSUPPORTED;
  if (x->nodes > C2T_MAX_BUDGET || x->tokens > (1 << 24) || q_row > (1 << 24)) return C2T_ERR_UNSUPPORTED;
  if (x->tokens == 0) return C2T_OK;
  AppendArgs a;
  a.q = (const char*)x->q; a.k = (const char*)x->k; a.v = (const char*)x->v; a.q_out = (char*)x->q_out; a.k_out = (char*)x->k_out;
  a.q_batch = x->q_batch_stride * 2; a.q_token = x->q_token_stride * 2; a.kv_batch = x->kv_batch_stride * 2; a.kv_token = x->kv_token_stride * 2;
  a.q_out_batch = x->q_out_batch_stride * 2; a.q_out_token = x->q_out_token_stride * 2; a.k_out_batch = x->k_out_batch_stride * 2; a.k_out_token = x->k_out_token_stride * 2;
  a.n_new = x->n_new; a.starts = x->starts; a.position = x->position; a.turns = x->turns; a.magnitude = x->magnitude;
  a.slots = x->tokens; a.q_heads = x->q_heads; a.layer = x->layer; a.nodes = x->nodes; a.pairs = x->pairs; a.neighbours = x->neighbours;
  const int passes = div_up((x->q_heads + 2 * c->kv_heads) * (c->head_dim / 16), WAVE);       // of a wavefront over a token
  const int64_t rows = (int64_t)x->tokens * (batches ? c->batch : 1);
  a.parts = append_parts(rows, passes);
  if ((int64_t)x->tokens * a.parts > INT32_MAX) return C2T_ERR_UNSUPPORTED;
  const int64_t blocks = div_up64((int64_t)x->tokens * a.parts, CACHE_NT / WAVE);
  const unsigned batch = batches ? (unsigned)c->batch : 1u;
  if (blocks * batch > MAX_BLOCKS) return C2T_ERR_UNSUPPORTED;
  if (c->dtype == C2T_BF16) hipLaunchKernelGGL(k_cache_append<__bf16>, dim3((unsigned)blocks, batch), dim3(CACHE_NT), 0, (hipStream_t)stream, view_of(*c), a);
  else hipLaunchKernelGGL(k_cache_append<_Float16>, dim3((unsigned)blocks, batch), dim3(CACHE_NT), 0, (hipStream_t)stream, view_of(*c), a);
  return hip_status();
}

int c2t_prompt_attention(const c2t_prompt* p, void* stream) {
  if (!p || p->rows < 0 || p->sequences <= 0 || p->q_heads <= 0 || p->kv_heads <= 0 || p->q_heads % p->kv_heads != 0) return C2T_ERR_INVALID_ARG;
  if (p->dtype != C2T_BF16 && p->dtype != C2T_F16) return p->dtype == C2T_F32 ? C2T_ERR_UNSUPPORTED : C2T_ERR_INVALID_ARG;
  if (!p->q || !p->k || !p->v || !p->out || !p->starts || !(p->scale >= 0.f) || p->scale > 1e30f) return C2T_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return C2T_ERR_UNSUPPORTED;
  if (p->sequences > C2T_MAX_CACHE_BATCH || p->rows > (1 << 24) || (int64_t)p->rows * (p->q_heads / p->kv_heads) > (1 << 30)) return C2T_ERR_UNSUPPORTED;
  const int64_t q_row = (int64_t)p->q_heads * p->head_dim, k_row = (int64_t)p->kv_heads * p->head_dim;
  if (p->q_stride < q_row || p->out_stride < q_row || p->k_stride < k_row || p->v_stride < k_row) return C2T_ERR_INVALID_ARG;
  for (int64_t s : {p->q_stride, p->k_stride, p->v_stride, p->out_stride}) if (s > MAX_PROMPT_STRIDE || !pieces(s)) return C2T_ERR_UNSUPPORTED;
  if (!aligned16(p->q) || !aligned16(p->k) || !aligned16(p->v) || !aligned16(p->out) || (uintptr_t)p->lse % 4) return C2T_ERR_UNSUPPORTED;
  if (p->out == p->q || p->out == p->k || p->out == p->v) return C2T_ERR_INVALID_ARG;
  if (p->rows == 0) return C2T_OK;
  PromptArgs a;
  a.q = (const char*)p->q; a.k = (const char*)p->k; a.v = (const char*)p->v; a.out = (char*)p->out; a.lse = p->lse;
  a.q_row = p->q_stride * 2; a.k_row = p->k_stride * 2; a.v_row = p->v_stride * 2; a.out_row = p->out_stride * 2;
  const int group = p->q_heads / p->kv_heads;
  a.scale_log2e = std::max(p->scale, 1e-30f) * 1.44269504088896341f;       // (a masked score is -infinity times it: not 0)
  // each sequence has one tile at most that it does not fill
  const auto tiles = [&](int of) { return ((int64_t)p->rows * group / of + std::min(p->sequences, p->rows)) * p->kv_heads; };
  const int build = prompt_build(tiles(prompt_rows(1, false)), p->rows, p->sequences, p->head_dim), kw = build == PROMPT_DIVIDED ? PROMPT_KEYS : 1;
  const int64_t blocks = tiles(prompt_rows(kw, p->head_dim > 128));
  if (blocks > MAX_BLOCKS) return C2T_ERR_UNSUPPORTED;
  const PromptKernel fn = p->dtype == C2T_BF16 ? prompt_kernel<Bf16>(p->head_dim, build, p->lse != nullptr) : prompt_kernel<F16>(p->head_dim, build, p->lse != nullptr);
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3((unsigned)(64 * prompt_waves(kw))), 0, (hipStream_t)stream, p->starts, p->rows, p->sequences, p->kv_heads, group,
                     1.f / (float)p->kv_heads, 1.f / (float)group, a);
  return hip_status();
}

}  // extern "C"
