// Penalties for repeated tokens, biases and a grammar's mask on logits rows that belong to the nodes of a tree.
//
//   a = times the token occurs in the sequence's context and on the row's path, o = the same without the prompt
//   y = x;  a > 0: y = x > 0 ? x / r : x r;   y -= alpha o + beta [o > 0];   y += sum of the token's biases;   not allowed: y = -inf
//
// A workgroup has a stretch of the vocabulary and some of a sequence's rows.  It counts the context's tokens of its stretch in
// LDS once and lists the tokens that anything is done to: a few hundred of 4096 at most usually.  Rows then pass through LDS,
// a few at a time: in as they are, the listed tokens changed in place (each by a thread of its own, so no lane waits for
// another's), and out with the mask.  In place and without a mask only the listed tokens are read and written.
//
// Bound by the rows' bytes: 64 sequences, 65 rows of 128256 bf16 logits each, contexts of 4000 and a mask: 448 us, 4.9 TB/s read and written, what a large
// copy gets (4.8); without a mask 430.  61 rows of 32000 fp32 logits of one sequence: 9.7 us, the launch and the lists.
// The draft's rows in place, contexts of 2000: 64 sequences of 16 rows of 128256 68 us (with a mask 95, into another buffer 105), 256 of 32 rows of 152064 714 (970, 954);
// 10 rows of 32000 of one sequence 10.5, the host's call.
#pragma once
#include "k_common.h"
#include "k_paged.h"

namespace c2t {

struct AdjustArgs {
  const char* in; char* out;               // [batch][rows][..]: strides in bytes
  int64_t in_row, in_batch, out_row, out_batch;
  int32_t batch, rows, vocab;              // rows of a sequence at most
  const int32_t* n_rows; int32_t more_rows;// [batch] + more_rows of them are live
  const int32_t* row_node;                 // [batch][rows] node of each row, -1: the root; null: node row - 1
  const int32_t* node_token; const int32_t* node_parent; int32_t nodes;      // [batch][nodes], a node's parent before it
  const int32_t* n_nodes;                  // [batch]
  const int32_t* tokens; int64_t token_stride; const int32_t* n_tokens; const int32_t* n_prompt;
  const float* repetition; const float* frequency; const float* presence;
  const int32_t* bias_token; const float* bias; const int32_t* n_bias; int32_t bias_stride;
  const uint32_t* allowed; int64_t allowed_row, allowed_batch;               // strides in words
  int32_t rows_each;                       // rows of a workgroup
  int32_t sparse;                          // in place and without a mask
};

template <typename X> struct Bits;
template <> struct Bits<float> { typedef uint32_t U; };
template <> struct Bits<__bf16> { typedef uint16_t U; };

constexpr int ADJUST_NT = 512;
constexpr int ADJUST_MAX_NODES = 1024, ADJUST_MAX_BIAS = 1024;
constexpr int ADJUST_STRETCH = 4096;       // tokens of a workgroup's stretch
constexpr int ADJUST_BATCH_CHUNKS = 4;     // 16-byte chunks a thread of the rows that are in LDS at once
// a token's word: flags, times in the output's part of the context (of a biased token: its first entry, which has the times and the sum of its biases)
constexpr uint32_t IN_PROMPT = 0x80000000u, BIASED = 0x40000000u, IN_TREE = 0x20000000u, TIMES = 0x1fffffffu;
constexpr int ADJUST_MAX_CONTEXT = 1 << 28;
constexpr int ADJUST_PATH_WORDS = 1024;    // 32 rows of a tree whose nodes' tokens all lie in the stretch, and hundreds usually

template <typename X> constexpr int ADJUST_ROWS = ADJUST_BATCH_CHUNKS * ADJUST_NT * (16 / (int)sizeof(X)) / ADJUST_STRETCH;     // rows in LDS at once

template <typename X>
__global__ __launch_bounds__(ADJUST_NT) void k_adjust(AdjustArgs a) {
  constexpr int N = 16 / sizeof(X), CPR = ADJUST_STRETCH / N / ADJUST_NT, RB = ADJUST_ROWS<X>;
  typedef uint32_t U4 __attribute__((ext_vector_type(4)));
  static_assert(CPR * RB == ADJUST_BATCH_CHUNKS && CPR >= 1, "");
  __shared__ __align__(16) X row_lds[RB * ADJUST_STRETCH];
  __shared__ uint32_t word[ADJUST_STRETCH];
  __shared__ uint16_t touched[ADJUST_STRETCH];
  __shared__ int16_t node_parent[ADJUST_MAX_NODES], node_here[ADJUST_MAX_NODES];       // the node's place in here_token, -1: its token is not in the stretch
  __shared__ uint16_t here_token[ADJUST_MAX_NODES];
  __shared__ uint32_t on_path[ADJUST_PATH_WORDS];            // of some rows: places in here_token of the nodes on the row's path
  __shared__ int32_t bias_at[ADJUST_MAX_BIAS];               // place in the stretch, -1: not in it; then, of a token's first entry: its times
  __shared__ float bias_value[ADJUST_MAX_BIAS];              // of a token's first entry: the sum of all of its entries
  __shared__ int n_touched, n_here, n_bias_here;
  __shared__ uint16_t bias_here[ADJUST_MAX_BIAS];            // first entries of tokens of the stretch
  const int tid = threadIdx.x, b = blockIdx.z, v0 = blockIdx.x * ADJUST_STRETCH, n_words = min(ADJUST_STRETCH, a.vocab - v0);
  const int rows = min(max(a.n_rows[b] + a.more_rows, 0), a.rows);
  const int row0 = blockIdx.y * a.rows_each, row1 = min(row0 + a.rows_each, rows);
  if (row0 >= row1) return;
  const char* const in0 = a.in + b * a.in_batch + (int64_t)v0 * sizeof(X);
  char* const out0 = a.out + b * a.out_batch + (int64_t)v0 * sizeof(X);
  const uint8_t* const ok0 = a.allowed ? (const uint8_t*)(a.allowed + b * a.allowed_batch) + v0 / 8 : nullptr;

  // rows r .. r + RB - 1 of the stretch, a thread's chunks of them; what is behind the vocabulary is not ours
  U4 x[ADJUST_BATCH_CHUNKS];
  uint32_t ok[ADJUST_BATCH_CHUNKS];
  auto request = [&](int r) {
#pragma unroll
    for (int i = 0; i < ADJUST_BATCH_CHUNKS; ++i) {
      const int at = (i % CPR * ADJUST_NT + tid) * N, row = min(r + i / CPR, row1 - 1);
      x[i] = U4{0u, 0u, 0u, 0u}; ok[i] = 0xffu;
      if (at + N <= n_words) x[i] = *(const U4*)(in0 + row * a.in_row + (int64_t)at * sizeof(X));
      if (ok0 && at < n_words) ok[i] = (uint32_t)ok0[row * a.allowed_row * 4 + at / 8] >> (at % 8);
    }
  };
  if (!a.sparse) request(row0);

  for (int i = tid; i < ADJUST_STRETCH; i += ADJUST_NT) word[i] = 0u;
  if (tid == 0) { n_touched = 0; n_here = 0; n_bias_here = 0; }
  __syncthreads();
  const int n_nodes = a.node_token ? min(max(a.n_nodes[b], 0), a.nodes) : 0;
  for (int i = tid; i < n_nodes; i += ADJUST_NT) {
    const int p = a.node_parent[(int64_t)b * a.nodes + i], t = a.node_token[(int64_t)b * a.nodes + i] - v0;
    node_parent[i] = (int16_t)(p < i ? max(p, -1) : -1);     // (a path ends however the tree was made)
    const bool here = (uint32_t)t < (uint32_t)n_words;
    int place = -1;
    if (here) { place = append_place(&n_here); here_token[place] = (uint16_t)t; atomicOr(&word[t], IN_TREE); }
    node_here[i] = (int16_t)place;
  }
  const int n_ctx = a.tokens ? (int)min((int64_t)max(a.n_tokens[b], 0), a.token_stride) : 0, n_prompt = a.n_prompt ? a.n_prompt[b] : 0;
  for (int i = tid; i < n_ctx; i += ADJUST_NT) {
    const int t = a.tokens[(int64_t)b * a.token_stride + i] - v0;
    if ((uint32_t)t < (uint32_t)n_words) { if (i < n_prompt) atomicOr(&word[t], IN_PROMPT); else atomicAdd(&word[t], 1u); }
  }
  const int n_bias = a.bias ? min(max(a.n_bias ? a.n_bias[b] : a.bias_stride, 0), a.bias_stride) : 0;
  for (int i = tid; i < n_bias; i += ADJUST_NT) {
    const int t = a.bias_token[(int64_t)b * a.bias_stride + i] - v0;
    bias_at[i] = (uint32_t)t < (uint32_t)n_words ? t : -1;
  }
  __syncthreads();
  // biases of one token add up in the order in which they are listed, in the place of the first
  for (int i = tid; i < n_bias; i += ADJUST_NT) if (bias_at[i] >= 0) bias_here[append_place(&n_bias_here)] = (uint16_t)i;
  __syncthreads();
  const int n_listed = uniform(n_bias_here);
  bool is_first[ADJUST_MAX_BIAS / ADJUST_NT];
#pragma unroll
  for (int x = 0; x < ADJUST_MAX_BIAS / ADJUST_NT; ++x) {
    const int k = x * ADJUST_NT + tid;
    is_first[x] = false;
    if (k >= n_listed) continue;
    const int i = bias_here[k], t = bias_at[i];
    bool first = true, alone = true;
    for (int e = 0; e < n_listed; ++e) { const int j = bias_here[e]; if (bias_at[j] == t) { alone = alone && j == i; first = first && j >= i; } }
    float sum = a.bias[(int64_t)b * a.bias_stride + i];
    if (!alone) { sum = 0.f; for (int j = 0; j < n_bias; ++j) if (bias_at[j] == t) sum += a.bias[(int64_t)b * a.bias_stride + j]; }
    bias_value[i] = sum;
    is_first[x] = first;
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < ADJUST_MAX_BIAS / ADJUST_NT; ++x) {
    if (!is_first[x]) continue;
    const int i = bias_here[x * ADJUST_NT + tid], t = bias_at[i];
    bias_at[i] = (int32_t)(word[t] & TIMES);                 // (nobody else's from here on)
    word[t] = (word[t] & ~TIMES) | BIASED | (uint32_t)i;
  }
  __syncthreads();
  for (int i = tid; i < n_words; i += ADJUST_NT) if (word[i] != 0u) touched[append_place(&n_touched)] = (uint16_t)i;
  __syncthreads();

  const float rep = a.repetition ? a.repetition[b] : 1.f, freq = a.frequency ? a.frequency[b] : 0.f, pres = a.presence ? a.presence[b] : 0.f;
  const int n_list = uniform(n_touched), bit_words = div_up(uniform(n_here), 32);
  const int rows_marked = bit_words == 0 ? a.rows_each : max(ADJUST_PATH_WORDS / bit_words / RB, 1) * RB;     // rows that on_path holds at once, a multiple of RB
  // the paths of rows r, r + 1, ... as far as they are marked at once: one lane walks each
  auto mark_paths = [&](int r) {
    const int n = min(rows_marked, row1 - r);
    for (int i = tid; i < n * bit_words; i += ADJUST_NT) on_path[i] = 0u;
    __syncthreads();
    if (bit_words > 0) for (int i = tid; i < n; i += ADJUST_NT) {
      int node = a.row_node ? a.row_node[(int64_t)b * a.rows + r + i] : r + i - 1;
      if (node >= n_nodes) node = -1;
      while (node >= 0) {
        const int h = node_here[node];
        node = node_parent[node];
        if (h >= 0) on_path[i * bit_words + h / 32] |= 1u << (h % 32);
      }
    }
    __syncthreads();
  };
  // token t of the row that is `row` behind the first marked one, made of its logit; false: nothing is done to it
  auto adjusted = [&](int t, int row, float* y) {
    const uint32_t w = word[t];
    const int entry = (int)(w & TIMES);
    uint32_t times = w & BIASED ? (uint32_t)bias_at[entry] : w & TIMES;
    if (w & IN_TREE) {
      for (int k = 0; k < bit_words; ++k)
        for (uint32_t bits = on_path[row * bit_words + k]; bits; bits &= bits - 1u) times += here_token[k * 32 + __builtin_ctz(bits)] == t;
    }
    float z = *y;
    if (times != 0u || (w & IN_PROMPT)) z = z > 0.f ? z / rep : z * rep;
    if (times != 0u) z -= freq * (float)times + pres;
    if (w & BIASED) z += bias_value[entry];
    *y = z;
    return times != 0u || (w & (IN_PROMPT | BIASED)) != 0u;
  };

  if (a.sparse) {
    for (int r = row0; r < row1; r += rows_marked) {
      mark_paths(r);
      const int live = min(rows_marked, row1 - r);
      for (int row = 0; row < live; ++row)
        for (int i = tid; i < n_list; i += ADJUST_NT) {
          const int t = touched[i];
          X* at = (X*)(out0 + (r + row) * a.out_row) + t;
          float y = (float)*at;
          if (adjusted(t, row, &y)) *at = (X)y;
        }
      __syncthreads();
    }
    return;
  }
  int marked = row0;                                         // the first row that on_path holds
  mark_paths(row0);
  for (int r = row0; r < row1; r += RB) {
    const int live = min(RB, row1 - r);
    uint32_t ok_now[ADJUST_BATCH_CHUNKS];
#pragma unroll
    for (int i = 0; i < ADJUST_BATCH_CHUNKS; ++i) {
      const int at = (i % CPR * ADJUST_NT + tid) * N, row = i / CPR;
      if (at + N <= n_words) *(U4*)(row_lds + row * ADJUST_STRETCH + at) = x[i];
      else if (row < live) for (int j = at; j < n_words; ++j) row_lds[row * ADJUST_STRETCH + j] = ((const X*)(in0 + (r + row) * a.in_row))[j];
      ok_now[i] = ok[i];
    }
    if (r + RB < row1) request(r + RB);
    if (r - marked >= rows_marked) { marked = r; mark_paths(r); }
    __syncthreads();
    for (int i = tid; i < n_list * live; i += ADJUST_NT) {
      const int row = i / n_list, t = touched[i - row * n_list];
      X* at = row_lds + row * ADJUST_STRETCH + t;
      float y = (float)*at;
      if (adjusted(t, r - marked + row, &y)) *at = (X)y;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ADJUST_BATCH_CHUNKS; ++i) {
      const int at = (i % CPR * ADJUST_NT + tid) * N, row = i / CPR;
      if (row >= live || at >= n_words) continue;
      U4 y = *(const U4*)(row_lds + row * ADJUST_STRETCH + at);
      constexpr uint32_t ALL = (1u << N) - 1u;
      if ((ok_now[i] & ALL) != ALL) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (sizeof(X) == 4) y[j] = ok_now[i] >> j & 1u ? y[j] : 0xff800000u;
          else y[j] = (ok_now[i] >> (2 * j) & 1u ? y[j] & 0xffffu : 0xff80u) | (ok_now[i] >> (2 * j + 1) & 1u ? y[j] & 0xffff0000u : 0xff800000u);
        }
      }
      char* to = out0 + (r + row) * a.out_row + (int64_t)at * sizeof(X);
      if (at + N <= n_words) *(U4*)to = y;
      else for (int j = 0; j < n_words - at; ++j) ((X*)to)[j] = sizeof(X) == 4 ? __builtin_bit_cast(X, (typename Bits<X>::U)y[j]) : __builtin_bit_cast(X, (typename Bits<X>::U)(y[j / 2] >> (j % 2 * 16)));
    }
    __syncthreads();
  }
}

}  // namespace c2t
