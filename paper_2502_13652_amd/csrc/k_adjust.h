// Penalties for repeated tokens, biases and a grammar's mask on logits rows that belong to the nodes of a tree.
//
//   a = times the token occurs in the sequence's context and on the row's path, o = the same without the prompt
//   y = x;  a > 0: y = x > 0 ? x / r : x r;   y -= alpha o + beta [o > 0];   y += sum of the token's biases;   not allowed: y = -inf
//
// A workgroup has a stretch of the vocabulary and some of a sequence's rows: it counts the context's tokens of its stretch
// in LDS once, and streams its stretch of each row past them, the tokens of the row's path added to the counts before and taken off
// after.  A chunk of 16 bytes without a counted, biased or masked token is copied as it is.
#pragma once
#include "k_common.h"

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
  int32_t stretch;                         // tokens of a workgroup's stretch, a multiple of ADJUST_ALIGN
  int32_t rows_each;                       // rows of a workgroup
};

constexpr int ADJUST_NT = 512;
constexpr int ADJUST_MAX_NODES = 1024, ADJUST_MAX_BIAS = 1024;
constexpr int ADJUST_ALIGN = 64;
constexpr int ADJUST_STRETCH = 8192;       // tokens at most
constexpr uint32_t IN_PROMPT = 0x80000000u, BIASED = 0x40000000u, TIMES = 0x3fffffffu;      // a token's word: flags, times in output and path

template <typename X> struct Chunk;        // 16 bytes of logits
template <> struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(const uint4& v, int i) { return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
  static __device__ __forceinline__ void set(uint4& v, int i, float x) { (i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w) = __float_as_uint(x); }
};
template <> struct Chunk<__bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float get(const uint4& v, int i) {
    const uint32_t w = i / 2 == 0 ? v.x : i / 2 == 1 ? v.y : i / 2 == 2 ? v.z : v.w;
    return i % 2 ? bf16_hi(w) : bf16_lo(w);
  }
  static __device__ __forceinline__ void set(uint4& v, int i, float x) {      // rounded to the nearest, ties to even
    uint32_t& w = i / 2 == 0 ? v.x : i / 2 == 1 ? v.y : i / 2 == 2 ? v.z : v.w;
    const uint32_t h = __builtin_bit_cast(uint16_t, (__bf16)x);
    w = i % 2 ? (w & 0xffffu) | (h << 16) : (w & 0xffff0000u) | h;
  }
};

template <typename X>
__global__ __launch_bounds__(ADJUST_NT) void k_adjust(AdjustArgs a) {
  constexpr int N = Chunk<X>::N;
  __shared__ __align__(16) uint32_t word[ADJUST_STRETCH];
  __shared__ int32_t node_token[ADJUST_MAX_NODES];
  __shared__ int16_t node_parent[ADJUST_MAX_NODES];
  __shared__ int32_t bias_at[ADJUST_MAX_BIAS];               // place in the stretch, -1: not in it
  __shared__ float bias_value[ADJUST_MAX_BIAS];              // of a token's first entry: the sum of all of its entries
  const int tid = threadIdx.x, b = blockIdx.z, v0 = blockIdx.x * a.stretch, n_words = min(a.stretch, a.vocab - v0);
  const int rows = min(max(a.n_rows[b] + a.more_rows, 0), a.rows);
  const int row0 = blockIdx.y * a.rows_each, row1 = min(row0 + a.rows_each, rows);
  if (row0 >= row1) return;

  for (int i = tid; i < a.stretch; i += ADJUST_NT) word[i] = 0u;
  const int n_nodes = a.node_token ? min(max(a.n_nodes[b], 0), a.nodes) : 0;
  for (int i = tid; i < n_nodes; i += ADJUST_NT) {
    const int p = a.node_parent[(int64_t)b * a.nodes + i];
    node_token[i] = a.node_token[(int64_t)b * a.nodes + i] - v0;
    node_parent[i] = (int16_t)(p < i ? max(p, -1) : -1);     // (a path ends however the tree was made)
  }
  __syncthreads();
  const int n_ctx = a.tokens ? (int)min((int64_t)max(a.n_tokens[b], 0), a.token_stride) : 0, n_prompt = a.n_prompt ? a.n_prompt[b] : 0;
  for (int i = tid; i < n_ctx; i += ADJUST_NT) {
    const int t = a.tokens[(int64_t)b * a.token_stride + i] - v0;
    if ((uint32_t)t < (uint32_t)n_words) { if (i < n_prompt) atomicOr(&word[t], IN_PROMPT); else atomicAdd(&word[t], 1u); }
  }
  // biases of one token add up in the order in which they are listed, in the place of the first
  const int n_bias = a.bias ? min(max(a.n_bias ? a.n_bias[b] : a.bias_stride, 0), a.bias_stride) : 0;
  for (int i = tid; i < n_bias; i += ADJUST_NT) {
    const int t = a.bias_token[(int64_t)b * a.bias_stride + i] - v0;
    bias_at[i] = (uint32_t)t < (uint32_t)n_words ? t : -1;
  }
  __syncthreads();
  for (int i = tid; i < n_bias; i += ADJUST_NT) {
    const int t = bias_at[i];
    float sum = 0.f;
    bool first = t >= 0;
    if (t >= 0) for (int j = 0; j < n_bias; ++j) {
      if (bias_at[j] != t) continue;
      if (j < i) { first = false; break; }
      sum += a.bias[(int64_t)b * a.bias_stride + j];
    }
    bias_value[i] = sum;
    if (first) atomicOr(&word[t], BIASED);
  }
  __syncthreads();

  const float rep = a.repetition ? a.repetition[b] : 1.f, freq = a.frequency ? a.frequency[b] : 0.f, pres = a.presence ? a.presence[b] : 0.f;
  // the tokens of a row's path counted (+1) or taken off again (-1); one lane walks it
  auto path = [&](int r, uint32_t by) {
    int node = a.row_node ? a.row_node[(int64_t)b * a.rows + r] : r - 1;
    if (node >= n_nodes) node = -1;
    while (node >= 0) {
      const int t = node_token[node];
      if ((uint32_t)t < (uint32_t)n_words) atomicAdd(&word[t], by);
      node = node_parent[node];
    }
  };
  for (int r = row0; r < row1; ++r) {
    if (tid == 0) path(r, 1u);
    __syncthreads();
    const char* in = a.in + b * a.in_batch + r * a.in_row + (int64_t)v0 * sizeof(X);
    char* out = a.out + b * a.out_batch + r * a.out_row + (int64_t)v0 * sizeof(X);
    const uint8_t* ok_bits = a.allowed ? (const uint8_t*)(a.allowed + b * a.allowed_batch + r * a.allowed_row) + v0 / 8 : nullptr;
    for (int i0 = tid * N; i0 < n_words; i0 += ADJUST_NT * N) {
      uint32_t ok = ok_bits ? (uint32_t)ok_bits[i0 / 8] >> (i0 % 8) : 0xffu;
      const bool end = i0 + N > n_words;                     // the row's last logits: what is behind them is not ours
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (!end) x = *(const uint4*)(in + (int64_t)i0 * sizeof(X));
      else for (int j = 0; j < n_words - i0; ++j) Chunk<X>::set(x, j, (float)((const X*)in)[i0 + j]);
      uint32_t w[N], any = 0u;
#pragma unroll
      for (int j = 0; j < N; ++j) { w[j] = word[i0 + j]; any |= w[j]; }
      const uint4 was = x;
      if (any != 0u) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          if (w[j] == 0u) continue;
          float y = Chunk<X>::get(x, j);
          const uint32_t times = w[j] & TIMES;
          if (times != 0u || (w[j] & IN_PROMPT)) y = y > 0.f ? y / rep : y * rep;
          if (times != 0u) y -= freq * (float)times + pres;
          if (w[j] & BIASED) for (int k = 0; k < n_bias; ++k) if (bias_at[k] == i0 + j) { y += bias_value[k]; break; }
          Chunk<X>::set(x, j, y);
        }
      }
      if ((ok & ((1u << N) - 1u)) != (1u << N) - 1u) {
#pragma unroll
        for (int j = 0; j < N; ++j) if (!(ok >> j & 1u)) Chunk<X>::set(x, j, -INFINITY);
      }
      if (!end) {
        if (in != out || was.x != x.x || was.y != x.y || was.z != x.z || was.w != x.w) *(uint4*)(out + (int64_t)i0 * sizeof(X)) = x;
      } else {
        for (int j = 0; j < n_words - i0; ++j) ((X*)out)[i0 + j] = (X)Chunk<X>::get(x, j);
      }
    }
    __syncthreads();
    if (tid == 0) path(r, ~0u);
  }
}

}  // namespace c2t
