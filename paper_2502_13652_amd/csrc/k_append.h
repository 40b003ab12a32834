// Queries and keys turned by their tokens' positions, keys and values into the pages of the paged cache.
//
//   (a, b) -> m (a cos p - b sin p, a sin p + b cos p),   p = position * turns 2^-64 of a full turn
//
// Angles are whole numbers, 64-bit fractions of a turn, so that position * turns wraps as the angle does and a position of any size loses nothing; the leading 32 bits
// of the product go into sine and cosine.  No table of angles is read: they are made anew for each token, once for all heads that a wavefront turns.
//
// Bound by the bytes, which move in rows of a head: 12000 packed tokens, 32 query heads over 8 of 128, 62 us, 5.2 TB/s as a large copy; 64 trees of up to 65 slots 17.4 us, 4.4; 24 prompts of 3 to
// 2011 tokens, 16 heads over 4 of 64, turned keys put out too, 37 us, 4.4; one token: the kernel 3.6 us, the whole call from the host 8.3.
#pragma once
#include "k_cache.h"

namespace c2t {

struct AppendArgs {
  const char* q; const char* k; const char* v; char* q_out; char* k_out;
  int64_t q_batch, q_token, kv_batch, kv_token, q_out_batch, q_out_token, k_out_batch, k_out_token;    // bytes
  const int32_t* n_new; const int32_t* starts; const int32_t* position;
  const uint64_t* turns;
  float magnitude;
  int32_t slots, q_heads, layer, nodes, pairs, neighbours;
  int32_t parts;                                             // wavefronts that share a token's heads
};

// Sine and cosine of an angle given as a 32-bit fraction of a turn.  The angle's distance from the nearest quarter turn, |x| <= pi / 4, goes into the Taylor series up to x^9 and
// x^8: what they leave is at most x^11 / 11! = 1.8e-9 and x^10 / 10! = 2.5e-8, under half of an fp32 number's last place at 1.
__device__ __forceinline__ void sine_cosine(uint32_t fraction, float* sine, float* cosine) {
  const uint32_t quarter = (fraction + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(fraction - (quarter << 30)) * 1.4629180792671596e-9f;       // 2 pi / 2^32
  const float z = x * x;
  float s = 1.f / 362880.f, c = 1.f / 40320.f;
  s = __builtin_fmaf(s, z, -1.f / 5040.f); s = __builtin_fmaf(s, z, 1.f / 120.f); s = __builtin_fmaf(s, z, -1.f / 6.f);
  s = __builtin_fmaf(x * z, s, x);
  c = __builtin_fmaf(c, z, -1.f / 720.f); c = __builtin_fmaf(c, z, 1.f / 24.f); c = __builtin_fmaf(c, z, -0.5f); c = __builtin_fmaf(c, z, 1.f);
  const float a = quarter & 1u ? c : s, b = quarter & 1u ? s : c;
  *sine = quarter & 2u ? -a : a;
  *cosine = ((quarter + 1u) & 2u) ? -b : b;
}

// The sequence that holds packed row `row` of `rows`, and which of its tokens that is; -1: none, or one that does not begin and end among the rows.  A trip to memory, of more than 64 sequences two:
// every 64th (or so) start, then the ones from the last that is not behind the row.  A sequence that begins ahead of the start that leads to it, or ends behind the next such (as it cannot where starts
// rise), is left out, or only a part of its rows would find it.  Where these starts fall themselves all sequences are gone through: no other list pays for that (4096 sequences of a token and 8000 rows
// of none take 12.0 us; where each such row went through all, 35).
__device__ __forceinline__ int sequence_of_row(const int32_t* starts, int n, int row, int rows, int* t) {
  const int lane = lane_id();
  const auto among = [&](int first, int end, int lo, int hi) {         // sequences `first` to end - 1, at most 64, from row `lo` to ahead of row `hi`
    const int i = min(first + lane, n - 1), from = starts[i], to = starts[i + 1];
    const uint64_t holds = __ballot((first + lane < end) & (from >= lo) & (from <= row) & (row < to) & (to <= hi));      // (&: both numbers in one trip)
    if (holds == 0ull) return -1;
    const int at = __builtin_ctzll(holds);
    *t = row - __builtin_amdgcn_readlane(from, at);
    return first + at;
  };
  if (n <= WAVE) return among(0, n, 0, rows);
  const int step = div_up(n, WAVE), led = div_up(n, step);   // (at most 64: C2T_MAX_CACHE_BATCH)
  const int start = starts[min(lane * step, n)], next = __shfl_down(start, 1);
  if (__any(lane + 1 < led && next < start)) {
    int b = -1;
    for (int first = 0; b < 0 && first < n; first += WAVE) b = among(first, n, 0, rows);
    return b;
  }
  const int up_to = (int)__popcll(__ballot(lane < led && start <= row)), at = up_to > 0 ? up_to - 1 : 0;
  return among(at * step, min(at * step + step, n), at > 0 ? max(__builtin_amdgcn_readlane(start, at), 0) : 0, at + 1 < led ? min(__builtin_amdgcn_readlane(start, at + 1), rows) : rows);
}

// A wavefront has a token, or one of `parts` shares of its heads.  A lane has 16 elements of a head, 8 pairs of them or 16 that only move, and keeps its pairs' sines for
// all heads that it comes to.  A pass's elements are asked for a pass ahead, the first ones ahead of where they go, which takes four trips to memory that wait for each
// other; without a condition (lanes behind the last head take its), or what some lanes leave alone would be waited for at once.
template <typename T>
__global__ __launch_bounds__(CACHE_NT) void k_cache_append(CacheView c, AppendArgs a) {
  const int lane = lane_id(), wave = uniform((int)threadIdx.x >> 6);
  const int item = blockIdx.x * (CACHE_NT / WAVE) + wave;    // (below 2^31: the host has seen to it)
  const int row = item / a.parts, part = item % a.parts;
  if (row >= a.slots) return;
  int b = blockIdx.y, t = row;
  if (a.n_new && t >= a.n_new[b]) return;
  const int64_t batch = a.starts ? 0 : b;                    // for the strides
  const char* const q = a.q + batch * a.q_batch + row * a.q_token;
  const char* const k = a.k + batch * a.kv_batch + row * a.kv_token;
  const char* const v = a.v + batch * a.kv_batch + row * a.kv_token;

  const int per_head = c.head_dim / 16, p = lane % per_head, at_once = WAVE / per_head, head_bytes = c.head_dim * 2;
  const bool turned = p * 8 < a.pairs;
  const int first = (turned && !a.neighbours ? p * 8 : p * 16) * 2;                            // bytes of the lane's two pieces of 8 elements
  const int second = turned && !a.neighbours ? first + a.pairs * 2 : first + 16;
  const int total = a.q_heads + 2 * c.kv_heads, each = a.parts * at_once, h0 = part * at_once;  // queries, keys, values
  typedef Eight<T> Piece;
  const auto load = [&](int h, Piece* x, Piece* y) {
    h = min(h + lane / per_head, total - 1);
    const char* const from = h < a.q_heads ? q + h * head_bytes : h < a.q_heads + c.kv_heads ? k + (h - a.q_heads) * head_bytes : v + (h - a.q_heads - c.kv_heads) * head_bytes;
    *x = *(const Piece*)(from + first); *y = *(const Piece*)(from + second);
  };
  Piece x, y, x_next, y_next;
  load(h0, &x, &y);
  uint64_t turns[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) turns[j] = a.turns[min(p * 8, a.pairs - 8) + j];

  if (a.starts) {
    b = sequence_of_row(a.starts, c.batch, row, a.slots, &t);
    if (b < 0) return;
  }
  const int len = tokens_in_cache(c, c.length[b]);
  const int64_t at = (int64_t)len + t;
  // where it goes, and why not
  int page = -1;
  uint32_t why = 0u;
  if (at >= capacity_of(c)) {
    why = CACHE_ROW_FULL;
  } else {
    page = valid_page(c, c.table[(int64_t)b * c.max_pages + (at >> c.page_shift)]);
    if (page < 0) why = CACHE_INVALID;
    else if (c.refcount[page] > 1) { why = CACHE_SHARED; page = -1; }
  }
  if (why && lane == 0 && part == 0) report(c, b, why);
  const int row_in = (int)(at & ((1 << c.page_shift) - 1)), chain = a.slots - a.nodes;
  int64_t position = at;
  if (a.nodes > 0 && t >= chain) position = (int64_t)len + chain - 1 + a.position[(int64_t)b * a.nodes + (t - chain)];
  float sine[8], cosine[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    sine_cosine((uint32_t)(((uint64_t)position * turns[j] + 0x80000000ull) >> 32), &sine[j], &cosine[j]);
    sine[j] *= a.magnitude; cosine[j] *= a.magnitude;
  }
  char* const q_out = a.q_out + batch * a.q_out_batch + row * a.q_out_token;
  char* const k_out = a.k_out ? a.k_out + batch * a.k_out_batch + row * a.k_out_token : nullptr;
  char* const k_page = c.k + row_offset(c, a.layer, max(page, 0), 0, row_in) * 2;
  char* const v_page = c.v + row_offset(c, a.layer, max(page, 0), 0, row_in) * 2;
  const int page_head = head_bytes << c.page_shift;
  for (int h1 = h0; h1 < total; h1 += each) {
    load(h1 + each, &x_next, &y_next);
    const int h = h1 + lane / per_head;
    if (h < total) {
      const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + c.kv_heads;
      const int head = is_q ? h : is_v ? h - a.q_heads - c.kv_heads : h - a.q_heads;
      if (turned && !is_v) {
        if (a.neighbours) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            T& ra = j < 4 ? x.v[2 * j] : y.v[2 * j - 8];
            T& rb = j < 4 ? x.v[2 * j + 1] : y.v[2 * j - 7];
            const float f = (float)ra, g = (float)rb;
            ra = (T)__builtin_fmaf(f, cosine[j], -(g * sine[j])); rb = (T)__builtin_fmaf(f, sine[j], g * cosine[j]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float f = (float)x.v[j], g = (float)y.v[j];
            x.v[j] = (T)__builtin_fmaf(f, cosine[j], -(g * sine[j])); y.v[j] = (T)__builtin_fmaf(f, sine[j], g * cosine[j]);
          }
        }
      }
      const auto put = [&](char* to) { *(Piece*)(to + first) = x; *(Piece*)(to + second) = y; };
      if (is_q) {
        put(q_out + head * head_bytes);
      } else {
        if (!is_v && k_out) put(k_out + head * head_bytes);
        if (page >= 0) put((is_v ? v_page : k_page) + (int64_t)head * page_head);
      }
    }
    x = x_next; y = y_next;
  }
}

}  // namespace c2t
