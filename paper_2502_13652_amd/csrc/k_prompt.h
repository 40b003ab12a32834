// Causal attention over whole prompts that are packed one behind the other.
//
//   s_j = scale q_i.k_j,  j <= i of the same sequence,  p_j = e^(s_j - m),  out_i = sum p_j v_j / sum p_j
//
// One pass over the keys with a running reference m and sum, as in k_attend.h and by its rules: m moves only where a tile passes it, the divisor is the
// sum of the weights as the second product takes them, rounded to 16 bits, and the log of the sum is that of the weights as they were.  Products are taken transposed,
// S^T = K Q^T in blocks of 32 keys and 32 rows: a lane then has one row (lane & 31) and, of each block, the keys 8 i + 4 (lane / 32) + 0..3, which are two operands of
// out^T = V^T P^T, so weights never leave their registers.
#pragma once
#include "k_attend.h"

namespace c2t {

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct PromptArgs {
  const char* q; const char* k; const char* v; char* out; float* lse;
  int64_t q_row, k_row, v_row, out_row;                      // bytes
  const int32_t* starts;
  int32_t rows, sequences, kv_heads, group;
  float scale_log2e;
};

__device__ __forceinline__ f32x16 product32(Bf16::T8 a, Bf16::T8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 product32(F16::T8 a, F16::T8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// A tile of rows of a sequence.
struct PromptTile { int first, n, tile; };                   // the sequence's first row and length

// The tile of rank `rank` of all sequences' tiles, those with the most keys first; equal ones in the sequences' order.  Every wavefront finds it for itself: a lane has every 64th
// sequence, and the number of tiles from a level on is a sum over lanes, so that the rank's level is searched by halves.  False: there is no such tile.
template <int ROWS>
__device__ __forceinline__ bool find_tile(const PromptArgs& a, int rank, PromptTile* u) {
  const int lane = lane_id();
  const auto length = [&](int b, int* first) {
    const int from = a.starts[min(b, a.sequences - 1)], end = a.starts[min(b, a.sequences - 1) + 1];
    *first = from;
    return b < a.sequences && from >= 0 && end >= from && end <= a.rows ? end - from : 0;
  };
  const auto tiles = [](int n) { return (int)(((int64_t)n + ROWS - 1) / ROWS); };
  int my_first;
  const int my_n = length(lane, &my_first), my_tiles = tiles(my_n);
  const auto from_level = [&](int level) {
    int mine = max(my_tiles - level, 0);
#pragma unroll 1
    for (int b = lane + WAVE; b < a.sequences; b += WAVE) { int f; mine += max(tiles(length(b, &f)) - level, 0); }
    return wave_sum_i(mine);
  };
  int level = 0, above = tiles(a.rows) + 1, ahead = 0;       // tiles of `above` and more: `ahead`, at most the rank
  if (from_level(0) <= rank) return false;
  while (above - level > 1) {
    const int mid = level + (above - level) / 2, count = from_level(mid);
    if (count > rank) level = mid; else { above = mid; ahead = count; }
  }
  int left = rank - ahead;                                   // which of the sequences that have that level
  u->tile = level;
#pragma unroll 1
  for (int b0 = 0; b0 < a.sequences; b0 += WAVE) {
    int f = my_first, n = my_n;
    if (b0 > 0) n = length(b0 + lane, &f);
    const bool has = tiles(n) > level;
    const uint64_t those = __ballot(has);
    const int count = __popcll(those);
    if (left >= count) { left -= count; continue; }
    const int before = __popcll(those & ((1ull << lane) - 1ull));
    const int from = __builtin_ctzll(__ballot(has && before == left));
    u->first = __builtin_amdgcn_readlane(f, from);
    u->n = __builtin_amdgcn_readlane(n, from);
    return true;
  }
  return false;
}

// Where 16-byte piece `piece` of row `row` lies in a tile in LDS: pieces change places within a row so that 16 rows' same piece (a K operand), and 32 bytes each of 4
// rows in a row (a V operand, read transposed), fall on different banks.
template <int D> __device__ __forceinline__ int piece_at(int row, int piece) {
  const int turn = D >= 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
  return row * (D * 2) + (piece ^ turn) * 16;
}

constexpr int PROMPT_WAVES = 4, PROMPT_ROWS = 32 * PROMPT_WAVES;

// KB blocks of 32 keys a tile; OCC workgroups a CU.
template <typename E, int D, int KB, int OCC, bool LSE>
__global__ __launch_bounds__(64 * PROMPT_WAVES, OCC) void k_prompt(PromptArgs a) {
  typedef typename E::T T; typedef typename E::T4 T4; typedef typename E::T8 T8;
  constexpr int NT = 64 * PROMPT_WAVES, KT = 32 * KB, CH = D / 8, DB = D / 32, DK = D / 16, LOADS = KT * CH / NT, TILE = KT * D * 2;
  constexpr float TOP = E::TOP, SLACK = E::SLACK, BIG = 0x1p22f;
  __shared__ __align__(16) char lds[4 * TILE];               // K and V, two buffers
  __shared__ int odd_value;

  // work: units are tiles of one cached head; the heads of a group, which share its keys, follow each other on one die
  const int in_die = blockIdx.x / DIES, unit = in_die / a.group * DIES + blockIdx.x % DIES, g = in_die % a.group;
  const int head = unit % a.kv_heads;
  PromptTile u;
  if (!find_tile<PROMPT_ROWS>(a, unit / a.kv_heads, &u)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, half = lane >> 5;
  const int row0 = u.tile * PROMPT_ROWS, wave_row0 = row0 + wave * 32, my_row = wave_row0 + col;
  const int keys = min(u.n, row0 + PROMPT_ROWS), n_tiles = (keys + KT - 1) / KT;
  const bool idle = wave_row0 >= u.n;
  const int64_t first = u.first;
  const char* const k_head = a.k + first * a.k_row + (int64_t)head * (D * 2);
  const char* const v_head = a.v + first * a.v_row + (int64_t)head * (D * 2);
  const int64_t q_head = query_offset(head, a.group, g, D) * 2;

  T8 q[DK];
  {
    const char* const from = a.q + (first + min(my_row, u.n - 1)) * a.q_row + q_head + half * 16;
#pragma unroll
    for (int kk = 0; kk < DK; ++kk) q[kk] = *(const T8*)(from + kk * 32);
  }
  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m_run = -INFINITY, e_run = 0.f, l_run = 0.f, factor = a.scale_log2e;
  int big = 0;

  u32x4 kr[LOADS], vr[LOADS];
  auto request = [&](int t) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int i = j * NT + tid, row = min(t * KT + i / CH, keys - 1);        // (rows behind the last key are masked)
      kr[j] = *(const u32x4*)(k_head + row * a.k_row + i % CH * 16);
      vr[j] = *(const u32x4*)(v_head + row * a.v_row + i % CH * 16);
    }
  };
  auto stage = [&](int t, char* to) {
    bool odd = false;
    if (t * KT + KT > row0) {
      // some rows see a value that others do not: one that is not finite is left out of the product and added for the rows that see it
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const uint32_t x = odd_halves<E>(vr[j].x), y = odd_halves<E>(vr[j].y), z = odd_halves<E>(vr[j].z), w = odd_halves<E>(vr[j].w);
        odd = odd || (x | y | z | w) != 0u;
        vr[j].x &= ~x; vr[j].y &= ~y; vr[j].z &= ~z; vr[j].w &= ~w;
      }
    }
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int i = j * NT + tid, at = piece_at<D>(i / CH, i % CH);
      *(u32x4*)(to + at) = kr[j];
      *(u32x4*)(to + TILE + at) = vr[j];
    }
    if (odd) odd_value = 1;
  };
  if (tid == 0) odd_value = 0;
  request(0);
  __syncthreads();
  stage(0, lds);
  if (n_tiles > 1) request(1);
  __syncthreads();

  for (int t = 0; t < n_tiles; ++t) {
    const int key0 = t * KT;
    const char* const k_lds = lds + (t & 1) * 2 * TILE;
    const char* const v_lds = k_lds + TILE;
    if (!idle && key0 <= wave_row0 + 31) {
      f32x16 s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) s[kb] = product32(*(const T8*)(k_lds + piece_at<D>(kb * 32 + col, kk * 2 + half)), q[kk], s[kb]);
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) settle(s[kb]);
      if (key0 + KT - 1 > wave_row0) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[kb][i] = key0 + kb * 32 + i / 4 * 8 + half * 4 + i % 4 <= my_row ? s[kb][i] : -INFINITY;
      }
      if (big != 0) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) s[kb] *= a.scale_log2e;
      }
      float top = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
      top *= factor;
      if (__any(top - m_run > TOP)) {                        // (uniform) of both lanes of a row, then
        top = fmaxf(top, __shfl_xor(top, 32));
        float m_new = fmaxf(m_run, top - (TOP - SLACK));
        if (top - m_new > TOP) m_new = top;                  // (it was rounded further down)
        if (big == 0 && __any(__builtin_fabsf(m_new) >= BIG && m_new != -INFINITY)) {
          big = 1; factor = 1.f;
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) s[kb] *= a.scale_log2e;
        }
        const float back = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
        m_run = m_new;
        l_run *= back; e_run *= back;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= back;
      }
      const float ref = m_run == -INFINITY ? 0.f : m_run;
      T8 p[KB * 2], ones;
#pragma unroll
      for (int r = 0; r < 8; ++r) ones[r] = (T)1.f;
#pragma unroll
      for (int h = 0; h < KB * 2; ++h)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h / 2][h % 2 * 8 + r], factor, -ref));
          if (LSE) e_run += w;
          p[h][r] = (T)w;
        }
      f32x16 sum;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[i] = 0.f;
#pragma unroll
      for (int h = 0; h < KB * 2; ++h) sum = product32(ones, p[h], sum);
#pragma unroll
      for (int h = 0; h < KB * 2; ++h)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const int row = h * 16 + half * 4 + (lane & 15) / 4, piece = d * 4 + (lane >> 4 & 1) * 2 + (lane & 3) / 2;
          typedef __attribute__((address_space(3))) s16x4* lds4;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(v_lds + piece_at<D>(row, piece) + (lane & 1) * 8));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(v_lds + piece_at<D>(row + 8, piece) + (lane & 1) * 8));
          struct { s16x4 a, b; } pair{lo, hi};
          o[d] = product32(__builtin_bit_cast(T8, pair), p[h], o[d]);
        }
      settle(sum);
      l_run += sum[0];
    }
    if (t + 1 < n_tiles) {
      stage(t + 1, lds + ((t + 1) & 1) * 2 * TILE);
      if (t + 2 < n_tiles) request(t + 2);
    }
    __syncthreads();
  }
#pragma unroll
  for (int d = 0; d < DB; ++d) settle(o[d]);
  if (idle) return;
  e_run += __shfl_xor(e_run, 32);

  if (odd_value != 0) {                                      // values that are not finite: a weight is made again from its key
    for (int key = row0 / KT * KT; key < min(keys, wave_row0 + 32); ++key) {
      const char* const v = v_head + key * a.v_row;
      T4 x[DB * 4];
      bool any = false;
#pragma unroll
      for (int d = 0; d < DB * 4; ++d) {
        x[d] = *(const T4*)(v + d * 16 + half * 8);
#pragma unroll
        for (int r = 0; r < 4; ++r) any = any || !(__builtin_fabsf((float)x[d][r]) < INFINITY);
      }
      if (!__any(any)) continue;
      float dot = 0.f;
#pragma unroll
      for (int kk = 0; kk < DK; ++kk) {
        const T8 y = *(const T8*)(k_head + key * a.k_row + kk * 32 + half * 16);
#pragma unroll
        for (int r = 0; r < 8; ++r) dot = __builtin_fmaf((float)y[r], (float)q[kk][r], dot);
      }
      dot += __shfl_xor(dot, 32);
      const float w = __builtin_amdgcn_exp2f(rounded_difference(dot, a.scale_log2e, m_run == -INFINITY ? 0.f : m_run));
      if (key > my_row) continue;
#pragma unroll
      for (int d = 0; d < DB * 4; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) { const float y = (float)x[d][r]; if (!(__builtin_fabsf(y) < INFINITY)) o[d / 4][d % 4 * 4 + r] += w * y; }
    }
  }
  if (my_row >= u.n) return;
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  char* const out = a.out + (first + my_row) * a.out_row + q_head;
#pragma unroll
  for (int d = 0; d < DB * 4; ++d) {
    T4 y;
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] = (T)(o[d / 4][d % 4 * 4 + r] * inv);
    *(T4*)(out + d * 16 + half * 8) = y;
  }
  if (LSE && half == 0) {
    // of a sum as if the reference were the largest score (k_attend.h)
    constexpr float BELOW = TOP - SLACK;
    const float UNIT = __builtin_ldexpf(1.f, -(int)BELOW);
    a.lse[(first + my_row) * a.kv_heads * a.group + query_offset(head, a.group, g, 1)] =
        l_run == 0.f ? -INFINITY : ((m_run + BELOW) + __builtin_amdgcn_logf(e_run * UNIT)) * 0.69314718055994531f;
  }
}

}  // namespace c2t
