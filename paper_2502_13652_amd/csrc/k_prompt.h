// Causal attention over whole prompts that are packed one behind the other.
//
//   s_j = scale q_i.k_j,  j <= i of the same sequence,  p_j = e^(s_j - m),  out_i = sum p_j v_j / sum p_j
//
// One pass over the keys with a running reference m and sum, as in k_attend.h and by its rules: m moves only where a tile passes it, the divisor is the
// sum of the weights as the second product takes them, rounded to 16 bits, and the log of the sum is that of the weights as they were.  That one rounding leaves outputs of Gaussian values off by 0.0018 to
// 0.0020 of their size (rms, of bf16, of which 0.0016 are their own rounding; of halves 0.00022 to 0.00025 and 0.0002).  A second number of 16 bits for what the first leaves of a weight, as k_attend.h has it for few rows, makes
// outputs as exact as their type, for half again of the matrix unit's time: one prompt of 200 tokens 8.6 us for 8.25, of 8192 738 for 522, the 64 prompts 1111 for 795, divided keys 15 % more.  Nowhere is that for nothing,
// and it is left out of all forms.  Products are taken transposed,
// S^T = K Q^T in blocks of 32 keys and 32 rows: a lane then has one row (lane & 31) and, of each block, the keys 8 i + 4 (lane / 32) + 0..3, which are two operands of
// out^T = V^T P^T, so weights never leave their registers.
//
// Keys and values go from memory into LDS without passing registers, a tile ahead.  A wavefront has 32 rows: of 64 it would read LDS half as often, but the sums of two would not fit its registers with
// three wavefronts a SIMD, which is what hides a workgroup's start (finding its tile 3000 to 5000 cycles under load, its first keys 4000) and end (3000) behind others' products: 64 prompts of
// up to 2000 tokens take 780 us, with two 850; workgroups that stay and take tile after tile, the next one's keys on their way, took 900 for 845 (tiles dealt ahead of time do not stay together in the L2).
//
// Measured, 32 heads over 8 of 128, from card to card: one prompt of 8192 tokens 490 to 530 us for 550 GFLOP, 1.04 to 1.12 PFLOP/s, where an 8192-cubed matrix product gets 1.20: the matrix unit is busy for
// 64 % of the cycles, whose rate the card's power then holds at 1.6 to 1.7 GHz; the 64 prompts 770 to 830 us, 0.85 to 0.91, busy for 50 %; one prompt of 200 7.8 us: the tile found after 1.4, its first keys there after 2.7, two tiles 2.5.
// Width 64 (3 prompts of 2100 to 5001, halves, with the log of the sums) 116 to 124 us, 0.69 to 0.74: vector instructions, five a score, take longer than its products.  Width 256 (6 prompts of 77 to 2500, 8 heads
// over one) 84 to 87 us, 0.66 to 0.69, of 8192 tokens 292 to 309, 0.89 to 0.94: pairs of wavefronts wait for keys, weights and values in turn, 3600 cycles a tile of 64 keys of which the products take 1024, beside one other
// workgroup.  Halves of the output by workgroups, with the scores made twice, took 97 and 348; a row's whole output in one wavefront, of which then one fits a SIMD, 170 for 4096 tokens where pairs take 114.
#pragma once
#include "k_attend.h"

namespace c2t {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

struct PromptArgs {
  const char* q; const char* k; const char* v; char* out; float* lse;
  int64_t q_row, k_row, v_row, out_row;                      // bytes
  float scale_log2e;
};
// What finding a tile takes: a kernel's first arguments, which are there when it starts.
struct PromptShape {
  const int32_t* starts;
  int32_t rows, sequences, kv_heads, group;
  float inv_kv_heads, inv_group;                             // their reciprocals
};

__device__ __forceinline__ f32x16 product32(Bf16::T8 a, Bf16::T8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 product32(F16::T8 a, F16::T8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// A tile of rows of a sequence.
struct PromptTile { int first, n, tile; };                   // the sequence's first row and length

// The tile of rank `rank`.  Sequences of 2^c tiles and more come ahead of shorter ones; those of one c in their order, TOGETHER at a time, whose tiles go by the number of keys, most first.
// So the longest start first, the tiles that run at one time share few sequences' keys in the dies' L2, and few sequences still end together: 64 prompts of up to 2000 tokens take
// 940 us so, one sequence after the other 950, all sequences' tiles by their keys 1030; four of 1000 53, 57 and 53 (of the kernel as it was then).
// Every wavefront finds it for itself: a lane has every 64th sequence, tiles of a class and above are a sum over lanes.  False: there is no such tile.
constexpr int TOGETHER = 4;
template <int ROWS>
__device__ __forceinline__ bool find_tile(const PromptShape& a, int rank, PromptTile* u) {
  const int lane = lane_id();
  const auto length = [&](int b, int* first) {
    const int at = min(b, a.sequences - 1), from = a.starts[at], end = a.starts[at + 1];
    *first = from;
    return b < a.sequences && from >= 0 && end >= from && end <= a.rows ? end - from : 0;
  };
  const auto tiles = [&](int n) { return (n * a.group + ROWS - 1) / ROWS; };  // (rows * group: at most 2^30, checked by the host)
  int first[TOGETHER], n[TOGETHER], has[TOGETHER], left = rank;
  if (a.sequences <= TOGETHER) {
#pragma unroll
    for (int i = 0; i < TOGETHER; ++i) {                     // (the same for all lanes)
      n[i] = uniform(length(i, &first[i]));
      first[i] = uniform(first[i]);
      has[i] = tiles(n[i]);
    }
  } else {
    int my_first;
    const int my_n = length(lane, &my_first), my_tiles = tiles(my_n);
    const auto from_class = [&](int c) {
      int mine = my_tiles >> c != 0 ? my_tiles : 0;
#pragma unroll 1
      for (int b = lane + WAVE; b < a.sequences; b += WAVE) { int f; const int t = tiles(length(b, &f)); mine += t >> c != 0 ? t : 0; }
      return wave_sum_i(mine);
    };
    if (from_class(0) <= rank) return false;
    int c = 0, above = 32 - __builtin_clz(tiles(a.rows)), ahead = 0;           // tiles of class `above` and more: `ahead`, at most the rank
    while (above - c > 1) {
      const int mid = (c + above) / 2, count = from_class(mid);
      if (count > rank) c = mid; else { above = mid; ahead = count; }
    }
    left -= ahead;                                           // which of the class's tiles
    int f = my_first, m = my_n, mine, to, b0 = 0;
    uint64_t past;
    for (;;) {
      const int t = tiles(m);
      mine = t >> c == 1 ? t : 0; to = wave_scan_incl(mine);
      past = __ballot(to > left);
      if (past != 0ull) break;
      b0 += WAVE;
      if (b0 >= a.sequences) return false;                   // (starts that change while they are read)
      left -= __builtin_amdgcn_readlane(to, WAVE - 1);
      m = length(b0 + lane, &f);
    }
    // the TOGETHER sequences of the class that it is among
    const int place = __popcll(__ballot(mine != 0) & ((1ull << lane) - 1ull)) / TOGETHER, at = __builtin_amdgcn_readlane(place, __builtin_ctzll(past));
    uint64_t members = __ballot(mine != 0 && place == at);
    left -= __builtin_amdgcn_readlane(to - mine, __builtin_ctzll(members));
#pragma unroll
    for (int i = 0; i < TOGETHER; ++i) {
      const int from = members != 0ull ? __builtin_ctzll(members) : 0;
      first[i] = __builtin_amdgcn_readlane(f, from);
      n[i] = __builtin_amdgcn_readlane(m, from);
      has[i] = members != 0ull ? __builtin_amdgcn_readlane(mine, from) : 0;
      members &= members - 1ull;
    }
  }
  const auto above_level = [&](int level) {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < TOGETHER; ++i) sum += max(has[i] - level, 0);
    return sum;
  };
  if (above_level(0) <= left) return false;
  int level = 0, most = 1;                                   // the highest with more than `left` tiles on it and above
#pragma unroll
  for (int i = 0; i < TOGETHER; ++i) most = max(most, has[i]);
  for (int span = most; span > 1;) {
    const int step = div_up(span, WAVE);
    level += (__popcll(__ballot(lane * step < span && above_level(level + lane * step) > left)) - 1) * step;
    span = step;
  }
  left -= above_level(level + 1);
  bool found = false;
#pragma unroll
  for (int i = 0; i < TOGETHER; ++i) {
    if (has[i] <= level) continue;
    if (left-- != 0) continue;
    u->first = first[i]; u->n = n[i]; u->tile = level;
    found = true;
  }
  return found;
}

// Where 16-byte piece `piece` of row `row` lies in a tile in LDS: pieces change places within a row so that 16 rows' same piece (a K operand), and 32 bytes each of 4
// rows in a row (a V operand, read transposed), fall on different banks.
template <int D> __device__ __forceinline__ int piece_at(int row, int piece) {
  const int turn = D >= 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
  return row * (D * 2) + (piece ^ turn) * 16;
}

// 16 bytes a lane from memory into LDS, without a register on the way: lane i's to `to` + 16 i.  The compiler does not count it: whoever reads waits for it (wait_vector_memory, and a
// barrier for what other wavefronts loaded), and no wavefront ends ahead of its own.
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t offset, uint32_t to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

// a + the sum of a pair's two numbers, in fp32
__device__ __forceinline__ float add_pair(Bf16::T8 x, int pair, float a) {
  typedef __bf16 T2 __attribute__((ext_vector_type(2)));
  const T2 one = {(__bf16)1.f, (__bf16)1.f}, y = {x[pair * 2], x[pair * 2 + 1]};
  return __builtin_amdgcn_fdot2_f32_bf16(y, one, a, false);
}
__device__ __forceinline__ float add_pair(F16::T8 x, int pair, float a) {
  typedef _Float16 T2 __attribute__((ext_vector_type(2)));
  const T2 one = {(_Float16)1.f, (_Float16)1.f}, y = {x[pair * 2], x[pair * 2 + 1]};
  return __builtin_amdgcn_fdot2(y, one, a, false);
}

constexpr int prompt_waves(int kw) { return kw > 1 ? kw : 4; }                   // of a workgroup, and its rows
constexpr int prompt_rows(int kw, bool pairs) { return kw > 1 ? 32 : 32 * prompt_waves(kw) / (pairs ? 2 : 1); }

// How a block of PRODUCTS matrix instructions and READS reads of their operands is to be laid out: AHEAD reads, then EACH reads behind each product.
template <int PRODUCTS, int READS, int AHEAD, int EACH> __device__ __forceinline__ void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
  for (int i = 0; i < PRODUCTS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    if (AHEAD + i * EACH < READS) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
  }
}
constexpr int K_AHEAD = 4, V_AHEAD = 2;                      // operands read ahead of their product

// Stands between products and a block behind theirs that reads their results: a result is there 12 issue slots behind its product, and the compiler, which has been seen to count too few of them from block to
// block (9 from the last product of the form whose wavefronts divide the keys to the sums' first reader behind the loop), is left none to count.
__device__ __forceinline__ void products_done() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 11");
  __builtin_amdgcn_sched_barrier(0);
}

// KB blocks of 32 keys a tile; OCC workgroups a CU.  The wavefronts have 32 rows each and share the tiles (KW = 1), or the same 32 rows and KW wavefronts every KW-th tile each, joined at
// the end: a quarter of the way along the keys where there are few rows.  DV of the D elements of an output row are one wavefront's: D; or half, as more sums do not fit its registers.
// Then two wavefronts have the same 32 rows (PAIRS): each makes the weights of one of a tile's two blocks, which both take from LDS, and half of the output.
template <typename E, int D, int DV, int KB, int KW, int OCC, bool LSE>
__global__ __launch_bounds__(64 * prompt_waves(KW), OCC) void k_prompt(const int32_t* starts, int32_t all_rows, int32_t sequences, int32_t kv_heads, int32_t G, float inv_kv_heads,
                                                                       float inv_group, PromptArgs a) {
  typedef typename E::T T; typedef typename E::T4 T4; typedef typename E::T8 T8;
  constexpr bool PAIRS = DV < D;
  static_assert(!PAIRS || (KB == 2 && KW == 1 && D == 2 * DV), "");
  constexpr int WAVES = prompt_waves(KW), NT = 64 * WAVES, ROWS = prompt_rows(KW, PAIRS), KT = 32 * KB, DB = DV / 32, DK = D / 16;
  constexpr int SHARERS = KW > 1 ? 64 : NT;                  // threads that load a tile together
  constexpr int K_LOADS = KT * D / 8 / SHARERS, V_LOADS = KT * D / 8 / SHARERS, K_TILE = KT * D * 2, TILE = K_TILE + KT * D * 2;
  constexpr float TOP = E::TOP, SLACK = E::SLACK, BIG = 0x1p22f;
  constexpr int WEIGHTS = 2 * 64 * 16;                       // PAIRS: a wavefront's of a tile, two operands a lane
  __shared__ __align__(16) char lds[PAIRS ? TILE + WAVES * WEIGHTS : 2 * TILE * KW];  // K and V, two buffers, of each wavefront that has tiles of its own; PAIRS: one, and weights
  __shared__ __align__(16) int moves_of[4];                  // PAIRS: whether a wavefront's scores ask for another reference,
  __shared__ float tops[PAIRS ? WAVES * 32 : 1];             // and its rows' largest then
  __shared__ int odd_value;                                  // a tile held a value that is not finite (KW = 1)
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col = lane & 31, half = lane >> 5;
  const int kw = KW > 1 ? wave : 0, lt = KW > 1 ? lane : tid;        // this thread among those that load a tile
  char* const tiles = lds + kw * 2 * TILE;
  bool my_odd = false;

  // The query heads of one cached head share its keys: a tile's rows are (token, head of the group) with the head fastest, so that its wavefronts come to their last key together, however
  // many heads there are, and short prompts fill tiles.
  if (KW == 1 && tid == 0) odd_value = 0;
  PromptTile u;
  const int part = PAIRS ? wave & 1 : 0;                     // of an output row
  int rank, head;
  split(blockIdx.x, kv_heads, inv_kv_heads, &rank, &head);
  rank = uniform(rank); head = uniform(head);
  if (!find_tile<ROWS>(PromptShape{starts, all_rows, sequences, kv_heads, G, inv_kv_heads, inv_group}, rank, &u)) return;
  const int row0 = u.tile * ROWS, wave_row0 = row0 + (KW > 1 ? 0 : PAIRS ? wave / 2 * 32 : wave * 32), rows = u.n * G;
  const auto token_of = [&](int row, int* g) { int t; split(min(row, rows - 1), G, inv_group, &t, g); return t; };      // (rows behind the last are not put out)
  int my_g, no_g;
  const int my_token = token_of(wave_row0 + col, &my_g);
  const int first_token = uniform(token_of(row0, &no_g)), wave_first = uniform(token_of(wave_row0, &no_g)), wave_last = uniform(token_of(wave_row0 + 31, &no_g));
  const int keys = uniform(token_of(row0 + ROWS - 1, &no_g)) + 1, n_tiles = div_up(keys, KT);
  const bool idle = wave_row0 >= rows;
  const char* const k_head = a.k + u.first * a.k_row + (int64_t)head * (D * 2);
  const char* const v_head = a.v + u.first * a.v_row + (int64_t)head * (D * 2);

  // A tile's pieces: this thread's j-th lies j SHARERS + lt pieces into K's or V's tile in LDS, and is the piece of its row that piece_at puts there: the same one in every 16th row, so
  // that one offset (two, of rows of 8 a load) does for all of a tile's.
  constexpr int K_ROWS = SHARERS / (D / 8), V_ROWS = SHARERS / (D / 8), K_KINDS = K_ROWS < 16 ? 16 / K_ROWS : 1, V_KINDS = V_ROWS < 16 ? 16 / V_ROWS : 1;      // rows a load, offsets
  const auto k_piece = [&](int j) { const int row = j * K_ROWS + lt / (D / 8); return (uint32_t)(piece_at<D>(row, lt % (D / 8)) - row * (D * 2)); };
  const auto v_piece = [&](int j) { const int row = j * V_ROWS + lt / (D / 8); return (uint32_t)(piece_at<D>(row, lt % (D / 8)) - row * (D * 2)); };
  uint32_t k_off[K_KINDS], v_off[V_KINDS];
#pragma unroll
  for (int j = 0; j < K_KINDS; ++j) k_off[j] = lt / (D / 8) * (uint32_t)a.k_row + k_piece(j);
#pragma unroll
  for (int j = 0; j < V_KINDS; ++j) v_off[j] = lt / (D / 8) * (uint32_t)a.v_row + v_piece(j);
  const uint32_t lds_wave = lds_address(tiles) + (KW > 1 ? 0 : wave * 1024);
  const char* k_at = k_head + kw * KT * a.k_row; const char* v_at = v_head + kw * KT * a.v_row;
  int ahead = keys - kw * KT;                                          // keys from there on
  const auto request = [&](int buffer) {
    const uint32_t to = lds_wave + buffer * TILE;
    if (ahead >= KT) {
#pragma unroll
      for (int j = 0; j < K_LOADS; ++j) load_to_lds(k_at + j * K_ROWS * a.k_row, k_off[j % K_KINDS], to + j * SHARERS * 16);
#pragma unroll
      for (int j = 0; j < V_LOADS; ++j) load_to_lds(v_at + j * V_ROWS * a.v_row, v_off[j % V_KINDS], to + K_TILE + j * SHARERS * 16);
    } else {                                                 // rows behind the last key are taken from it (and masked)
#pragma unroll
      for (int j = 0; j < K_LOADS; ++j) load_to_lds(k_at, (uint32_t)min(j * K_ROWS + lt / (D / 8), ahead - 1) * (uint32_t)a.k_row + k_piece(j), to + j * SHARERS * 16);
#pragma unroll
      for (int j = 0; j < V_LOADS; ++j) load_to_lds(v_at, (uint32_t)min(j * V_ROWS + lt / (D / 8), ahead - 1) * (uint32_t)a.v_row + v_piece(j), to + K_TILE + j * SHARERS * 16);
    }
    k_at += KW * KT * a.k_row; v_at += KW * KT * a.v_row; ahead -= KW * KT;
  };
  // PAIRS: K or V alone (whose tiles are alike), a load at a time between the products: asked for at once, a tile's loads wait 700 cycles for each other.  Loads behind the one with the last of `left`
  // keys ask for that one's rows, rows behind the last key for the last key's.
  struct Ask { const char* at; int last; uint32_t off[K_KINDS], end[K_KINDS]; };
  const auto ask = [&](const char* at, const uint32_t* off, int64_t row, int left) {
    Ask x;
    x.at = at; x.last = min((left - 1) / K_ROWS, K_LOADS - 1);
#pragma unroll
    for (int j = 0; j < K_KINDS; ++j) x.off[j] = x.end[j] = off[j];
    if (left < KT) {
      int t = lt;
      settle(t);                                             // (rare: nothing of it is kept in registers)
#pragma unroll
      for (int j = 0; j < K_KINDS; ++j) {
        const int r = j * K_ROWS + t / (D / 8);
        x.end[j] = (uint32_t)min(t / (D / 8), left - 1 - x.last * K_ROWS) * (uint32_t)row + (uint32_t)(piece_at<D>(r, t % (D / 8)) - r * (D * 2));
      }
    }
    return x;
  };
  const auto ask_piece = [&](const Ask& x, int64_t row, uint32_t to, int j) {
    load_to_lds(x.at + (uint32_t)min(j, x.last) * (uint32_t)(K_ROWS * row), j < x.last ? x.off[j % K_KINDS] : x.end[j % K_KINDS], to + j * SHARERS * 16);
  };
  // Waits for this wavefront's pieces.  Where some rows see a value that others do not, one that is not finite is left out of the product and added for the rows that see it.
  const auto arrived = [&](int buffer, bool diagonal) {
    wait_vector_memory();
    if (!diagonal) return;
    u32x4* const mine = (u32x4*)(tiles + buffer * TILE + K_TILE + lt * 16);
    // Of all together whether there is one: one piece after the other takes 2500 cycles of 8 (one prompt of 200 tokens 8.7 us, so 7.8).
    u16x2 most = {0, 0};                                     // of the halves without their signs
#pragma unroll
    for (int j = 0; j < V_LOADS; ++j) {
      if (PAIRS && j % 2 == 0) __builtin_amdgcn_sched_barrier(0);        // (two at a time: scores are in registers here)
      const u32x4 x = mine[j * SHARERS] & 0x7fff7fffu;
#pragma unroll                                               // (by way of `two`: a bit cast of x[i] itself takes the vector's first element)
      for (int i = 0; i < 4; ++i) { const uint32_t two = x[i]; most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, two)); }
    }
    if (!__any(odd_halves<E>(__builtin_bit_cast(uint32_t, most)) != 0u)) return;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < V_LOADS; ++j) {                      // (rare; as a loop it costs registers that the scores' loop has not)
      __builtin_amdgcn_sched_barrier(0);
      const u32x4 x = mine[j * SHARERS];
      const u32x4 bad = {odd_halves<E>(x.x), odd_halves<E>(x.y), odd_halves<E>(x.z), odd_halves<E>(x.w)};
      if ((bad.x | bad.y | bad.z | bad.w) != 0u) { odd = true; mine[j * SHARERS] = x & ~bad; }
    }
    if (KW > 1) my_odd = my_odd || __any(odd);
    else if (odd) odd_value = 1;
  };
  // Where this lane's operands begin: of K row `col` and piece `half`, of V rows 4 half + (lane & 15) / 4 and the lane's 8 bytes of a block of 32 elements.  The others lie at these
  // places but for whole rows and bits of the piece's number.
  const int k_place = piece_at<D>(col, half);
  const int v_place = K_TILE + piece_at<D>(half * 4 + (lane & 15) / 4, (lane >> 4 & 1) * 2 + (lane & 3) / 2) + (lane & 1) * 8 + part * (DV * 2);
  if constexpr (PAIRS) {
    const Ask x = ask(k_at, k_off, a.k_row, keys);
#pragma unroll
    for (int j = 0; j < K_LOADS; ++j) ask_piece(x, a.k_row, lds_wave, j);
    k_at += KT * a.k_row;
  } else {
    if (kw < n_tiles) request(0);
  }
  T8 q[DK];
  {
    const char* const from = a.q + ((int64_t)u.first + my_token) * a.q_row + query_offset(head, G, my_g, D) * 2 + half * 16;
#pragma unroll
    for (int kk = 0; kk < DK; ++kk) q[kk] = *(const T8*)(from + kk * 32);
  }
  if (KW == 1 && KT > first_token) __syncthreads();          // (odd_value)
  if constexpr (PAIRS) wait_vector_memory();
  else if (kw < n_tiles) arrived(0, kw * KT + KT > first_token);
  // The queries are here before the loop, or each of its rounds would wait for them, and for the next tile's pieces, which are younger, with them.
#pragma unroll
  for (int kk = 0; kk < DK; ++kk) { u32x4 x = __builtin_bit_cast(u32x4, q[kk]); settle(x); q[kk] = __builtin_bit_cast(T8, x); }
  if (KW == 1) __syncthreads();
  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m_run = -INFINITY, e_run = 0.f, l_run = 0.f, factor = a.scale_log2e;
  int big = 0;

  if constexpr (PAIRS) {
    // One buffer each: V of this tile comes while its scores are made, K of the next one during the second product.  Weights are made with the reference as it is; where a row's scores ask for another,
    // all wavefronts know it behind the barrier, and they are made once more.
    const int my_keys = part * 32;
    char* const pair_weights = lds + TILE + (wave & ~1) * WEIGHTS + lane * 16; char* const my_weights = pair_weights + part * WEIGHTS;
    for (int t = 0; t < n_tiles; ++t) {
      const int key0 = t * KT;
      const bool sees = !idle && key0 + my_keys <= wave_last;
      const Ask ask_v = ask(v_at, v_off, a.v_row, keys - key0);
      v_at += KT * a.v_row;
      f32x16 s;
      float top = -INFINITY, l_add = 0.f, e_add = 0.f;
      T8 p[4];
      const auto weights = [&](float ref) {
        l_add = e_add = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int pair = 0; pair < 4; ++pair) {
#pragma unroll
            for (int r = pair * 2; r < pair * 2 + 2; ++r) {
              const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h * 8 + r], factor, -ref));
              if (LSE) e_add += w;
              p[h][r] = (T)w;
            }
            l_add = add_pair(p[h], pair, l_add);
          }
#pragma unroll
        for (int h = 0; h < 2; ++h) *(T8*)(my_weights + h * 1024) = p[h];
      };
      bool moves = false;
      if (sees) {
        int k_base = k_place + part * 32 * (D * 2);
        settle(k_base);
        T8 k[DK];
        const auto read_k = [&](int i) { k[i] = *(const T8*)(tiles + (k_base ^ i * 32)); };
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int i = 0; i < K_AHEAD; ++i) read_k(i);
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) {
          __builtin_amdgcn_sched_barrier(0);
          s = product32(k[kk], q[kk], s);
          if (kk + K_AHEAD < DK) read_k(kk + K_AHEAD);
          if (kk % 2 == 1) ask_piece(ask_v, a.v_row, lds_wave + K_TILE, kk / 2);
        }
        __builtin_amdgcn_sched_barrier(0);
        settle(s);
        if (key0 + my_keys + 31 > wave_first) {
          const int last_seen = my_token - key0 - my_keys - half * 4;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = i / 4 * 8 + i % 4 <= last_seen ? s[i] : -INFINITY;
        }
        if (big != 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] *= a.scale_log2e;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
        top *= factor;
        moves = __any(top - m_run > TOP);
        if (!moves) {
          weights(m_run == -INFINITY ? 0.f : m_run);
        } else {
          top = fmaxf(top, __shfl_xor(top, 32));
          if (half == 0) tops[wave * 32 + col] = top;
        }
      } else {
#pragma unroll
        for (int j = 0; j < V_LOADS; ++j) ask_piece(ask_v, a.v_row, lds_wave + K_TILE, j);
#pragma unroll
        for (int h = 0; h < 2; ++h) *(u32x4*)(my_weights + h * 1024) = u32x4{0u, 0u, 0u, 0u};
      }
      if (lane == 0) moves_of[wave] = moves;
      arrived(0, key0 + KT > first_token);
      __syncthreads();
      typedef int i32x4 __attribute__((ext_vector_type(4)));
      const i32x4 moving = *(const i32x4*)moves_of;
      const int other_moves = moves_of[wave ^ 1];
      const auto read_p = [&]() {
#pragma unroll
        for (int h = 0; h < 4; ++h) p[h] = *(const T8*)(pair_weights + h * 1024);
      };
      read_p();
      if (uniform(moving.x | moving.y | moving.z | moving.w) != 0) {       // of all wavefronts together
        if (!moves) top = -INFINITY;
        if (uniform(other_moves) != 0) top = fmaxf(top, tops[(wave ^ 1) * 32 + col]);
        float m_new = fmaxf(m_run, top - (TOP - SLACK));
        if (top - m_new > TOP) m_new = top;
        if (big == 0 && __any(__builtin_fabsf(m_new) >= BIG && m_new != -INFINITY)) {
          big = 1; factor = 1.f;
          if (sees)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] *= a.scale_log2e;
        }
        const float back = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
        m_run = m_new;
        l_run *= back; e_run *= back;
#pragma unroll
        for (int i = 0; i < DB * 16; ++i) o[i / 16][i % 16] *= back;
        if (sees) weights(m_run == -INFINITY ? 0.f : m_run);
        __syncthreads();
        read_p();
      }
      const bool more = t + 1 < n_tiles;                     // (behind the last tile: the first key's row, which nothing reads)
      const Ask ask_k = ask(more ? k_at : k_head, k_off, a.k_row, more ? keys - key0 - KT : 1);
      k_at += KT * a.k_row;
      l_run += l_add; e_run += e_add;
      // (Wavefronts whose rows see none of the tile take part with weights of zero; from such a tile, values that are not finite have been taken out.)
      int v_base = v_place;
      settle(v_base);
      T8 v[4 * DB];
      const auto read_v = [&](int i) {
        const int h = i / DB, d = i % DB;
        typedef __attribute__((address_space(3))) s16x4* lds4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tiles + (v_base ^ d * 64) + h * 16 * (D * 2)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tiles + (v_base ^ (d * 64 + 32)) + (h * 16 + 8) * (D * 2)));
        struct { s16x4 a, b; } both{lo, hi};
        v[i] = __builtin_bit_cast(T8, both);
      };
#pragma unroll
      for (int i = 0; i < V_AHEAD; ++i) read_v(i);
#pragma unroll
      for (int i = 0; i < 4 * DB; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        o[i % DB] = product32(v[i], p[i / DB], o[i % DB]);
        if (i + V_AHEAD < 4 * DB) read_v(i + V_AHEAD);
        if (i % 2 == 1) ask_piece(ask_k, a.k_row, lds_wave, i / 2);
      }
      products_done();
      wait_vector_memory();
      __syncthreads();
    }
  } else for (int t = kw; t < n_tiles; t += KW) {
    const int key0 = t * KT, buffer = t / KW & 1;
    if (t + KW < n_tiles) request(buffer ^ 1);
    if (!idle && key0 <= wave_last) {
      int k_base = k_place + buffer * TILE, v_base = v_place + buffer * TILE;
      settle(k_base); settle(v_base);                        // (what follows from them is made anew each time, and holds no registers)
      f32x16 s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < DK; ++kk)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) s[kb] = product32(*(const T8*)(tiles + (k_base ^ kk * 32) + kb * 32 * (D * 2)), q[kk], s[kb]);
      reads_ahead<KB * DK, KB * DK, K_AHEAD, 1>();
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) settle(s[kb]);
      if (key0 + KB * 32 - 1 > wave_first) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[kb][i] = key0 + kb * 32 + i / 4 * 8 + half * 4 + i % 4 <= my_token ? s[kb][i] : -INFINITY;
      }
      if (big != 0) {
#pragma unroll
        for (int i = 0; i < KB * 16; ++i) s[i / 16][i % 16] *= a.scale_log2e;
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
          for (int i = 0; i < KB * 16; ++i) s[i / 16][i % 16] *= a.scale_log2e;
        }
        const float back = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
        m_run = m_new;
        l_run *= back; e_run *= back;
#pragma unroll
        for (int i = 0; i < DB * 16; ++i) o[i / 16][i % 16] *= back;
      }
      const float ref = m_run == -INFINITY ? 0.f : m_run;
      // Products by steps of 16 keys.  Weights are made, two at a time, a step ahead of the products that take them, V's operands read V_AHEAD products ahead: between a step's products
      // are the next one's instructions, in the order that is written here.
      constexpr int STEPS = KB * 2;
      T8 p[2], v[STEPS * DB];
      const auto weights = [&](int h, int pair) {
#pragma unroll
        for (int r = pair * 2; r < pair * 2 + 2; ++r) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h / 2][h % 2 * 8 + r], factor, -ref));
          if (LSE) e_run += w;
          p[h & 1][r] = (T)w;
        }
        l_run = add_pair(p[h & 1], pair, l_run);
      };
      const auto read_v = [&](int i) {
        const int h = i / DB, d = i % DB;
        typedef __attribute__((address_space(3))) s16x4* lds4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tiles + (v_base ^ d * 64) + h * 16 * (D * 2)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tiles + (v_base ^ (d * 64 + 32)) + (h * 16 + 8) * (D * 2)));
        struct { s16x4 a, b; } both{lo, hi};
        v[i] = __builtin_bit_cast(T8, both);
      };
#pragma unroll
      for (int i = 0; i < V_AHEAD; ++i) read_v(i);
#pragma unroll
      for (int pair = 0; pair < 4; ++pair) weights(0, pair);
#pragma unroll
      for (int i = 0; i < STEPS * DB; ++i) {
        const int h = i / DB, d = i % DB;
        __builtin_amdgcn_sched_barrier(0);
        o[d] = product32(v[i], p[h & 1], o[d]);
        if (i + V_AHEAD < STEPS * DB) read_v(i + V_AHEAD);
        if (h + 1 < STEPS)
#pragma unroll
          for (int pair = d * 4 / DB; pair < (d + 1) * 4 / DB; ++pair) weights(h + 1, pair);
      }
    }
    if (t + KW < n_tiles) arrived(buffer ^ 1, key0 + (KW + 1) * KT > first_token);
    else if (KW > 1) products_done();
    if (KW == 1) __syncthreads();
  }
  if (KW == 1 && !PAIRS) products_done();                    // (behind a barrier; within the loop it takes prompts of 1000 tokens 1.3 % longer)
#pragma unroll
  for (int d = 0; d < DB; ++d) settle(o[d]);
  if (!PAIRS && idle) return;
  l_run += __shfl_xor(l_run, 32); e_run += __shfl_xor(e_run, 32);
  if constexpr (PAIRS) {                                     // (each has those of its keys, by one reference)
    float* const sums = (float*)(lds + TILE);
    if (half == 0) { sums[wave * 64 + col] = l_run; sums[wave * 64 + 32 + col] = e_run; }
    __syncthreads();
    l_run += sums[(wave ^ 1) * 64 + col]; e_run += sums[(wave ^ 1) * 64 + 32 + col];
    if (idle) return;
  }

  if (KW > 1 ? my_odd : odd_value != 0) {                    // values that are not finite: a weight is made again from its key
    const char* const k_odd = k_head + half * 16;
    const char* const v_odd = v_head + part * (DV * 2) + half * 8;
    for (int key = first_token / KT * KT; key <= wave_last; ++key) {
      if (KW > 1 && key / KT % KW != kw) continue;
      const auto value = [&](int d) { return *(const T4*)(v_odd + key * a.v_row + d * 16); };
      bool any = false;
      for (int d = 0; d < DB * 4; ++d) {
        const T4 x = value(d);
#pragma unroll
        for (int r = 0; r < 4; ++r) any = any || !(__builtin_fabsf((float)x[r]) < INFINITY);
      }
      if (!__any(any)) continue;
      float dot = 0.f;
#pragma unroll
      for (int kk = 0; kk < DK; ++kk) {
        __builtin_amdgcn_sched_barrier(0);                   // (one piece at a time, and none made ahead of the loop: this is rare, and the loop above has the registers)
        u32x4 mine = __builtin_bit_cast(u32x4, q[kk]);
        settle(mine);
        const T8 x = __builtin_bit_cast(T8, mine);
        const T8 y = *(const T8*)(k_odd + key * a.k_row + kk * 32);
#pragma unroll
        for (int r = 0; r < 8; ++r) dot = __builtin_fmaf((float)y[r], (float)x[r], dot);
      }
      dot += __shfl_xor(dot, 32);
      const float w = __builtin_amdgcn_exp2f(rounded_difference(dot, a.scale_log2e, m_run == -INFINITY ? 0.f : m_run));
      if (key > my_token) continue;
#pragma unroll
      for (int d = 0; d < DB * 4; ++d) {
        __builtin_amdgcn_sched_barrier(0);
        const T4 x = value(d);
#pragma unroll
        for (int r = 0; r < 4; ++r) { const float y = (float)x[r]; if (!(__builtin_fabsf(y) < INFINITY)) o[d / 4][d % 4 * 4 + r] += w * y; }
      }
    }
  }
  // of a sum as if the reference were the largest score (k_attend.h)
  const auto log_of = [&](float m, float e) {
    constexpr float BELOW = TOP - SLACK;
    return ((m + BELOW) + __builtin_amdgcn_logf(e * __builtin_ldexpf(1.f, -(int)BELOW))) * 0.69314718055994531f;
  };
  if constexpr (KW > 1) {
    // The wavefronts' shares of the rows, joined through LDS: sums of products with their pieces of 16 bytes at other places from row to row, references and sums of weights behind them.
    constexpr int SUMS = 32 * DV * 4;
    static_assert(SUMS + 3 * 32 * 4 <= 2 * TILE, "");
    const auto place = [&](int row, int piece) { return (row * (DV / 4) + (piece ^ (row & (DV / 4 - 1)))) * 16; };
    float* const stats = (float*)(tiles + SUMS);
#pragma unroll
    for (int d = 0; d < DB * 4; ++d) {
      f32x4 x;
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = o[d / 4][d % 4 * 4 + r];
      *(f32x4*)(tiles + place(col, d * 2 + half)) = x;
    }
    if (half == 0) { stats[col] = m_run; stats[32 + col] = l_run; stats[64 + col] = e_run; }
    __syncthreads();
#pragma unroll
    for (int i0 = 0; i0 < 32 * (DV / 8); i0 += NT) {
      const int i = i0 + tid, row = i / (DV / 8), piece = i % (DV / 8);
      if (wave_row0 + row >= rows) continue;
      const auto of = [&](int w) { return (const float*)(lds + w * 2 * TILE + SUMS) + row; };
      float m = -INFINITY, l = 0.f, e = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) m = fmaxf(m, of(w)[0]);
      const float ref = m == -INFINITY ? 0.f : m;
      f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float f = __builtin_amdgcn_exp2f(of(w)[0] - ref);
        l += f * of(w)[32]; e += f * of(w)[64];
        x += f * *(const f32x4*)(lds + w * 2 * TILE + place(row, piece * 2));
        y += f * *(const f32x4*)(lds + w * 2 * TILE + place(row, piece * 2 + 1));
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      T8 z;
#pragma unroll
      for (int r = 0; r < 4; ++r) { z[r] = (T)(x[r] * inv); z[4 + r] = (T)(y[r] * inv); }
      int g;
      const int64_t t = u.first + token_of(wave_row0 + row, &g);
      *(T8*)(a.out + t * a.out_row + query_offset(head, G, g, D) * 2 + part * (DV * 2) + piece * 16) = z;
      if (LSE && piece == 0 && part == 0) a.lse[t * kv_heads * G + query_offset(head, G, g, 1)] = l == 0.f ? -INFINITY : log_of(m, e);
    }
    return;
  }
  if (LSE && half == 0 && part == 0 && wave_row0 + col < rows)
    a.lse[((int64_t)u.first + my_token) * kv_heads * G + query_offset(head, G, my_g, 1)] = l_run == 0.f ? -INFINITY : log_of(m_run, e_run);
  // Out by whole lines: 64 elements of the wavefront's 32 rows at a time pass through LDS, in its own pieces of a tile (4 stretches of 1024 bytes).  A row's pieces of 16
  // bytes change places so that 8 rows' fall on different banks.
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  const auto place = [&](int row, int piece) { const int at = row * 128 + (piece ^ (row & 7)) * 16; return at / 1024 * (NT * 16) + wave * 1024 + at % 1024; };
  char* to[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int g;
    const int t = token_of(wave_row0 + i * 8 + lane / 8, &g);
    to[i] = a.out + ((int64_t)u.first + t) * a.out_row + query_offset(head, G, g, D) * 2 + part * (DV * 2) + lane % 8 * 16;
  }
#pragma unroll
  for (int d0 = 0; d0 < DB; d0 += 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      T4 y;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = (T)(o[d0 + i / 4][i % 4 * 4 + r] * inv);
      *(T4*)(lds + place(col, i) + half * 8) = y;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront"); __builtin_amdgcn_wave_barrier(); __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    u32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *(const u32x4*)(lds + place(i * 8 + lane / 8, lane % 8));
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront"); __builtin_amdgcn_wave_barrier(); __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < 4; ++i) if (wave_row0 + i * 8 + lane / 8 < rows) *(u32x4*)(to[i] + d0 * 64) = x[i];
  }
}

}  // namespace c2t
