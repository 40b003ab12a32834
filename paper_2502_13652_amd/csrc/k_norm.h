// Root-mean-square norm with the residual's addition, outputs in the inputs' type or in 8 bits with scales.
//
//   h = x + residual,  y = h r w,  r = (mean h^2 + eps)^-1/2;   8 bits: out = y / s,  s = max |y| / 448 over a block of the row
//
// A row passes once: its threads keep h in registers between the sum and the output.  The sum of squares is held in 64 bits, in which the square of any
// fp32 number fits, and r is used as a number in [1/2, 1) and a power of two, so rows of any size have their norm; a sum in 32 bits takes as long (4160 rows of 4096 27.4 us
// either way, 16384 of 8192 259, 20000 of 2048 58.4).
//
// Bound by the bytes: 16384 rows of 8192 bf16 with an fp32 residual, 8 bits with a scale for each 128, 260 us for 1.48 GB, 5.7 TB/s (a large copy gets 5.2); 20000 of 2048 bf16 58 us,
// 5.6; 4160 of 4096, 8 bits with a scale a row, 26.7 us, 4.4, of which some 4 us are the launch's start and end; one row: the kernel 2.4 us, the whole call from the host 7.  Rows that are not made of
// aligned pieces of 8 elements are loaded and stored by single elements, a wavefront's lanes next to each other: 3001 of 1111 fp32 8.3 to 9 us from memory, with a thread's elements next to each other 21.5.
// (Of 8 bits with a scale a block they are next to each other all the same, as its largest is looked for among neighbouring pieces.)
#pragma once
#include "k_common.h"

namespace c2t {

constexpr int NORM_NT = 256;
constexpr float E4M3_MAX = 448.f;

struct NormArgs {
  const char* x; const char* weight; const char* residual; char* residual_out; char* out; float* scales;
  int64_t x_row, residual_row, residual_out_row, out_row;    // bytes
  int64_t scales_row;                                        // elements
  int32_t rows, width;
  int32_t block;                                             // elements a scale; 0: the row
  bool weight_f32, residual_f32;
  float eps;
};

// Which elements of a row the eight of a thread's piece are: next to each other from `first` on, or `step` apart, so that a wavefront's lanes have neighbours: what rows that are not
// made of aligned pieces are loaded and stored by.
template <bool WHOLE> struct Piece { int first, step; };
template <typename T, bool WHOLE>
__device__ __forceinline__ void load_eight(const char* row, const Piece<WHOLE>& e, int width, float (&to)[8]) {
  const T* p = (const T*)row + e.first;
  if (WHOLE) {
    const Eight<T> x = *(const Eight<T>*)p;
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j] = (float)x.v[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j] = e.first + j * e.step < width ? (float)p[j * e.step] : 0.f;      // (zeros behind the row's end)
  }
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void store_eight(char* row, const Piece<WHOLE>& e, int width, const float (&from)[8]) {
  T* p = (T*)row + e.first;
  if (WHOLE) {
    Eight<T> x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x.v[j] = (T)from[j];
    *(Eight<T>*)p = x;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) if (e.first + j * e.step < width) p[j * e.step] = (T)from[j];
  }
}
// four numbers as e4m3, to nearest even; a NaN stays one, and none is above 448 but by an fp32 rounding
__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// the largest of a group of 4, 8 or 16 lanes next to each other
__device__ __forceinline__ float group_max(float v, int lanes) {
  const auto with = [&](auto ctrl) { v = fmaxf(v, __uint_as_float(dpp_u32<decltype(ctrl)::value, 0xf>(0u, __float_as_uint(v)))); };
  with(std::integral_constant<int, C2T_DPP_QUAD_XOR1>{});
  with(std::integral_constant<int, C2T_DPP_QUAD_XOR2>{});
  if (lanes > 4) with(std::integral_constant<int, C2T_DPP_ROW_HALF_MIRROR>{});
  if (lanes > 8) with(std::integral_constant<int, C2T_DPP_ROW_MIRROR>{});
  return v;
}

// NT threads a row, which has at most 8 CH of its elements each.  WHOLE: rows are made of pieces that are aligned.
template <typename T, bool E4, int NT, int CH, bool WHOLE>
__global__ __launch_bounds__(NT < NORM_NT ? NORM_NT : NT) void k_rms_norm(NormArgs a) {
  constexpr int ROWS = NT < NORM_NT ? NORM_NT / NT : 1, WAVES = NT / WAVE;
  static_assert(NT == WAVE || ROWS == 1, "a wavefront a row, or the workgroup");
  __shared__ double sums[WAVES];
  __shared__ float tops[WAVES];
  const int t = threadIdx.x % NT, wave = t / WAVE;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / NT;
  if (row >= a.rows) return;                                 // (wavefronts of a workgroup that meet have the same row)
  const bool apart = !WHOLE && !(E4 && a.block != 0);        // (a block's largest is looked for among neighbouring pieces)
  const auto piece = [&](int c) { return apart ? Piece<WHOLE>{c * 8 * NT + t, NT} : Piece<WHOLE>{(c * NT + t) * 8, 1}; };
  float h[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) h[c][j] = 0.f;
    if (piece(c).first < a.width) load_eight<T>(a.x + row * a.x_row, piece(c), a.width, h[c]);
  }
  if (a.residual) {
    const char* const from = a.residual + row * a.residual_row;
    char* const to = a.residual_out + row * a.residual_out_row;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (piece(c).first >= a.width) continue;
      float r[8];
      if (a.residual_f32) load_eight<float>(from, piece(c), a.width, r); else load_eight<T>(from, piece(c), a.width, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[c][j] += r[j];
      if (a.residual_f32) store_eight<float>(to, piece(c), a.width, h[c]); else store_eight<T>(to, piece(c), a.width, h[c]);
    }
  }
  double sum = 0.;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = __builtin_fma((double)h[c][j], (double)h[c][j], sum);
  sum = wave_sum(sum);
  if (NT > WAVE) {
    if (t % WAVE == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) sum += sums[i];
  }
  const double r = 1. / sqrt(sum / (double)a.width + (double)a.eps);
  int power;
  const float part = (float)frexp(r, &power);

  float top = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (piece(c).first >= a.width) continue;
    float w[8];
    if (a.weight_f32) load_eight<float>(a.weight, piece(c), a.width, w); else load_eight<T>(a.weight, piece(c), a.width, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      h[c][j] = ldexpf(h[c][j], power) * part * w[j];
      if (E4) top = fmaxf(top, __builtin_fabsf(h[c][j]));
    }
    if (!E4) store_eight<T>(a.out + row * a.out_row, piece(c), a.width, h[c]);
  }
  if constexpr (E4) {
    if (a.block == 0) {
      top = wave_max(top);
      if (NT > WAVE) {
        if (t % WAVE == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) top = fmaxf(top, tops[i]);
      }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const Piece<WHOLE> e = piece(c);
      float m = top;
      if (a.block != 0) {
        m = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, __builtin_fabsf(h[c][j]));      // (zeros behind the row's end)
        m = group_max(m, a.block / 8);
      }
      if (e.first >= a.width) continue;
      const float scale = m == 0.f ? 1.f : fmaxf(m / E4M3_MAX, 0x1p-126f);
      if (a.block == 0 ? c == 0 && t == 0 : e.first % a.block == 0) a.scales[row * a.scales_row + (a.block == 0 ? 0 : e.first / a.block)] = scale;
      const float inv = 1.f / scale;
      // x / scale as one rounding makes it (Markstein: a product with the rounded reciprocal, corrected by what it leaves of x), or a number between two of 8 bits goes to the wrong one: the product alone
      // takes 4160 rows of 4096 1 % less, a division by the instruction set's steps 11 % more.
      const float back = inv == 0.f ? 0.f : scale;           // (of an infinite scale: what is finite is 0)
      const auto divided = [&](float x) { const float q = x * inv; return __builtin_fmaf(__builtin_fmaf(-q, back, x), inv, q); };
      uint2 y;
      y.x = four_e4m3(divided(h[c][0]), divided(h[c][1]), divided(h[c][2]), divided(h[c][3]));
      y.y = four_e4m3(divided(h[c][4]), divided(h[c][5]), divided(h[c][6]), divided(h[c][7]));
      char* const to = a.out + row * a.out_row + e.first;
      if (WHOLE) {
        *(uint2*)to = y;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (e.first + j * e.step < a.width) to[j * e.step] = (char)((j < 4 ? y.x : y.y) >> (j % 4 * 8));
      }
    }
  }
}

}  // namespace c2t
