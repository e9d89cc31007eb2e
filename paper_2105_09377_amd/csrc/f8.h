// 8-bit floats (e4m3) in blocks of 128 that share a scale in 32 bits, rows of them dealt to experts: what the kernels and the
// entry points share.
#pragma once

#include "mx4.h"

namespace gs {

constexpr int kF8Block = 128;        // numbers that share a scale
constexpr int kF8ScaleRun = 4;       // rows of scales are padded to multiples of this: 16 bytes
constexpr float kF8Most = 448.0f;    // the largest number of the type
constexpr float kF8LeastScale = 0x1p-126f;

__host__ __device__ inline int64_t f8_blocks(int64_t k) { return ceil_div(k, kF8Block); }
__host__ __device__ inline int64_t f8_scale_pitch(int64_t k) { return round_up(f8_blocks(k), kF8ScaleRun); }

// The scale of a block whose largest magnitude has these bits (of a float without its sign); NaN for infinities and NaN.
__device__ __forceinline__ float f8_scale(uint32_t top) {
  const float s = __uint_as_float(top) * (1.0f / kF8Most);
  return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : s > kF8LeastScale ? s : kF8LeastScale;
}
// Four floats -> four codes: times 1 / scale (which is below 2^127, and no number then above 448 (1 + 2^-22), which rounds to
// 448), rounded to the nearest code, ties to even.  A scale of NaN gives zeros.
__device__ __forceinline__ int32_t f8_encode4(const float* x, float factor) {
  int32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * factor, x[1] * factor, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * factor, x[3] * factor, w, true);
  return factor == factor ? w : 0;
}
__device__ __forceinline__ void f8_decode4(int32_t w, float scale, float* x) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  x[0] = a[0] * scale;
  x[1] = a[1] * scale;
  x[2] = b[0] * scale;
  x[3] = b[1] * scale;
}
// The largest of the bits of sixteen neighbouring lanes (a row of the wave).
__device__ __forceinline__ uint32_t max_of_16_lanes(uint32_t v) {
  uint32_t o = __builtin_amdgcn_mov_dpp(v, 0x128, 0xF, 0xF, true);     // turned by eight lanes, four, two, one
  v = v > o ? v : o;
  o = __builtin_amdgcn_mov_dpp(v, 0x124, 0xF, 0xF, true);
  v = v > o ? v : o;
  o = __builtin_amdgcn_mov_dpp(v, 0x122, 0xF, 0xF, true);
  v = v > o ? v : o;
  o = __builtin_amdgcn_mov_dpp(v, 0x121, 0xF, 0xF, true);
  return v > o ? v : o;
}
// Of the lanes that have a block's 128 numbers, N each.
template <int N>
__device__ __forceinline__ uint32_t f8_block_top(const float (&x)[N]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    top = top > b ? top : b;
  }
  top = max_of_16_lanes(top);
  if constexpr (N == 4) {
    const uint32_t o = __builtin_amdgcn_ds_swizzle(top, 0x401f);       // the other sixteen of 32
    top = top > o ? top : o;
  }
  return top;
}

struct F8ConvertArgs {    // matrices of `rows` rows of `cols` numbers <-> blocks of 1 or 128 rows
  void* plain;
  void* values;
  float* scales;
  int dtype;              // of the plain side
  int block_rows;
  int64_t mats, rows, cols;
};
hipError_t launch_f8_quantize(const F8ConvertArgs& a, hipStream_t s);
hipError_t launch_f8_dequantize(const F8ConvertArgs& a, hipStream_t s);

struct NormArgs {
  const void* x;
  const void* residual;   // may be null
  const void* weight;     // may be null
  void* sum;              // may be null
  void* out;              // numbers, or codes where there are scales
  float* scales;
  int dtype, w_dtype, out_dtype;
  float eps;
  int64_t rows, cols;
};
hipError_t launch_norm(const NormArgs& a, hipStream_t s);

struct F8DotArgs {        // out[m][n] = sum_b xs[m][b] ws[n / w_rows][b] sum_{k in b} x[m][k] w[n][k]
  const uint8_t* x;
  const float* xs;
  const uint8_t* w;
  const float* ws;
  void* out;
  int out_dtype, relu;
  int x_rows, w_rows;     // of a block: 1 or 128
  int64_t M, N, K;        // K a multiple of 128: codes behind the last number are zeros
  int64_t pitch;          // of rows of scales
  // experts: rows offsets[e] .. offsets[e + 1] - 1 of the result are of expert e's matrix; row r is of x's row tokens[r], or r
  const int32_t* offsets; // null: one matrix for all rows
  const int32_t* tokens;
  int64_t experts, x_count;            // x_count: rows of x
  int32_t splits;         // set by the launcher: workgroups that share the sum over K of a tile
};
// How a product is done.
enum F8DotWay { kF8Rows1, kF8Rows2, kF8Tile32x64, kF8Tile64x64, kF8Tile64x128, kF8Tile128x128Few, kF8Tile128x128, kF8Tile128x256, kF8Tile256x256 };
struct F8DotPlan {
  F8DotWay way;
  int splits;             // workgroups that share the sum of a tile
  size_t part_bytes;
};
F8DotPlan plan_f8_dot(int64_t M, int64_t N, int64_t K, int64_t experts);
hipError_t launch_f8_dot(const F8DotArgs& a, const F8DotPlan& p, void* workspace, hipStream_t s);

struct ExpertSortArgs {
  const int32_t* experts;
  int32_t* offsets;
  int32_t* tokens;
  int32_t* places;
  int32_t* counts;        // workspace of several workgroups
  int64_t n, choices, n_experts;
};
size_t expert_sort_workspace(int64_t n, int64_t n_experts);
hipError_t launch_expert_sort(const ExpertSortArgs& a, hipStream_t s);

struct ExpertRowsArgs {   // tokens (T, cols) <-> rows (count, cols) at places (T, choices)
  const void* flat;       // the tokens' side: what is spread out, or the gradient of what was joined
  void* flat_out;         // what is joined
  const void* rows;
  void* rows_out;
  const int32_t* places;
  const float* weights;   // may be null: ones
  float* grad_weights;
  int dtype, out_dtype;
  int64_t tokens, choices, cols, count;
};
hipError_t launch_expert_split(const ExpertRowsArgs& a, hipStream_t s);
hipError_t launch_expert_join(const ExpertRowsArgs& a, hipStream_t s);
hipError_t launch_expert_join_grad(const ExpertRowsArgs& a, hipStream_t s);

}  // namespace gs
