// Microscaled 4-bit floats: what the kernels and the entry points share.
#pragma once

#include "common.h"

namespace gs {

constexpr int kMx4Block = 32;        // numbers that share a scale; 16 bytes
constexpr int kMx4ScaleRun = 8;      // rows of scale bytes are padded to multiples of this

typedef float f32x4 __attribute__((ext_vector_type(4)));

__host__ __device__ inline int64_t mx4_blocks(int64_t k) { return ceil_div(k, kMx4Block); }
__host__ __device__ inline int64_t mx4_scale_pitch(int64_t k) { return round_up(mx4_blocks(k), kMx4ScaleRun); }

// 2^(byte - 127); byte 0 is a subnormal, 255 NaN.
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
  uint32_t u = byte << 23;
  u = byte == 0 ? 0x00400000u : u;
  return __uint_as_float(byte == 255 ? 0x7fc00000u : u);
}
// The scale byte of a block whose largest magnitude has these bits (of a float without its sign).
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const uint32_t e = top >> 23;       // floor(log2) + 127; 0 for subnormals, whose scale is the smallest too
  return e > 2 ? e - 2 : 0;
}
// Eight floats -> eight codes in a dword.  The conversion rounds to the nearest code, ties to even, and saturates; a
// scale of NaN gives code zero (the block's numbers are NaN through the scale).
__device__ __forceinline__ uint32_t mx4_encode8(const float (&x)[8], uint32_t scale_byte) {
  const float s = mx4_scale(scale_byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  return scale_byte == 255 ? 0u : w;
}
// Codes of byte SEL of w, times the scale, as two bfloat16 (exact within bfloat16's range).
template <int SEL>
__device__ __forceinline__ uint32_t mx4_decode2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}
// Eight codes -> eight bfloat16.
__device__ __forceinline__ i32x4 mx4_decode8(uint32_t w, float scale) {
  return i32x4{int32_t(mx4_decode2<0>(w, scale)), int32_t(mx4_decode2<1>(w, scale)), int32_t(mx4_decode2<2>(w, scale)),
               int32_t(mx4_decode2<3>(w, scale))};
}
template <int SEL>
__device__ __forceinline__ void mx4_decode2_f32(uint32_t w, float scale, float* out) {
  const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, SEL);
  out[0] = v[0];
  out[1] = v[1];
}

// The largest of the bits of four neighbouring lanes.
__device__ __forceinline__ uint32_t max_of_4_lanes(uint32_t v) {
  uint32_t o = __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true);      // lanes 1 0 3 2
  v = v > o ? v : o;
  o = __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);               // lanes 2 3 0 1
  return v > o ? v : o;
}

// Where a cache keeps a token; offsets in bytes from the beginning of a (page, head) block.
struct Mx4CacheShape {
  uint8_t* data;
  int64_t n_pages;
  int32_t page, heads, dim;
  FastDiv by_page;
  __host__ __device__ int blocks() const { return dim / kMx4Block; }
  __host__ __device__ int64_t block_bytes() const { return int64_t(page) * dim + int64_t(2) * page * blocks(); }
  __device__ uint8_t* block(int64_t page_id, int head) const { return data + (page_id * heads + head) * block_bytes(); }
  __device__ uint32_t key(uint32_t slot) const { return slot * uint32_t(dim / 2); }
  __device__ uint32_t value(uint32_t slot, uint32_t piece) const {       // piece: 8 numbers
    return uint32_t(page) * uint32_t(dim / 2) + ((slot / 4 * uint32_t(dim / 8) + piece) * 4 + slot % 4) * 4;
  }
  __device__ uint32_t key_scale(uint32_t slot, uint32_t block) const { return uint32_t(page) * uint32_t(dim) + slot * uint32_t(blocks()) + block; }
  __device__ uint32_t value_scale(uint32_t slot, uint32_t block) const {
    return uint32_t(page) * uint32_t(dim + blocks()) + (slot / 4 * uint32_t(blocks()) + block) * 4 + slot % 4;
  }
};

struct Mx4ConvertArgs {   // rows of `cols` numbers <-> blocks
  void* plain;
  void* values;
  void* scales;
  int dtype;              // of the plain side
  int64_t rows, cols;
};
hipError_t launch_mx4_quantize(const Mx4ConvertArgs& a, hipStream_t s);
hipError_t launch_mx4_dequantize(const Mx4ConvertArgs& a, hipStream_t s);

struct Mx4TokenArgs {     // tokens (batch, T, heads, dim) <-> cache
  Mx4CacheShape cache;
  const int32_t* table;   // (batch, width)
  const int32_t* first;
  const int32_t* counts;  // may be null
  void* k;
  void* v;
  int dtype;
  int64_t batch, width, tokens;
};
hipError_t launch_mx4_append(const Mx4TokenArgs& a, hipStream_t s);
hipError_t launch_mx4_read(const Mx4TokenArgs& a, hipStream_t s);

struct Mx4DotArgs {       // out[m][n] = sum_k x[m][k] w[n][k]
  const void* x;          // MX4 values, or bf16 rows of K
  const uint8_t* xs;      // MX4 scales, null for bf16
  const void* w;
  const uint8_t* ws;
  void* out;
  int out_dtype, relu;
  int64_t M, N, K;
  int32_t splits;         // set by the launcher: workgroups that share the sum over K of a tile; above 1, `out` has as many
                          // results in fp32, one after the other
};
// How a product is done.
enum Mx4DotWay { kRows1, kRows2, kTile64x64Few, kTile64x64, kTile128x128Few, kTile128x128Long, kTile128x128, kTile256x256,   // two MX4 operands
                 kWeight32x128, kWeight64x64, kWeight64x128, kWeight128x128, kWeight128x256 };
struct Mx4DotPlan {
  Mx4DotWay way;
  int splits;             // workgroups that share the sum of a tile
  int64_t ldx;            // bfloat16 x in tiles: numbers between rows
  bool pad;               // into the workspace first
  size_t pad_bytes, part_bytes;
  size_t workspace() const { return pad_bytes + part_bytes; }
};
Mx4DotPlan plan_mx4_dot(bool x_is_bf16, int64_t M, int64_t N, int64_t K);
hipError_t launch_mx4_dot(const Mx4DotArgs& a, const Mx4DotPlan& plan, void* workspace, hipStream_t s);

struct Mx4AttendArgs {
  Mx4CacheShape cache;
  const int32_t* table;   // (batch, width)
  const int32_t* lengths;
  const void* q;
  void* out;
  float* partial;         // workspace of the parts, null where there is one
  int out_dtype;
  float scale;
  int64_t window, sinks;  // window 0: everything
  int64_t batch, width;
  int32_t queries, group;
  int32_t parts, tiles;   // set by the launcher: workgroups along a sequence; 16-row tiles of a workgroup;
  int32_t least;          // 64-token tiles of a part
  FastDiv by_group, by_rows, by_heads, by_parts;      // rows: queries * group
  int32_t slots;          // parts of all sequences together where they are cut to the same length, else 0
};
// How an attention is done.
struct Mx4AttendPlan {
  int rows, waves;        // of a workgroup
  int parts, slots;       // of a sequence at most; of all sequences together where they are cut to the same length, else 0
  bool joined_alone;      // a row's parts have a workgroup to join them
};
Mx4AttendPlan mx4_attend_plan(const Mx4AttendArgs& a);
hipError_t launch_mx4_attend(const Mx4AttendArgs& a, hipStream_t s);
size_t mx4_attend_workspace(const Mx4AttendArgs& a);

}  // namespace gs
