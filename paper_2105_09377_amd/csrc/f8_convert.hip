// Conversion to and from scaled 8-bit floats, and the root-mean-square norm whose result they are.
//
// A scale is its block's largest magnitude over 448, the largest number of e4m3.  A lane has 8 numbers, sixteen neighbouring
// lanes a row's 128; blocks of 128 rows are a workgroup's, 64 numbers per lane in registers, so that numbers are read once.
//
// Bound by memory.
#include "f8.h"
#include "pieces.h"

namespace gs {

namespace {

// 8 numbers of a row from element `at` on into memory, as far as `left` goes.
template <int DT>
__device__ __forceinline__ void store_8(void* row, int64_t at, int64_t left, const float (&x)[8]) {
  if constexpr (DT == GS_BF16) {
    uint16_t* dst = static_cast<uint16_t*>(row) + at;
    const i32x4 v = {int32_t(pack_bf16x2(x[0], x[1])), int32_t(pack_bf16x2(x[2], x[3])), int32_t(pack_bf16x2(x[4], x[5])), int32_t(pack_bf16x2(x[6], x[7]))};
    if (left >= 8) {
      __builtin_nontemporal_store((i32x4_any2)v, reinterpret_cast<i32x4_any2*>(dst));
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) dst[i] = uint16_t(uint32_t(v[i / 2]) >> (16 * (i & 1)));
    }
  } else {
    float* dst = static_cast<float*>(row) + at;
    if (left >= 8) {
#pragma unroll
      for (int h = 0; h < 2; ++h) __builtin_nontemporal_store((f32x4_any{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]}), reinterpret_cast<f32x4_any*>(dst + 4 * h));
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) dst[i] = x[i];
    }
  }
}

// Blocks of one row.  Pieces are counted up to whole blocks.
template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) f8_quantize_kernel(F8ConvertArgs a, Pieces<BIG> n) {
  using Index = typename Pieces<BIG>::Index;
  const Index cols = Index(a.cols), blocks = Index(f8_blocks(a.cols)), pitch = Index(f8_scale_pitch(a.cols));
  const Index base = Index(blockIdx.x) * (kThreads * P) + threadIdx.x;
  Index row[P], piece[P];
  float x[P][8];
  n.places(base, row, piece);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Index at = piece[p] * 8;
    load_numbers<DT, 8>(a.plain, int64_t(row[p] * cols + at), at + 8 <= cols ? 8 : at < cols ? int(cols - at) : 0, x[p]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const float scale = f8_scale(max_of_16_lanes(top_of_8(x[p])));
    if (base + p * kThreads >= n.total) continue;
    static_cast<i32x2*>(a.values)[row[p] * n.per_row + piece[p]] = f8_encode8(x[p], scale);
    if (piece[p] % 16 == 0) {
      const Index block = piece[p] / 16;
      float* const to = a.scales + (row[p] * pitch + block);
      *to = scale;
      if (block + 1 == blocks)
        for (Index i = 1; block + i < pitch; ++i) to[i] = 0.0f;
    }
  }
}

// Blocks of 128 rows: one of 128 x 128 numbers to a workgroup.
template <int DT>
__global__ void __launch_bounds__(kThreads) f8_quantize_square_kernel(F8ConvertArgs a, uint32_t row_blocks, uint32_t blocks) {
  const uint32_t mb = blockIdx.x / blocks, kb = blockIdx.x - mb * blocks, mat = mb / row_blocks, rb = mb - mat * row_blocks;
  const int lane16 = threadIdx.x & 15, r0 = threadIdx.x >> 4;
  const int64_t k = int64_t(kb) * kF8Block + lane16 * 8, left = a.cols - k, row0 = int64_t(mat) * a.rows + int64_t(rb) * 128;
  const int rows = a.rows - int64_t(rb) * 128 < 128 ? int(a.rows - int64_t(rb) * 128) : 128;
  float x[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    load_numbers<DT, 8>(a.plain, (row0 + (r < rows ? r : 0)) * a.cols + k, r < rows ? left : 0, x[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t t = top_of_8(x[i]);
    top = top > t ? top : t;
  }
  __shared__ uint32_t tops[kThreads / 16];
  top = max_of_16_lanes(top);
  if (lane16 == 0) tops[r0] = top;
  __syncthreads();
  const float scale = f8_scale(max_of_16_lanes(tops[lane16]));
  const int64_t pitch = int64_t(blocks) * kF8Block;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r < rows) *reinterpret_cast<i32x2*>(static_cast<uint8_t*>(a.values) + (row0 + r) * pitch + k) = f8_encode8(x[i], scale);
  }
  if (threadIdx.x == 0) {
    const int64_t run = round_up(blocks, kF8ScaleRun);
    float* const to = a.scales + int64_t(mb) * run;
    to[kb] = scale;
    if (kb + 1 == blocks)
      for (int64_t i = blocks; i < run; ++i) to[i] = 0.0f;
  }
}

// Rows as they are counted here are those of all matrices; a block of 128 rows ends with its matrix.
template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) f8_dequantize_kernel(F8ConvertArgs a, Pieces<BIG> n, FastDiv by_rows) {
  using Index = typename Pieces<BIG>::Index;
  const Index cols = Index(a.cols), pitch = Index(f8_scale_pitch(a.cols)), codes = Index(f8_blocks(a.cols)) * 16;
  const Index base = Index(blockIdx.x) * (kThreads * P) + threadIdx.x;
  Index row[P], piece[P];
  i32x2 w[P];
  float scale[P];
  n.places(base, row, piece);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    Index of = row[p];
    if (a.block_rows != 1) {
      Index mat = 0;
      if (a.mats > 1) {
        if constexpr (BIG) mat = row[p] / Index(a.rows);
        else mat = by_rows.div(row[p]);
      }
      of = mat * Index(ceil_div(a.rows, 128)) + (row[p] - mat * Index(a.rows)) / 128;
    }
    w[p] = static_cast<const i32x2*>(a.values)[row[p] * codes + piece[p]];
    scale[p] = a.scales[of * pitch + piece[p] / 16];
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (base + p * kThreads >= n.total) continue;
    const Index at = piece[p] * 8;
    float x[8];
    f8_decode8(w[p], scale[p], x);
    store_8<DT>(a.plain, int64_t(row[p] * cols + at), int64_t(cols - at), x);
  }
}

template <int DT, int P, bool BIG>
hipError_t launch_convert(const F8ConvertArgs& a, int64_t per_row, bool quantize, hipStream_t s) {
  const int64_t total = a.mats * a.rows * per_row, groups = ceil_div(total, kThreads * P);
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  using Index = typename Pieces<BIG>::Index;
  const Pieces<BIG> n{Index(per_row), Index(total), FastDiv::make(BIG ? 1u : uint32_t(per_row))};
  if (quantize) hipLaunchKernelGGL((f8_quantize_kernel<DT, P, BIG>), dim3(unsigned(groups)), dim3(kThreads), 0, s, a, n);
  else
    hipLaunchKernelGGL((f8_dequantize_kernel<DT, P, BIG>), dim3(unsigned(groups)), dim3(kThreads), 0, s, a, n,
                       FastDiv::make(BIG ? 1u : uint32_t(a.rows)));
  return hipGetLastError();
}
// Four pieces per lane where that still leaves eight workgroups for every compute unit.
template <int DT>
hipError_t convert(const F8ConvertArgs& a, int64_t per_row, bool quantize, hipStream_t s) {
  const int64_t total = a.mats * a.rows * per_row;
  if (total == 0) return hipSuccess;
  if (total > (int64_t(1) << 27)) return launch_convert<DT, 4, true>(a, per_row, quantize, s);
  if (total >= int64_t(256) * 8 * 4 * kThreads) return launch_convert<DT, 4, false>(a, per_row, quantize, s);
  return launch_convert<DT, 1, false>(a, per_row, quantize, s);
}

// ---------------------------------------------------------------------------------------------
// Norm: h = x + residual, rounded to their type; y = h / sqrt(mean(h^2) + eps) weight.
// ---------------------------------------------------------------------------------------------

// 8 numbers as bfloat16 keeps them.
__device__ __forceinline__ void round_8(float (&x)[8], std::integral_constant<int, GS_BF16>) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    x[2 * i] = __uint_as_float(w << 16);
    x[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
  }
}
__device__ __forceinline__ void round_8(float (&)[8], std::integral_constant<int, GS_F32>) {}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
  return v;
}

// WAVES waves have a row, or one wave each of four; NP pieces of 8 numbers per lane stay in registers between the sum and the
// result (NP 0: rows of any length, read twice).
template <int DT, int OUT, int WAVES, int NP>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) norm_kernel(NormArgs a) {
  constexpr int T = WAVES * 64;
  __shared__ float part[WAVES];
  const int64_t row = WAVES == 1 ? int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  if (row >= a.rows) return;          // (a whole wave, and there is no barrier with one wave per row)
  const int64_t base = row * a.cols, blocks = f8_blocks(a.cols), pieces = OUT == GS_F8 ? blocks * 16 : ceil_div(a.cols, 8);
  auto load = [&](int64_t piece, float (&h)[8]) {
    const int64_t at = piece * 8, left = a.cols - at;
    load_numbers<DT, 8>(a.x, base + at, left, h);
    if (a.residual) {
      float r[8];
      load_numbers<DT, 8>(a.residual, base + at, left, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += r[i];
      round_8(h, std::integral_constant<int, DT>{});
    }
  };
  auto squares = [&](int64_t piece, const float (&h)[8]) {
    if (a.sum && piece * 8 < a.cols) store_8<DT>(a.sum, base + piece * 8, a.cols - piece * 8, h);
    float s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += h[i] * h[i];
    return s;
  };
  auto finish = [&](int64_t piece, float (&h)[8], float r) {
    const int64_t at = piece * 8, left = a.cols - at;
    float w[8];
    if (a.weight) {
      if (a.w_dtype == GS_BF16) load_numbers<GS_BF16, 8>(a.weight, at, left, w);
      else load_numbers<GS_F32, 8>(a.weight, at, left, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = h[i] * r * w[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] *= r;
    }
    if constexpr (OUT == GS_F8) {
      // (what a row has behind its end is zero: infinities of r must not make it NaN)
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = i < left ? h[i] : 0.0f;
      const float scale = f8_scale(max_of_16_lanes(top_of_8(h)));
      if (piece >= pieces) return;
      static_cast<i32x2*>(a.out)[row * pieces + piece] = f8_encode8(h, scale);
      if (piece % 16 == 0) {
        const int64_t block = piece / 16, run = round_up(blocks, kF8ScaleRun);
        float* const to = a.scales + (row * run + block);
        *to = scale;
        if (block + 1 == blocks)
          for (int64_t i = blocks; i < run; ++i) to[i - block] = 0.0f;
      }
    } else {
      if (piece < pieces) store_8<OUT>(a.out, base + at, left, h);
    }
  };
  float sum = 0;
  if constexpr (NP > 0) {
    float h[NP][8];
#pragma unroll
    for (int p = 0; p < NP; ++p) load(t + p * T, h[p]);
#pragma unroll
    for (int p = 0; p < NP; ++p) sum += squares(t + p * T, h[p]);
    sum = wave_sum(sum);
    if constexpr (WAVES > 1) {
      if ((t & 63) == 0) part[t >> 6] = sum;
      __syncthreads();
      sum = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += part[w];
    }
    const float r = 1.0f / sqrtf(sum / float(a.cols) + a.eps);
#pragma unroll
    for (int p = 0; p < NP; ++p) finish(t + p * T, h[p], r);
  } else {
    const int64_t end = round_up(pieces, T);         // (all lanes of a block's sixteen, whatever the row's length)
    for (int64_t piece = t; piece < end; piece += T) {
      float h[8];
      load(piece, h);
      sum += squares(piece, h);
    }
    sum = wave_sum(sum);
    if ((t & 63) == 0) part[t >> 6] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += part[w];
    const float r = 1.0f / sqrtf(sum / float(a.cols) + a.eps);
    for (int64_t piece = t; piece < end; piece += T) {
      float h[8];
      load(piece, h);
      finish(piece, h, r);
    }
  }
}

template <int DT, int OUT, int WAVES, int NP>
hipError_t launch_norm_as(const NormArgs& a, hipStream_t s) {
  const int64_t groups = WAVES == 1 ? ceil_div(a.rows, 4) : a.rows;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((norm_kernel<DT, OUT, WAVES, NP>), dim3(unsigned(groups)), dim3(WAVES == 1 ? 256 : WAVES * 64), 0, s, a);
  return hipGetLastError();
}
template <int DT, int OUT>
hipError_t norm(const NormArgs& a, hipStream_t s) {
  const int64_t pieces = OUT == GS_F8 ? f8_blocks(a.cols) * 16 : ceil_div(a.cols, 8);
  if (pieces <= 64) return launch_norm_as<DT, OUT, 1, 1>(a, s);
  if (pieces <= 128) return launch_norm_as<DT, OUT, 1, 2>(a, s);
  if (pieces <= 256) return launch_norm_as<DT, OUT, 4, 1>(a, s);
  if (pieces <= 512) return launch_norm_as<DT, OUT, 4, 2>(a, s);
  if (pieces <= 1024) return launch_norm_as<DT, OUT, 4, 4>(a, s);
  if (pieces <= 2048) return launch_norm_as<DT, OUT, 8, 4>(a, s);
  return launch_norm_as<DT, OUT, 16, 0>(a, s);
}

}  // namespace

hipError_t launch_f8_quantize(const F8ConvertArgs& a, hipStream_t s) {
  if (a.block_rows == 1) {
    const int64_t per_row = f8_blocks(a.cols) * 16;
    return a.dtype == GS_BF16 ? convert<GS_BF16>(a, per_row, true, s) : convert<GS_F32>(a, per_row, true, s);
  }
  const int64_t row_blocks = ceil_div(a.rows, 128), blocks = f8_blocks(a.cols), groups = a.mats * row_blocks * blocks;
  if (groups == 0) return hipSuccess;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid{unsigned(groups)}, block(kThreads);
  if (a.dtype == GS_BF16) hipLaunchKernelGGL((f8_quantize_square_kernel<GS_BF16>), grid, block, 0, s, a, uint32_t(row_blocks), uint32_t(blocks));
  else hipLaunchKernelGGL((f8_quantize_square_kernel<GS_F32>), grid, block, 0, s, a, uint32_t(row_blocks), uint32_t(blocks));
  return hipGetLastError();
}
hipError_t launch_f8_dequantize(const F8ConvertArgs& a, hipStream_t s) {
  const int64_t per_row = ceil_div(a.cols, 8);
  return a.dtype == GS_BF16 ? convert<GS_BF16>(a, per_row, false, s) : convert<GS_F32>(a, per_row, false, s);
}

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  if (a.rows == 0 || a.cols == 0) return hipSuccess;
  if (a.dtype == GS_BF16) {
    if (a.scales) return norm<GS_BF16, GS_F8>(a, s);
    return a.out_dtype == GS_BF16 ? norm<GS_BF16, GS_BF16>(a, s) : norm<GS_BF16, GS_F32>(a, s);
  }
  if (a.scales) return norm<GS_F32, GS_F8>(a, s);
  return a.out_dtype == GS_BF16 ? norm<GS_F32, GS_BF16>(a, s) : norm<GS_F32, GS_F32>(a, s);
}

}  // namespace gs
