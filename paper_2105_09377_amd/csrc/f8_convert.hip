// Conversion to and from scaled 8-bit floats, and the root-mean-square norm whose result they are.
//
// A scale is its block's largest magnitude over 448, the largest number of e4m3.  A lane has 16 bytes of numbers, so that a wave's access is 1 KB
// of a row: sixteen neighbouring lanes have 128 of bfloat16, 32 those of floats.  Blocks of 128 rows are a workgroup's, 64 numbers per lane
// in registers, so that numbers are read once.
//
// Bound by memory: 16384 x 8192 floats to codes with a scale for 128 rows 103 us, 6.5 TB/s, and back 95, 7.0; bfloat16 62 and 58; 16380 x 8190
// floats, whose rows begin on 8 bytes, 133 and 96; the norm of 16384 x 8192 bfloat16 numbers with a residual 160, 5.9 TB/s.
#include "f8.h"
#include "pieces.h"

namespace gs {

namespace {

// The codes of a lane's numbers.
template <int N>
using Codes = std::conditional_t<N == 8, i32x2, int32_t>;
template <int N>
__device__ __forceinline__ Codes<N> encode(const float (&x)[N], float scale) {
  const float f = 1.0f / scale;
  if constexpr (N == 8) return i32x2{f8_encode4(x, f), f8_encode4(x + 4, f)};
  else return f8_encode4(x, f);
}
template <int N>
__device__ __forceinline__ void decode(const Codes<N>& w, float scale, float (&x)[N]) {
  if constexpr (N == 8) {
    f8_decode4(w[0], scale, x);
    f8_decode4(w[1], scale, x + 4);
  } else {
    f8_decode4(w, scale, x);
  }
}

// Blocks of one row.  Pieces are counted up to whole blocks.
template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) f8_quantize_kernel(F8ConvertArgs a, Pieces<BIG> n) {
  using Index = typename Pieces<BIG>::Index;
  constexpr int N = kNumbers<DT>, kLanes = kF8Block / N;
  const Index cols = Index(a.cols), blocks = Index(f8_blocks(a.cols)), pitch = Index(f8_scale_pitch(a.cols));
  const Index base = Index(blockIdx.x) * (kThreads * P) + threadIdx.x;
  Index row[P], piece[P];
  float x[P][N];
  n.places(base, row, piece);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Index at = piece[p] * N;
    load_row_numbers<DT, N>(a.plain, int64_t(row[p] * cols + at), at + N <= cols ? N : at < cols ? int(cols - at) : 0, x[p]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const float scale = f8_scale(f8_block_top(x[p]));
    if (base + p * kThreads >= n.total) continue;
    static_cast<Codes<N>*>(a.values)[row[p] * n.per_row + piece[p]] = encode(x[p], scale);
    if (piece[p] % kLanes == 0) {
      const Index block = piece[p] / kLanes;
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
  constexpr int N = kNumbers<DT>, kLanes = kF8Block / N, kRows = kThreads / kLanes, I = 128 / kRows;
  const uint32_t mb = blockIdx.x / blocks, kb = blockIdx.x - mb * blocks, mat = mb / row_blocks, rb = mb - mat * row_blocks;
  const int piece = threadIdx.x % kLanes, r0 = threadIdx.x / kLanes;
  const int64_t k = int64_t(kb) * kF8Block + piece * N, left = a.cols - k, row0 = int64_t(mat) * a.rows + int64_t(rb) * 128;
  const int rows = a.rows - int64_t(rb) * 128 < 128 ? int(a.rows - int64_t(rb) * 128) : 128;
  float x[I][N];
#pragma unroll
  for (int i = 0; i < I; ++i) {
    const int r = r0 + kRows * i;
    load_row_numbers<DT, N>(a.plain, (row0 + (r < rows ? r : 0)) * a.cols + k, r < rows ? left : 0, x[i]);
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t b = __float_as_uint(x[i][j]) & 0x7fffffffu;
      top = top > b ? top : b;
    }
  __shared__ uint32_t tops[kThreads / 16];
  top = max_of_16_lanes(top);
  if (threadIdx.x % 16 == 0) tops[threadIdx.x / 16] = top;
  __syncthreads();
  static_assert(kThreads / 16 == 16, "a row of lanes has them all");
  const float scale = f8_scale(max_of_16_lanes(tops[threadIdx.x % 16]));
  const int64_t pitch = int64_t(blocks) * kF8Block;
#pragma unroll
  for (int i = 0; i < I; ++i) {
    const int r = r0 + kRows * i;
    if (r < rows) *reinterpret_cast<Codes<N>*>(static_cast<uint8_t*>(a.values) + (row0 + r) * pitch + k) = encode(x[i], scale);
  }
  if (threadIdx.x == 0) {
    const int64_t run = round_up(blocks, kF8ScaleRun);
    float* const to = a.scales + int64_t(mb) * run;
    to[kb] = scale;
    if (kb + 1 == blocks)
      for (int64_t i = blocks; i < run; ++i) to[i] = 0.0f;
  }
}

// The row of scales of a row, rows being counted over all matrices; a block of 128 rows ends with its matrix.
template <bool BIG, typename Index>
__device__ __forceinline__ Index scale_row(const F8ConvertArgs& a, Index row, const FastDiv& by_rows) {
  if (a.block_rows == 1) return row;
  Index mat = 0;
  if (a.mats > 1) {
    if constexpr (BIG) mat = row / Index(a.rows);
    else mat = by_rows.div(row);
  }
  return mat * Index(ceil_div(a.rows, 128)) + (row - mat * Index(a.rows)) / 128;
}

template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) f8_dequantize_kernel(F8ConvertArgs a, Pieces<BIG> n, FastDiv by_rows) {
  using Index = typename Pieces<BIG>::Index;
  constexpr int N = kNumbers<DT>, kLanes = kF8Block / N;
  const Index cols = Index(a.cols), pitch = Index(f8_scale_pitch(a.cols)), codes = Index(f8_blocks(a.cols)) * kLanes;
  const Index base = Index(blockIdx.x) * (kThreads * P) + threadIdx.x;
  Index row[P], piece[P];
  Codes<N> w[P];
  float scale[P];
  n.places(base, row, piece);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    w[p] = static_cast<const Codes<N>*>(a.values)[row[p] * codes + piece[p]];
    scale[p] = a.scales[scale_row<BIG>(a, row[p], by_rows) * pitch + piece[p] / kLanes];
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (base + p * kThreads >= n.total) continue;
    const Index at = piece[p] * N;
    float x[N];
    decode<N>(w[p], scale[p], x);
    store_row_numbers<DT, N>(a.plain, int64_t(row[p] * cols + at), int64_t(cols - at), x);
  }
}

// Back into rows that do not all begin on 16 bytes: pieces are those of the result's memory, so that whole lines are written.  A piece may have
// numbers of two blocks; one with numbers of two rows is written number by number.  There are cols >= N numbers in a row, n.per_row of
// them.
template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) f8_dequantize_flat_kernel(F8ConvertArgs a, Pieces<BIG> n, FastDiv by_rows) {
  using Index = typename Pieces<BIG>::Index;
  constexpr int N = kNumbers<DT>;
  using CodesAny = std::conditional_t<N == 8, i32x2_any, i32_any>;
  const Index cols = n.per_row, pitch = Index(f8_scale_pitch(a.cols)), row_codes = Index(f8_blocks(a.cols)) * kF8Block;
  const Index base = (Index(blockIdx.x) * (kThreads * P) + threadIdx.x) * N;
  const uint8_t* const values = static_cast<const uint8_t*>(a.values);
  Index row[P], first[P];             // of the piece's first number
  Codes<N> w[P];
  float scale[P][2];
  int border[P];                      // numbers from here on are of the second block
#pragma unroll
  for (int p = 0; p < P; ++p) {
    n.divide(base + p * (kThreads * N) < n.total ? base + p * (kThreads * N) : 0, &row[p], &first[p]);
    const Index last = first[p] + N <= cols ? first[p] + N - 1 : cols - 1, at = first[p] + N <= row_codes ? first[p] : row_codes - N;
    w[p] = *reinterpret_cast<const CodesAny*>(values + (row[p] * row_codes + at));
    const float* const scales = a.scales + scale_row<BIG>(a, row[p], by_rows) * pitch;
    scale[p][0] = scales[first[p] / kF8Block];
    scale[p][1] = scales[last / kF8Block];
    border[p] = int(last / kF8Block * kF8Block) - int(first[p]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Index number = base + p * (kThreads * N);
    if (number >= n.total) continue;
    if (first[p] + N > cols) {
#pragma unroll 1
      for (int i = 0; i < N && number + i < n.total; ++i) {
        const bool wraps = first[p] + i >= cols;
        const Index r = wraps ? row[p] + 1 : row[p], c = wraps ? first[p] + i - cols : first[p] + i;
        float four[4];
        f8_decode4(values[r * row_codes + c], a.scales[scale_row<BIG>(a, r, by_rows) * pitch + c / kF8Block], four);
        if constexpr (DT == GS_BF16) static_cast<uint16_t*>(a.plain)[number + i] = float_to_bf16_bits(four[0]);
        else static_cast<float*>(a.plain)[number + i] = four[0];
      }
      continue;
    }
    float x[N], y[N];
    decode<N>(w[p], scale[p][0], x);
    decode<N>(w[p], scale[p][1], y);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < border[p] ? x[i] : y[i];
    store_row_numbers<DT, N>(a.plain, int64_t(number), N, x);
  }
}

enum Convert { kQuantize, kDequantize, kDequantizeFlat };
template <int DT, int P, bool BIG>
hipError_t launch_convert(const F8ConvertArgs& a, int64_t per_row, Convert what, hipStream_t s) {
  // (the flat kernel counts numbers, the others pieces)
  const bool flat = what == kDequantizeFlat;
  const int64_t rows = a.mats * a.rows, step = flat ? a.cols : per_row, total = rows * step;
  const int64_t groups = ceil_div(total, kThreads * P * (flat ? kNumbers<DT> : 1));
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  using Index = typename Pieces<BIG>::Index;
  const Pieces<BIG> n{Index(step), Index(total), FastDiv::make(BIG ? 1u : uint32_t(step))};
  const FastDiv by_rows = FastDiv::make(BIG ? 1u : uint32_t(a.rows));
  const dim3 grid{unsigned(groups)}, block(kThreads);
  if (what == kQuantize) hipLaunchKernelGGL((f8_quantize_kernel<DT, P, BIG>), grid, block, 0, s, a, n);
  else if (what == kDequantize) hipLaunchKernelGGL((f8_dequantize_kernel<DT, P, BIG>), grid, block, 0, s, a, n, by_rows);
  else hipLaunchKernelGGL((f8_dequantize_flat_kernel<DT, P, BIG>), grid, block, 0, s, a, n, by_rows);
  return hipGetLastError();
}
// Four pieces per lane where that still leaves eight workgroups for every compute unit.
template <int DT>
hipError_t convert(const F8ConvertArgs& a, int64_t per_row, Convert what, hipStream_t s) {
  const int64_t total = a.mats * a.rows * per_row;
  if (total == 0) return hipSuccess;
  // (a row has 512 bytes of scales and codes at least, whatever its length: places are counted in 32 bits up to 2^22 rows)
  if (total > (int64_t(1) << 30) / kNumbers<DT> || a.mats * a.rows > (int64_t(1) << 22)) return launch_convert<DT, 4, true>(a, per_row, what, s);
  if (total >= int64_t(256) * 8 * 4 * kThreads) return launch_convert<DT, 4, false>(a, per_row, what, s);
  return launch_convert<DT, 1, false>(a, per_row, what, s);
}
template <int DT>
hipError_t quantize(const F8ConvertArgs& a, hipStream_t s) {
  return convert<DT>(a, f8_blocks(a.cols) * (kF8Block / kNumbers<DT>), kQuantize, s);
}
template <int DT>
hipError_t dequantize(const F8ConvertArgs& a, hipStream_t s) {
  constexpr int N = kNumbers<DT>;
  return convert<DT>(a, ceil_div(a.cols, N), a.cols % N == 0 || a.mats * a.rows <= 1 || a.cols < 128 ? kDequantize : kDequantizeFlat, s);
}

// ---------------------------------------------------------------------------------------------
// Norm: h = x + residual, rounded to their type; y = h / sqrt(mean(h^2) + eps) weight.
//
// Squares, their sum, the root and y before it is rounded to float are 64 bits: there no square overflows, and y is the float nearest to its
// definition whatever the order of the sum, so that numbers on a border between two codes, which products of bfloat16 numbers often are, get
// the code that the definition gives them (in 32 bits 6 of 100000 had the other one).
// ---------------------------------------------------------------------------------------------

// A lane's 8 numbers of a row between the sum and the result, as they are stored.
template <int DT>
struct Kept;
template <>
struct Kept<GS_BF16> {
  i32x4 v;
  __device__ void put(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = int32_t(pack_bf16x2(x[2 * i], x[2 * i + 1]));
  }
  __device__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(uint32_t(v[i]) << 16);
      x[2 * i + 1] = __uint_as_float(uint32_t(v[i]) & 0xffff0000u);
    }
  }
};
template <>
struct Kept<GS_F32> {
  float v[8];
  __device__ void put(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
  }
  __device__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i];
  }
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ double inverse_root(double d) {
  const double r = __builtin_amdgcn_rsq(d);
  if (!(d > 0.0) || d == __builtin_huge_val()) return r;
  const double half = 0.5 * d, s = r * (1.5 - half * r * r);       // (26 bits, then 50, then all)
  return s * (1.5 - half * s * s);
}

// WAVES waves have a row, or one wave each of four; NP pieces of 8 numbers per lane stay in registers between the sum and the
// result (NP 0: rows of any length, read twice).
template <int DT, int OUT, int WAVES, int NP>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) norm_kernel(NormArgs a) {
  constexpr int T = WAVES * 64;
  __shared__ double part[WAVES];
  const int64_t row = WAVES == 1 ? int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
  const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  if (row >= a.rows) return;          // (a whole wave, and there is no barrier with one wave per row)
  const int64_t base = row * a.cols, blocks = f8_blocks(a.cols), pieces = OUT == GS_F8 ? blocks * 16 : ceil_div(a.cols, 8);
  auto load = [&](int64_t piece, Kept<DT>& kept) {
    const int64_t at = piece * 8, left = a.cols - at;
    float h[8];
    load_row_numbers<DT, 8>(a.x, base + at, left, h);
    if (a.residual) {
      float r[8];
      load_row_numbers<DT, 8>(a.residual, base + at, left, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += r[i];
    }
    kept.put(h);
  };
  auto squares = [&](int64_t piece, const Kept<DT>& kept) {
    float h[8];
    kept.get(h);
    if (a.sum && piece * 8 < a.cols) store_row_numbers<DT, 8>(a.sum, base + piece * 8, a.cols - piece * 8, h);
    double s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fma(double(h[i]), double(h[i]), s);
    return s;
  };
  auto finish = [&](int64_t piece, const Kept<DT>& kept, double r) {
    const int64_t at = piece * 8, left = a.cols - at;
    float h[8], w[8];
    kept.get(h);
    if (a.weight) {
      if (a.w_dtype == GS_BF16) load_row_numbers<GS_BF16, 8, false>(a.weight, at, left, w);
      else load_row_numbers<GS_F32, 8, false>(a.weight, at, left, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = float(double(h[i]) * r * double(w[i]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = float(double(h[i]) * r);
    }
    if constexpr (OUT == GS_F8) {
      // (what a row has behind its end is zero: infinities of r must not make it NaN)
      if (left < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i < left ? h[i] : 0.0f;
      const float scale = f8_scale(f8_block_top(h));
      if (piece >= pieces) return;
      static_cast<i32x2*>(a.out)[row * pieces + piece] = encode(h, scale);
      if (piece % 16 == 0) {
        const int64_t block = piece / 16, run = round_up(blocks, kF8ScaleRun);
        float* const to = a.scales + (row * run + block);
        *to = scale;
        if (block + 1 == blocks)
          for (int64_t i = blocks; i < run; ++i) to[i - block] = 0.0f;
      }
    } else {
      if (piece < pieces) store_row_numbers<OUT, 8>(a.out, base + at, left, h);
    }
  };
  double sum = 0;
  if constexpr (NP > 0) {
    Kept<DT> h[NP];
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
    const double r = inverse_root(sum / double(a.cols) + double(a.eps));
#pragma unroll
    for (int p = 0; p < NP; ++p) finish(t + p * T, h[p], r);
  } else {
    const int64_t end = round_up(pieces, T);         // (all lanes of a block's sixteen, whatever the row's length)
    for (int64_t piece = t; piece < end; piece += T) {
      Kept<DT> h;
      load(piece, h);
      sum += squares(piece, h);
    }
    sum = wave_sum(sum);
    if ((t & 63) == 0) part[t >> 6] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += part[w];
    const double r = inverse_root(sum / double(a.cols) + double(a.eps));
    for (int64_t piece = t; piece < end; piece += T) {
      Kept<DT> h;
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
  // Two pieces per lane, whose loads are all under way and whose registers leave room for eight waves on a SIMD (16384 x 8192 bfloat16 with a
  // residual: 165 us, four pieces in half the waves 191, one in twice as many 188; 4096 x 16384 86, 111 with four); one where there are no more
  // rows than compute units (256 x 4096 5.0 and 6.1).
  if (pieces <= 64) return launch_norm_as<DT, OUT, 1, 1>(a, s);
  if (pieces <= 128) return launch_norm_as<DT, OUT, 1, 2>(a, s);
  if (pieces <= 256) return launch_norm_as<DT, OUT, 4, 1>(a, s);
  if (pieces <= 1024 && a.rows <= 256) return launch_norm_as<DT, OUT, 16, 1>(a, s);
  if (pieces <= 512) return launch_norm_as<DT, OUT, 4, 2>(a, s);
  if (pieces <= 1024) return launch_norm_as<DT, OUT, 8, 2>(a, s);
  if (pieces <= 2048) return launch_norm_as<DT, OUT, 16, 2>(a, s);
  if (pieces <= 4096) return launch_norm_as<DT, OUT, 16, 4>(a, s);
  return launch_norm_as<DT, OUT, 16, 0>(a, s);
}

}  // namespace

hipError_t launch_f8_quantize(const F8ConvertArgs& a, hipStream_t s) {
  if (a.block_rows == 1) return a.dtype == GS_BF16 ? quantize<GS_BF16>(a, s) : quantize<GS_F32>(a, s);
  const int64_t row_blocks = ceil_div(a.rows, 128), blocks = f8_blocks(a.cols), groups = a.mats * row_blocks * blocks;
  if (groups == 0) return hipSuccess;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid{unsigned(groups)}, block(kThreads);
  if (a.dtype == GS_BF16) hipLaunchKernelGGL((f8_quantize_square_kernel<GS_BF16>), grid, block, 0, s, a, uint32_t(row_blocks), uint32_t(blocks));
  else hipLaunchKernelGGL((f8_quantize_square_kernel<GS_F32>), grid, block, 0, s, a, uint32_t(row_blocks), uint32_t(blocks));
  return hipGetLastError();
}
hipError_t launch_f8_dequantize(const F8ConvertArgs& a, hipStream_t s) { return a.dtype == GS_BF16 ? dequantize<GS_BF16>(a, s) : dequantize<GS_F32>(a, s); }

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
