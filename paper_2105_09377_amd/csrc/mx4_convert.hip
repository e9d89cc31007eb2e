// Conversion to and from microscaled 4-bit floats: whole matrices, and tokens of a paged cache.
//
// A scale is the power of two of its block's largest magnitude, over 4 (the largest power of two of e2m1),
// so a block is read once, reduced over its 32 numbers, and written: 16 bytes of numbers per lane where they lie in rows, four (bfloat16) or
// eight (floats) neighbouring lanes per block, the maximum over them by lane exchanges; 8 numbers per lane of a cache's tokens.  Bound by memory: n numbers of s bytes move n (s + 17/32).
#include "mx4.h"

namespace gs {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_plain(const void* p, int64_t i, std::integral_constant<int, GS_BF16>) {
  return bf16_bits_to_float(static_cast<const uint16_t*>(p)[i]);
}
__device__ __forceinline__ float load_plain(const void* p, int64_t i, std::integral_constant<int, GS_F32>) {
  return static_cast<const float*>(p)[i];
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));

// N numbers (8 or 4) of a row from element `at` on, zero beyond `left` of them.
template <int DT, int N>
__device__ __forceinline__ void load_numbers(const void* row, int64_t at, int64_t left, float (&x)[N]) {
  if (left >= N) {
    if constexpr (DT == GS_BF16) {
      static_assert(N == 8, "16 bytes");
      const i32x4 v = *reinterpret_cast<const i32x4_any2*>(static_cast<const uint16_t*>(row) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(uint32_t(v[i]) << 16);
        x[2 * i + 1] = __uint_as_float(uint32_t(v[i]) & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int h = 0; h < N / 4; ++h) {
        const f32x4_any v = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(row) + at + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * h + i] = v[i];
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = i < left ? load_plain(row, at + i, std::integral_constant<int, DT>{}) : 0.0f;
}

template <int DT, int N>
__device__ __forceinline__ void store_numbers(void* row, int64_t at, int64_t left, uint32_t w, float scale) {
  if constexpr (DT == GS_BF16) {
    static_assert(N == 8, "16 bytes");
    uint16_t* dst = static_cast<uint16_t*>(row) + at;
    const i32x4 v = mx4_decode8(w, scale);
    if (left >= 8) {
      *reinterpret_cast<i32x4_any2*>(dst) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) dst[i] = uint16_t(uint32_t(v[i / 2]) >> (16 * (i & 1)));
    }
  } else {
    float* dst = static_cast<float*>(row) + at;
    float x[N];
    mx4_decode2_f32<0>(w, scale, x);
    mx4_decode2_f32<1>(w, scale, x + 2);
    if constexpr (N == 8) {
      mx4_decode2_f32<2>(w, scale, x + 4);
      mx4_decode2_f32<3>(w, scale, x + 6);
    }
    if (left >= N) {
#pragma unroll
      for (int h = 0; h < N / 4; ++h) *reinterpret_cast<f32x4_any*>(dst + 4 * h) = f32x4_any{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
    } else {
#pragma unroll
      for (int i = 0; i < N - 1; ++i)
        if (i < left) dst[i] = x[i];
    }
  }
}

// The scale byte of the block that 32 / N neighbouring lanes have.
template <int N>
__device__ __forceinline__ uint32_t block_scale_byte(const float (&x)[N]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    top = top > b ? top : b;
  }
  top = max_of_4_lanes(top);
  if constexpr (N == 4) {
    const uint32_t o = __builtin_amdgcn_mov_dpp(top, 0x141, 0xF, 0xF, true);       // the eight lanes in reverse
    top = top > o ? top : o;
  }
  return mx4_scale_byte(top);
}

// Pieces of 16 bytes of all rows' numbers, one after the other: a workgroup takes 256 P of them, a lane P that lie 256 apart, whose loads are
// all under way before the first is used.  Rows and places in them come from a division by multiplication where all pieces count in 31
// bits (BIG: 64-bit divisions).
template <int DT>
constexpr int kNumbers = DT == GS_BF16 ? 8 : 4;
template <bool BIG>
struct Pieces {
  int64_t per_row, total;
  FastDiv by_row;
  __device__ void place(int64_t at, int64_t* row, int64_t* piece) const {
    if constexpr (BIG) {
      *row = at / per_row;
      *piece = at - *row * per_row;
    } else {
      uint32_t q, r;
      by_row.divmod(uint32_t(at), &q, &r);
      *row = q;
      *piece = r;
    }
  }
};

// A row's pieces are counted up to whole runs of scale bytes, the padding written as zeros by the same lanes.
template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) mx4_quantize_kernel(Mx4ConvertArgs a, Pieces<BIG> n) {
  constexpr int N = kNumbers<DT>;
  const int64_t blocks = mx4_blocks(a.cols), pitch = mx4_scale_pitch(a.cols), base = int64_t(blockIdx.x) * (kThreads * P) + threadIdx.x;
  int64_t row[P], piece[P];
  float x[P][N];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int64_t at = base + p * kThreads;
    const bool there = at < n.total;
    n.place(there ? at : 0, &row[p], &piece[p]);
    if (!there) row[p] = -1;
    const void* const src = static_cast<const uint8_t*>(a.plain) + row[p] * a.cols * int64_t(dtype_size(DT));
    load_numbers<DT, N>(src, piece[p] * N, there ? a.cols - piece[p] * N : 0, x[p]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const uint32_t byte = block_scale_byte<N>(x[p]);
    if (row[p] < 0) continue;
    const int64_t block = piece[p] / (kMx4Block / N);
    if (block < blocks) {
      float eight[8] = {};
#pragma unroll
      for (int i = 0; i < N; ++i) eight[i] = x[p][i];
      const int64_t to = row[p] * blocks * (kMx4Block / N) + piece[p];
      if constexpr (N == 8) static_cast<uint32_t*>(a.values)[to] = mx4_encode8(eight, byte);
      else static_cast<uint16_t*>(a.values)[to] = uint16_t(mx4_encode8(eight, byte));
    }
    if (piece[p] % (kMx4Block / N) == 0) static_cast<uint8_t*>(a.scales)[row[p] * pitch + block] = uint8_t(block < blocks ? byte : 0);
  }
}

template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) mx4_dequantize_kernel(Mx4ConvertArgs a, Pieces<BIG> n) {
  constexpr int N = kNumbers<DT>;
  const int64_t blocks = mx4_blocks(a.cols), pitch = mx4_scale_pitch(a.cols), base = int64_t(blockIdx.x) * (kThreads * P) + threadIdx.x;
  int64_t row[P], piece[P];
  uint32_t w[P], byte[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int64_t at = base + p * kThreads;
    n.place(at < n.total ? at : 0, &row[p], &piece[p]);
    const int64_t from = row[p] * blocks * (kMx4Block / N) + piece[p];
    if constexpr (N == 8) w[p] = static_cast<const uint32_t*>(a.values)[from];
    else w[p] = static_cast<const uint16_t*>(a.values)[from];
    byte[p] = static_cast<const uint8_t*>(a.scales)[row[p] * pitch + piece[p] / (kMx4Block / N)];
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (base + p * kThreads >= n.total) continue;
    void* const dst = static_cast<uint8_t*>(a.plain) + row[p] * a.cols * int64_t(dtype_size(DT));
    store_numbers<DT, N>(dst, piece[p] * N, a.cols - piece[p] * N, w[p], mx4_scale(byte[p]));
  }
}

unsigned grid_for(int64_t total) {
  const int64_t n = ceil_div(total, kThreads);
  return unsigned(n < 256 * 64 ? n : 256 * 64);
}

template <int DT, int P, bool BIG>
hipError_t launch_convert(const Mx4ConvertArgs& a, int64_t per_row, bool quantize, hipStream_t s) {
  const int64_t total = a.rows * per_row, groups = ceil_div(total, kThreads * P);
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  const Pieces<BIG> n{per_row, total, FastDiv::make(BIG ? 1u : uint32_t(per_row))};
  if (quantize) hipLaunchKernelGGL((mx4_quantize_kernel<DT, P, BIG>), dim3(unsigned(groups)), dim3(kThreads), 0, s, a, n);
  else hipLaunchKernelGGL((mx4_dequantize_kernel<DT, P, BIG>), dim3(unsigned(groups)), dim3(kThreads), 0, s, a, n);
  return hipGetLastError();
}
// Four pieces per lane where that still leaves eight workgroups for every compute unit.
template <int DT>
hipError_t convert(const Mx4ConvertArgs& a, int64_t per_row, bool quantize, hipStream_t s) {
  const int64_t total = a.rows * per_row;
  if (total == 0) return hipSuccess;
  if (total > 0x7fffffff) return launch_convert<DT, 4, true>(a, per_row, quantize, s);
  if (total >= int64_t(256) * 8 * 4 * kThreads) return launch_convert<DT, 4, false>(a, per_row, quantize, s);
  return launch_convert<DT, 1, false>(a, per_row, quantize, s);
}

// Lanes run over (batch, token, head, piece of 8 numbers); blockIdx.y: keys or values.
struct Token {
  uint8_t* block;         // null: no place in the cache
  uint32_t slot;
};
__device__ __forceinline__ Token place_of(const Mx4TokenArgs& a, int64_t b, int64_t t, int head, bool counted) {
  Token k{nullptr, 0};
  if (counted && a.counts && t >= a.counts[b]) return k;
  const int64_t pos = int64_t(a.first[b]) + t;
  if (pos < 0 || pos >= a.width * a.cache.page) return k;
  uint32_t entry;
  a.cache.by_page.divmod(uint32_t(pos), &entry, &k.slot);
  const int32_t id = a.table[b * a.width + entry];
  if (id < 0 || id >= a.cache.n_pages) return k;
  k.block = a.cache.block(id, head);
  return k;
}

struct TokenDivs {
  FastDiv pieces, heads, tokens;
};
template <int DT, bool WRITE, bool BIG>
__global__ void __launch_bounds__(kThreads) mx4_tokens_kernel(Mx4TokenArgs a, int64_t total, TokenDivs by) {
  const uint32_t pieces = uint32_t(a.cache.dim / 8);
  const bool values = blockIdx.y;
  void* plain = values ? a.v : a.k;
  for (int64_t at = int64_t(blockIdx.x) * kThreads + threadIdx.x; at < total; at += int64_t(gridDim.x) * kThreads) {
    uint32_t piece;
    int head;
    int64_t b, t;
    if constexpr (BIG) {
      const int64_t r = at / pieces, token = r / a.cache.heads;
      piece = uint32_t(at - r * pieces);
      head = int(r - token * a.cache.heads);
      b = token / a.tokens;
      t = token - b * a.tokens;
    } else {
      uint32_t r, token, of, seq, in;
      by.pieces.divmod(uint32_t(at), &r, &piece);
      by.heads.divmod(r, &token, &of);
      by.tokens.divmod(token, &seq, &in);
      head = int(of);
      b = seq;
      t = in;
    }
    const Token place = place_of(a, b, t, head, WRITE);
    const uint32_t codes = values ? a.cache.value(place.slot, piece) : a.cache.key(place.slot) + piece * 4;
    const uint32_t scale = values ? a.cache.value_scale(place.slot, piece / 4) : a.cache.key_scale(place.slot, piece / 4);
    if constexpr (WRITE) {
      float x[8];
      load_numbers<DT, 8>(plain, at * 8, 8, x);
      const uint32_t byte = block_scale_byte(x);
      if (place.block) {
        *reinterpret_cast<uint32_t*>(place.block + codes) = mx4_encode8(x, byte);
        if (piece % 4 == 0) place.block[scale] = uint8_t(byte);
      }
    } else {
      uint32_t w = 0;
      float s = 1.0f;
      if (place.block) {
        w = *reinterpret_cast<const uint32_t*>(place.block + codes);
        s = mx4_scale(place.block[scale]);
      }
      store_numbers<DT, 8>(plain, at * 8, 8, w, s);
    }
  }
}

template <int DT, bool WRITE>
hipError_t launch_tokens_of(const Mx4TokenArgs& a, hipStream_t s) {
  const int64_t total = a.batch * a.tokens * a.cache.heads * (a.cache.dim / 8);
  if (total == 0) return hipSuccess;
  const dim3 grid(grid_for(total), 2);
  if (total > 0x7fffffff) {
    hipLaunchKernelGGL((mx4_tokens_kernel<DT, WRITE, true>), grid, dim3(kThreads), 0, s, a, total, TokenDivs{});
  } else {
    const TokenDivs by{FastDiv::make(uint32_t(a.cache.dim / 8)), FastDiv::make(uint32_t(a.cache.heads)), FastDiv::make(uint32_t(a.tokens))};
    hipLaunchKernelGGL((mx4_tokens_kernel<DT, WRITE, false>), grid, dim3(kThreads), 0, s, a, total, by);
  }
  return hipGetLastError();
}
template <bool WRITE>
hipError_t launch_tokens(const Mx4TokenArgs& a, hipStream_t s) {
  return a.dtype == GS_BF16 ? launch_tokens_of<GS_BF16, WRITE>(a, s) : launch_tokens_of<GS_F32, WRITE>(a, s);
}

}  // namespace

hipError_t launch_mx4_quantize(const Mx4ConvertArgs& a, hipStream_t s) {
  const int64_t per_row = mx4_scale_pitch(a.cols) * kMx4Block;
  return a.dtype == GS_BF16 ? convert<GS_BF16>(a, per_row / 8, true, s) : convert<GS_F32>(a, per_row / 4, true, s);
}

hipError_t launch_mx4_dequantize(const Mx4ConvertArgs& a, hipStream_t s) {
  return a.dtype == GS_BF16 ? convert<GS_BF16>(a, ceil_div(a.cols, 8), false, s) : convert<GS_F32>(a, ceil_div(a.cols, 4), false, s);
}

hipError_t launch_mx4_append(const Mx4TokenArgs& a, hipStream_t s) { return launch_tokens<true>(a, s); }
hipError_t launch_mx4_read(const Mx4TokenArgs& a, hipStream_t s) { return launch_tokens<false>(a, s); }

}  // namespace gs
