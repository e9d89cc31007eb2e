// Rows of numbers in pieces of a lane each: how they are counted and read.
#pragma once

#include "common.h"

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
      const i32x4 v = __builtin_nontemporal_load(reinterpret_cast<const i32x4_any2*>(static_cast<const uint16_t*>(row) + at));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(uint32_t(v[i]) << 16);
        x[2 * i + 1] = __uint_as_float(uint32_t(v[i]) & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int h = 0; h < N / 4; ++h) {
        const f32x4_any v = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(static_cast<const float*>(row) + at + 4 * h));
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * h + i] = v[i];
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = i < left ? load_plain(row, at + i, std::integral_constant<int, DT>{}) : 0.0f;
}

// Pieces of 16 bytes of all rows' numbers, one after the other: a workgroup takes 256 P of them, a lane P that lie 256 apart, whose loads are
// all under way before the first is used.  What pieces cost in instructions counts (16384 x 8190 floats read back with 64-bit places 118 us):
// rows and places are counted in 32 bits where all numbers do (BIG: in 64), the first of a lane's from a division by multiplication, the others
// from it.
template <int DT>
constexpr int kNumbers = DT == GS_BF16 ? 8 : 4;
template <bool BIG>
struct Pieces {
  using Index = std::conditional_t<BIG, int64_t, uint32_t>;
  Index per_row, total;
  FastDiv by_row;
  // of pieces at, at + 256 ..; those behind the last are the first
  template <int P>
  __device__ void places(Index at, Index (&row)[P], Index (&piece)[P]) const {
    divide(at < total ? at : 0, &row[0], &piece[0]);
    const bool wide = per_row >= kThreads;               // (uniform)
#pragma unroll
    for (int p = 1; p < P; ++p) {
      if (wide) {
        const Index next = piece[p - 1] + kThreads;
        const bool same = next < per_row;
        row[p] = same ? row[p - 1] : row[p - 1] + 1;
        piece[p] = same ? next : next - per_row;
      } else {
        divide(at + p * kThreads < total ? at + p * kThreads : 0, &row[p], &piece[p]);
      }
      if (at + p * kThreads >= total) row[p] = piece[p] = 0;
    }
  }
  __device__ void divide(Index at, Index* row, Index* piece) const {
    if constexpr (BIG) {
      *row = at / per_row;
      *piece = at - *row * per_row;
    } else {
      by_row.divmod(at, row, piece);
    }
  }
};

}  // namespace

}  // namespace gs
