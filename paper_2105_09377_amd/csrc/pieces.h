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

typedef int32_t i32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef int32_t i32_any __attribute__((aligned(1)));

// 16 bytes of a tensor from byte `at` on, zeros beyond `left` of them.  STREAM: they are not read again soon.  What ends a row is read with what is in
// front of it, which is then moved out: one access, as for the others, where bytes one by one would have the wave wait for one lane's (rows of 2050
// bfloat16 numbers joined in 66 us that way, 55 this one).
template <bool STREAM>
__device__ __forceinline__ i32x4 load_16(const void* base, int64_t at, int64_t left) {
  const uint8_t* const p = static_cast<const uint8_t*>(base);
  if (left <= 0) return i32x4{0, 0, 0, 0};
  if (left < 16 && at + left < 16) {         // the tensor's first bytes
    i32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 15; ++i)
      if (i < left) v[i / 4] |= int32_t(uint32_t(p[at + i]) << (8 * (i % 4)));
    return v;
  }
  const int64_t over = left < 16 ? 16 - left : 0;
  const i32x4_any* const src = reinterpret_cast<const i32x4_any*>(p + at - over);
  i32x4 v;
  if constexpr (STREAM) v = __builtin_nontemporal_load(src);
  else v = *src;
  return row_piece_fix(v, over);
}
// N numbers (a multiple of 16 bytes) of a tensor from element `at` on, zero beyond `left` of them.
template <int DT, int N, bool STREAM = true>
__device__ __forceinline__ void load_row_numbers(const void* base, int64_t at, int64_t left, float (&x)[N]) {
  if constexpr (DT == GS_BF16) {
    static_assert(N == 8, "16 bytes");
    const i32x4 v = load_16<STREAM>(base, at * 2, left * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(uint32_t(v[i]) << 16);
      x[2 * i + 1] = __uint_as_float(uint32_t(v[i]) & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
      const i32x4 v = load_16<STREAM>(base, at * 4 + h * 16, left * 4 - h * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = __int_as_float(v[i]);
    }
  }
}
// The first `left` bytes of 16, left >= 1 and a multiple of an element's UNIT bytes, to any place.
template <int UNIT, bool STREAM>
__device__ __forceinline__ void store_16(uint8_t* p, int64_t left, i32x4 v) {
  if (left >= 16) {
    if constexpr (STREAM) __builtin_nontemporal_store((i32x4_any)v, reinterpret_cast<i32x4_any*>(p));
    else *reinterpret_cast<i32x4_any*>(p) = v;
    return;
  }
  if (left & 8) {
    *reinterpret_cast<i32x2_any*>(p) = i32x2_any{v[0], v[1]};
    v[0] = v[2];
    v[1] = v[3];
    p += 8;
  }
  if (left & 4) {
    *reinterpret_cast<i32_any*>(p) = v[0];
    v[0] = v[1];
    p += 4;
  }
  if constexpr (UNIT <= 2) {
    if (left & 2) {
      *reinterpret_cast<uint16_t*>(p) = uint16_t(v[0]);
      v[0] = int32_t(uint32_t(v[0]) >> 16);
      p += 2;
    }
  }
  if constexpr (UNIT == 1)
    if (left & 1) *p = uint8_t(v[0]);
}
// N numbers of a row from element `at` on into memory, as far as `left` goes.
template <int DT, int N, bool STREAM = true>
__device__ __forceinline__ void store_row_numbers(void* base, int64_t at, int64_t left, const float (&x)[N]) {
  uint8_t* const p = static_cast<uint8_t*>(base) + at * (DT == GS_BF16 ? 2 : 4);
  if constexpr (DT == GS_BF16) {
    static_assert(N == 8, "16 bytes");
    const i32x4 v = {int32_t(pack_bf16x2(x[0], x[1])), int32_t(pack_bf16x2(x[2], x[3])), int32_t(pack_bf16x2(x[4], x[5])), int32_t(pack_bf16x2(x[6], x[7]))};
    if (left > 0) store_16<2, STREAM>(p, left * 2, v);
  } else {
#pragma unroll
    for (int h = 0; h < N / 4; ++h)
      if (left > 4 * h)
        store_16<4, STREAM>(p + 16 * h, (left - 4 * h) * 4,
                            i32x4{__float_as_int(x[4 * h]), __float_as_int(x[4 * h + 1]), __float_as_int(x[4 * h + 2]), __float_as_int(x[4 * h + 3])});
  }
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
