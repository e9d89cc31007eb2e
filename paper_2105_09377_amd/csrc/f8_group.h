// Which rows of the result a workgroup has.
#pragma once

#include "f8.h"

namespace gs {

namespace {

struct F8Rows {
  int64_t first, end;                  // rows of the result; none where end is not above first
  int64_t expert;
};

// Sums over the lanes up to and with this one.
__device__ __forceinline__ int32_t lanes_up_to(int32_t v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int32_t o = __shfl_up(v, d);
    v += lane >= d ? o : 0;
  }
  return v;
}

// The rows of 64 experts from e0 on, one's to a lane (none behind the last expert): offsets are taken as at least 0, at most M and none as
// below one before it, so that no row is two experts' and there are no more tiles than f8_most_tiles says.  `most` is the largest offset before
// e0, and then that before e0 + 64.  Offsets that go up, as sorting gives them, are used as they are.
__device__ __forceinline__ void f8_rows_of(const F8DotArgs& a, int64_t e0, int lane, int32_t* most, int32_t* lo, int32_t* hi) {
  const int64_t e = e0 + lane < a.experts ? e0 + lane : a.experts, next = e < a.experts ? e + 1 : e;
  int32_t l = a.offsets[e], h = a.offsets[next];
  const int32_t m = int32_t(a.M);
  l = l < 0 ? 0 : l < m ? l : m;
  h = h < 0 ? 0 : h < m ? h : m;
  if (__ballot(l < *most || h < l)) {
    if (lane == 0) l = l > *most ? l : *most;
    if (lane == 0) h = h > l ? h : l;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int32_t o = __shfl_up(h, d);
      h = lane >= d && o > h ? o : h;
    }
    const int32_t o = __shfl_up(h, 1);
    l = lane == 0 ? l : o;
  }
  *most = __builtin_amdgcn_readlane(h, 63);
  *lo = l;
  *hi = h;
}

// How many tiles of `size` rows the experts' rows are cut into, expert by expert.
__device__ __forceinline__ int64_t f8_group_tiles(const F8DotArgs& a, int size) {
  const int lane = threadIdx.x & 63;
  int64_t all = 0;
  int32_t most = 0;
  for (int64_t e0 = 0; e0 < a.experts; e0 += 64) {
    int32_t lo, hi;
    f8_rows_of(a, e0, lane, &most, &lo, &hi);
    all += __builtin_amdgcn_readlane(lanes_up_to((hi - lo + size - 1) / size, lane), 63);
  }
  return all;
}

// The tile-th of those tiles; every wave finds it by itself.
__device__ __forceinline__ F8Rows f8_group_tile(const F8DotArgs& a, int64_t tile, int size) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  int32_t most = 0;
  for (int64_t e0 = 0; e0 < a.experts; e0 += 64) {
    int32_t lo, hi;
    f8_rows_of(a, e0, lane, &most, &lo, &hi);
    const int32_t tiles = (hi - lo + size - 1) / size;
    const int32_t upto = lanes_up_to(tiles, lane);
    const uint64_t behind = __ballot(before + upto > tile);
    if (behind) {
      const int first = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)behind) - 1);
      const int64_t row = lo + (tile - before - (upto - tiles)) * size;
      F8Rows r;
      r.first = __builtin_amdgcn_readlane(int32_t(row), first);
      r.end = __builtin_amdgcn_readlane(hi, first);
      r.expert = e0 + first;
      return r;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return F8Rows{0, 0, 0};
}

// The row of x that a row of the result is of, -1 where there is none.
__device__ __forceinline__ int64_t f8_x_row(const F8DotArgs& a, int64_t row) {
  if (!a.tokens) return row;
  const int64_t t = a.tokens[row];
  return t >= 0 && t < a.x_count ? t : -1;
}

}  // namespace

}  // namespace gs
