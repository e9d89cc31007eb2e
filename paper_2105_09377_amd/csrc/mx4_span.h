// What a workgroup of the attention kernels looks at: tokens in tiles, cut into parts.
#pragma once

#include "mx4.h"

namespace gs {

namespace {

constexpr int kTile = 64;            // tokens of a wave's step
constexpr int kMaxParts = 64;
constexpr int kPartHead = 4;         // floats in front of a part's results: its maximum and sum
// Weights are 2^(score - maximum - kHeadroom): their sum over 2^24 tokens, times the largest number of the format, does not
// overflow before it is divided by their sum.
constexpr float kHeadroom = 24.0f;

// What the rows row0 .. row1 of a sequence of `len` tokens have to look at, in tiles: the first `sink_tiles`, then
// those from `window_tile` on.  Cut into parts of `per` tiles.
struct Span {
  int32_t hi;                        // tokens from here on are seen by no row
  int32_t sink_tiles, window_tile, total, per, parts;
  __device__ int32_t token(int32_t i) const { return (i < sink_tiles ? i : window_tile + i - sink_tiles) * kTile; }
};
__device__ __forceinline__ Span span_of(const Mx4AttendArgs& a, int32_t len, int32_t row0, int32_t row1) {
  Span s;
  const int32_t first = len - a.queries + row0 / a.group, last = len - a.queries + row1 / a.group;    // positions
  s.hi = last + 1 > 0 ? last + 1 : 0;
  int32_t lo = 0;
  if (a.window > 0 && first >= a.window) lo = first - int32_t(a.window) + 1;
  const int32_t sinks = a.sinks < lo ? int32_t(a.sinks) : lo;
  s.sink_tiles = (sinks + kTile - 1) / kTile;
  s.window_tile = lo / kTile > s.sink_tiles ? lo / kTile : s.sink_tiles;
  const int32_t end = (s.hi + kTile - 1) / kTile;
  s.total = s.sink_tiles + (end > s.window_tile ? end - s.window_tile : 0);
  s.per = (s.total + a.parts - 1) / a.parts;
  s.per = s.per > a.least ? s.per : a.least;
  s.parts = s.total > s.per ? (s.total + s.per - 1) / s.per : 1;
  return s;
}
__device__ __forceinline__ int32_t length_of(const Mx4AttendArgs& a, int64_t b) {
  const int32_t len = a.lengths[b], most = int32_t(a.width) * a.cache.page;
  return len < 0 ? 0 : len < most ? len : most;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace

}  // namespace gs
