// What a workgroup of the attention kernels looks at: tokens in tiles, cut into parts.
#pragma once

#include "mx4.h"

namespace gs {

namespace {

constexpr int kTile = 64;            // tokens of a wave's step
constexpr int kMaxParts = 64;
constexpr int kPartHead = 4;         // floats in front of a part's results: its maximum and sum
// Weights are 2^(score - maximum - kHeadroom): their sum over 2^24 tokens, times the largest number of the format, does not
// overflow before it is divided by their sum.  (So values below 2^-102 are multiplied into numbers below float's normal ones.)
constexpr float kHeadroom = 24.0f;

// What the rows row0 .. row1 of a sequence of `len` tokens have to look at, in tiles: the first `sink_tiles`, then
// those from `window_tile` on.
struct Span {
  int32_t hi;                        // tokens from here on are seen by no row
  int32_t sink_tiles, window_tile, total;
  __device__ int32_t token(int32_t i) const { return (i < sink_tiles ? i : window_tile + i - sink_tiles) * kTile; }
};
__device__ __forceinline__ Span span_of(const Mx4AttendArgs& a, int32_t len, int32_t row0, int32_t row1) {
  Span s;
  const int32_t first = len - a.queries + int32_t(a.by_group.div(uint32_t(row0))),
                last = len - a.queries + int32_t(a.by_group.div(uint32_t(row1)));    // positions
  s.hi = last + 1 > 0 ? last + 1 : 0;
  int32_t lo = 0;
  if (a.window > 0 && first >= a.window) lo = first - int32_t(a.window) + 1;
  const int32_t sinks = a.sinks < lo ? int32_t(a.sinks) : lo;
  s.sink_tiles = (sinks + kTile - 1) / kTile;
  s.window_tile = lo / kTile > s.sink_tiles ? lo / kTile : s.sink_tiles;
  const int32_t end = (s.hi + kTile - 1) / kTile;
  s.total = s.sink_tiles + (end > s.window_tile ? end - s.window_tile : 0);
  return s;
}

// A sequence's tiles are cut into `parts` of `per`; the partial results of part p lie at base + p * stride, in results of a workgroup.
struct Cut {
  int32_t per, parts;
  int64_t base, stride;
};
// Every task (sequence, cache head, row tile) into as many parts, `least` tiles long at least.
__device__ __forceinline__ Cut cut_alike(const Mx4AttendArgs& a, int32_t total, int64_t task) {
  Cut c;
  c.per = int32_t(a.by_parts.div(uint32_t(total + a.parts - 1)));
  c.per = c.per > a.least ? c.per : a.least;
  c.parts = total > c.per ? (total + c.per - 1) / c.per : 1;
  c.base = task * a.parts;
  c.stride = 1;
  return c;
}

__device__ __forceinline__ int32_t length_of(const Mx4AttendArgs& a, int64_t b) {
  const int32_t len = a.lengths[b], most = int32_t(a.width) * a.cache.page;
  return len < 0 ? 0 : len < most ? len : most;
}

// Sums over the lanes up to and with this one.
__device__ __forceinline__ int32_t running_sum(int32_t v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // one to the right in rows of 16, two, four, eight
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // the last of rows 0 and 2 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // the last of row 1 to rows 2 and 3
  return v;
}
// Up to 64 sequences with one row tile each: all cut into parts of the same length, so that together they are no more than `slots`.  A lane has
// a sequence's number of parts, and how many those before it have.
struct Shares {
  int32_t per, parts, before;
};
__device__ __forceinline__ Shares shares_of(const Mx4AttendArgs& a, int lane) {
  const bool there = lane < a.batch;
  const int32_t tiles = there ? span_of(a, length_of(a, lane), 0, a.queries * a.group - 1).total : 0;
  const int32_t all = __builtin_amdgcn_readlane(running_sum(tiles), 63), batch = int32_t(a.batch);
  Shares s;
  int32_t sum;
  // each sequence's last part is half empty on average; if that was too few, count all of them
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int32_t room = a.slots - (i ? batch : batch / 2);
    s.per = (all + room - 1) / room;
    s.per = s.per > a.least ? s.per : a.least;
    s.parts = there ? tiles > s.per ? (tiles + s.per - 1) / s.per : 1 : 0;
    sum = running_sum(s.parts);
    if (__builtin_amdgcn_readlane(sum, 63) <= a.slots) break;
  }
  s.before = sum - s.parts;
  return s;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The 64 tokens from token0 on that a row at this position sees, a bit each.
__device__ __forceinline__ uint64_t seen_tokens(int32_t pos, int32_t token0, int32_t window, int32_t sinks) {
  auto below = [](int32_t n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : ~0ull >> (64 - n); };      // the first n
  return below(pos - token0 + 1) & (~below(pos - token0 - window + 1) | below(sinks - token0));
}

// A negative scale turns the signs of the queries and one of zero makes them zero (infinite ones NaN), so that a score is its product
// times a positive number: the largest is the largest, and that of a token that is not seen may be set to -infinity before.
__device__ __forceinline__ i32x4 scaled_signs(i32x4 q, float scale) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = uint32_t(q[i]);
    if (scale < 0) q[i] = int32_t(x ^ 0x80008000u);
    if (scale == 0) q[i] = int32_t(pack_bf16x2(__uint_as_float(x << 16) * 0.0f, __uint_as_float(x & 0xffff0000u) * 0.0f));
  }
  return q;
}
// Products times the scale and log2(e) are scores in the unit of the weights, 2^(score - m), m being the largest one and the headroom.  One
// fused multiplication and subtraction gives that power; it does not round the score, as m is rounded, so all weights of a row are off by the
// same power, up to half a unit in the last place of the scores: 2 where they are 2^25, beyond the numbers' range where they are above 2^31.  So
// where a row of the wave has a score that is `far`, scores are rounded first and products replaced by what they are `apart` from m: the largest
// one's weight is that of the headroom, or 1 where the headroom is less than such a unit.
struct ScoreScale {
  float to_log2;                     // above 0
  __device__ explicit ScoreScale(float given) : to_log2(given == 0 ? 1.0f : fabsf(given) * 1.44269504088896340736f) {}
  __device__ float score(float product) const {
#pragma clang fp contract(off)
    return product * to_log2;
  }
  __device__ float apart(float product, float ref) const {
#pragma clang fp contract(off)
    return (score(product) - ref) / to_log2;
  }
  static __device__ bool far(float m) { return fabsf(m) > 268435456.0f; }      // 2^28
};

// The sum of a lane's four weights (two dwords of bfloat16), added to each of the four numbers of l: a product of 4x4x4 with ones.  The
// rounded weights are summed, those that the values are multiplied with.
__device__ __forceinline__ f32x4 add_weights(int32_t w0, int32_t w1, f32x4 l) {
  typedef short bf16x4_bits __attribute__((ext_vector_type(4)));
  const i32x2 four = {w0, w1}, ones = {0x3f803f80, 0x3f803f80};
  return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(bf16x4_bits, ones), __builtin_bit_cast(bf16x4_bits, four), l, 0, 0, 0);
}

}  // namespace

}  // namespace gs
