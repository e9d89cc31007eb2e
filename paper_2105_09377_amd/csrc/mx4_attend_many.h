// Attention over the 4-bit cache for many rows: prompts, and chunks of them over what was cached before.
//
// A workgroup has 128 or 256 rows, 32 per wave, that share a cache head, and walks the tokens in tiles of 64 that all of its waves use: the
// tile's codes are converted to bfloat16 once (exactly) into LDS, the next tile's while this one is multiplied, the one
// behind that on its way into registers.  With r = lane % 32, h = lane / 32 (32x32x16 bfloat16):
//   scores: 32 tokens x 32 rows per product.  Keys lie in LDS as they are, token after token.  Lane (r, h) receives the scores of
//     row r with tokens 8 (v / 4) + 4 h + v % 4.
//   output: 32 numbers x 32 rows per product, over 16 tokens whose weights a lane already has: values lie in LDS one row of 64 tokens per
//     number, the tokens of each 16 in the order 0..3, 8..11, 4..7, 12..15, so that a lane's eight are 16 bytes.
// Rows in LDS are an odd multiple of 16 bytes long: reads and writes of 16 rows fall on different banks.
//
// Bound by vector instructions (a tile of 64 numbers per head: 230 per wave, 32 of them exponentials, beside 16 products of 32
// cycles; 36 of them only where one of the wave's 32 rows has a new maximum, which on random scores is two tiles in five after
// 64): two sequences' 512 queries in a window of 4096 tokens (32 heads of 64 numbers on 8) 65 to 72 us over cards, 480 to 523
// TFLOP/s; 512 over 4096 tokens of 128 numbers 91 us, 569.  128 rows per workgroup, two workgroups on a compute unit: 80 and
// 102 us; a wave's next scores between its weights: 82 and 152 (registers).
#pragma once

#include "mx4_span.h"

namespace gs {

namespace {

template <int D, int NW>
struct ManyShape {
  static constexpr int NB = D / 32;                      // blocks of a token; 64 units of 16 bytes of a tile's keys each, and of its values
  static constexpr int U = (2 * NB + NW - 1) / NW;       // units of a lane
  static constexpr int kKeyRow = 2 * D + 16, kValueRow = 2 * kTile + 16;
  static constexpr int kBuf = kTile * kKeyRow + D * kValueRow;
  static constexpr int kMeta = 16;                       // bytes: 0-3 whether a run of 16 tokens has a page, 4-11 scales of 2^126 and more
  static constexpr int kRows = 32 * NW;
  static constexpr int kBufs = NW == 8 || D == 64 ? 3 : 2;
  static constexpr size_t kLds = kBufs * (kBuf + kMeta);
};

template <int D, int NW>
__global__ void __launch_bounds__(64 * NW, NW == 8 || D > 128 ? 1 : 2) mx4_attend_many_kernel(Mx4AttendArgs a) {
  using S = ManyShape<D, NW>;
  constexpr int NB = S::NB, U = S::U, kRows = S::kRows, kKeyRow = S::kKeyRow, kValueRow = S::kValueRow;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds_many[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
  const int32_t rows = a.queries * a.group, row_tiles = (rows + kRows - 1) / kRows;
  // each XCD (every eighth workgroup) gets consecutive tasks: row tiles of one cache head read the same pages
  const uint32_t per = gridDim.x / 8, rem = gridDim.x % 8, xcd = blockIdx.x % 8;
  uint32_t at = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / 8;
  const uint32_t part = at % uint32_t(a.parts);
  at /= uint32_t(a.parts);
  // (from the last row tile on: it sees the most, and short ones at the end leave less of the chip waiting)
  const uint32_t bh = at / uint32_t(row_tiles), row_tile = uint32_t(row_tiles) - 1 - (at - bh * uint32_t(row_tiles));
  const uint32_t b = bh / uint32_t(a.cache.heads), head = bh - b * uint32_t(a.cache.heads);
  const int32_t row0 = int32_t(row_tile) * kRows, row1 = (row0 + kRows < rows ? row0 + kRows : rows) - 1;
  const int32_t len = length_of(a, b);
  const Span span = span_of(a, len, row0, row1);
  const Cut cut = cut_alike(a, span.total, int64_t(bh) * row_tiles + row_tile);
  if (int32_t(part) >= cut.parts) return;
  const int32_t begin = int32_t(part) * cut.per, stop = begin + cut.per < span.total ? begin + cut.per : span.total;

  // the wave's rows
  const int32_t first_row = row0 + wave * 32, last_row = first_row + 31 < rows ? first_row + 31 : rows - 1;
  const bool active = first_row < rows;
  const int32_t pos_first = len - a.queries + first_row / a.group, pos_last = len - a.queries + last_row / a.group;
  const int32_t row = first_row + r, qi = row / a.group, qh = row - qi * a.group;
  const int32_t pos = row < rows ? len - a.queries + qi : -1;
  const int64_t row_at = ((int64_t(b) * a.queries + qi) * a.cache.heads + head) * a.group * D + int64_t(qh) * D;
  const ScoreScale unit(a.scale);
  bool far = false;
  i32x4 q[2 * NB];
#pragma unroll
  for (int s = 0; s < 2 * NB; ++s) {
    q[s] = i32x4{0, 0, 0, 0};
    if (row < rows) q[s] = scaled_signs(*reinterpret_cast<const i32x4*>(static_cast<const uint16_t*>(a.q) + row_at + s * 16 + h * 8), a.scale);
  }

  f32x16 o[NB];
  float m = -__builtin_inff();
  f32x4 l = {0, 0, 0, 0};
#pragma unroll
  for (int d = 0; d < NB; ++d)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[d][v] = 0;

  // A lane's units of a tile: a block of a token's key, or 8 numbers of 4 tokens' values.  The first NB of the wave's share are keys.
  const int32_t* const table = a.table + int64_t(b) * a.width;
  const uint32_t page = uint32_t(a.cache.page);
  int32_t ids[U];
  uint32_t have = 0;                                     // units of `raw` whose token has a page
  i32x4 raw[U];
  uint32_t raw_scale[U];
  auto key_unit = [&](int u) { return wave + NW * u < NB; };
  auto value_unit = [&](int u) { return wave + NW * u >= NB && wave + NW * u < 2 * NB; };
  auto lane_of = [&](int u) { return (wave + NW * u < NB ? wave + NW * u : wave + NW * u - NB) * 64 + lane; };
  auto token_of = [&](int u) { return key_unit(u) ? lane_of(u) / NB : lane_of(u) % 16 * 4; };
  auto find = [&](int32_t i) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      ids[u] = -1;
      const int32_t token = span.token(i) + token_of(u);
      if (i < stop && wave + NW * u < 2 * NB && token < span.hi) {
        uint32_t entry, slot;
        a.cache.by_page.divmod(uint32_t(token), &entry, &slot);
        ids[u] = table[entry];
      }
    }
  };
  auto load = [&](int32_t i) {
    have = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (ids[u] < 0 || ids[u] >= a.cache.n_pages) {
        raw[u] = i32x4{0, 0, 0, 0};
        raw_scale[u] = 0x7f7f7f7fu;
        continue;
      }
      have |= 1u << u;
      uint32_t entry, slot;
      a.cache.by_page.divmod(uint32_t(span.token(i) + token_of(u)), &entry, &slot);
      const uint8_t* const block = a.cache.block(ids[u], int(head));
      const uint32_t of = uint32_t(lane_of(u));
      if (key_unit(u)) {
        raw[u] = *reinterpret_cast<const i32x4*>(block + slot * (D / 2) + of % NB * 16);
        raw_scale[u] = block[page * D + slot * NB + of % NB];
      } else {
        raw[u] = *reinterpret_cast<const i32x4*>(block + page * (D / 2) + slot * (D / 2) + of / 16 * 16);
        raw_scale[u] = *reinterpret_cast<const uint32_t*>(block + page * (D + NB) + slot * NB + of / 64 * 4);
      }
    }
  };
  auto convert = [&](uint8_t* buf) {
    uint8_t* const meta = buf + S::kBuf;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (key_unit(u)) {
        const int token = lane_of(u) / NB, block = lane_of(u) % NB;
        uint8_t* const dst = buf + token * kKeyRow + block * 64;
        const float s = mx4_scale(raw_scale[u]);
#pragma unroll
        for (int c = 0; c < 4; ++c) *reinterpret_cast<i32x4*>(dst + 16 * c) = mx4_decode8(uint32_t(raw[u][c]), s);
        if (block == 0 && token % 16 == 0) meta[token / 16] = uint8_t((have >> u) & 1u);
      } else if (value_unit(u)) {
        // Scale bytes of 253 and more could make infinities or NaN of numbers, and those times a weight of zero would spoil rows
        // that do not see the token: their numbers are zero here and added one by one below.
        const bool wild = ((((raw_scale[u] & 0x7f7f7f7fu) + 0x03030303u) & raw_scale[u]) & 0x80808080u) != 0;
        if (__any(wild)) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (((raw_scale[u] >> (8 * j)) & 255u) >= 253u) {
              raw[u][j] = 0;
              raw_scale[u] &= ~(255u << (8 * j));
            }
          if (lane == 0) meta[4 + wave + NW * u - NB] = 1;
        } else if (lane == 0) {
          meta[4 + wave + NW * u - NB] = 0;
        }
        uint32_t d[4][4];                                // [token][pair of numbers]
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t x = ((raw_scale[u] >> (8 * j)) & 255u) << 23;
          const i32x4 y = mx4_decode8(uint32_t(raw[u][j]), __uint_as_float(x > 0x00400000u ? x : 0x00400000u));
#pragma unroll
          for (int c = 0; c < 4; ++c) d[j][c] = uint32_t(y[c]);
        }
        const int four = lane_of(u) % 16, piece = lane_of(u) / 16;
        uint8_t* const dst = buf + kTile * kKeyRow + piece * 8 * kValueRow + four / 4 * 32 + four % 2 * 16 + four / 2 % 2 * 8;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int odd = 0; odd < 2; ++odd) {
            const uint32_t sel = odd ? 0x07060302u : 0x05040100u;
            *reinterpret_cast<i32x2*>(dst + (2 * c + odd) * kValueRow) =
                i32x2{int32_t(__builtin_amdgcn_perm(d[1][c], d[0][c], sel)), int32_t(__builtin_amdgcn_perm(d[3][c], d[2][c], sel))};
          }
      }
    }
  };
  const int32_t window = a.window > 0 ? int32_t(a.window) : 1 << 30, sinks = int32_t(a.sinks);
  auto sees = [&](int32_t position, int32_t token) {
    return token <= position && (position - token < window || token < sinks);
  };

  auto compute = [&](const uint8_t* buf, int32_t token0) {
    const i32x4 meta = *reinterpret_cast<const i32x4*>(buf + S::kBuf);
    const uint32_t pages = __builtin_amdgcn_readfirstlane(meta[0]);
    const bool tame = __builtin_amdgcn_readfirstlane(meta[1] | meta[2]) == 0;
    // scores: both halves of the tile in turn, their keys requested two steps ahead
    f32x16 s[2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[n][v] = 0;
    i32x4 kf[3][2];
    const uint8_t* const keys = buf + r * kKeyRow + h * 16;
    auto read_keys = [&](auto c_) {
      constexpr int c = decltype(c_)::value;
#pragma unroll
      for (int n = 0; n < 2; ++n) kf[c % 3][n] = *reinterpret_cast<const i32x4*>(keys + n * 32 * kKeyRow + c * 32);
    };
    read_keys(std::integral_constant<int, 0>{});
    read_keys(std::integral_constant<int, 1>{});
    static_for<2 * NB>([&](auto c_) {
      constexpr int c = decltype(c_)::value;
      if constexpr (c + 2 < 2 * NB) read_keys(std::integral_constant<int, c + 2>{});
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < 2; ++n)
        s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[c % 3][n]), __builtin_bit_cast(bf16x8, q[c]), s[n], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    });
    i32x4 vf[2][NB];
    const uint8_t* const values = buf + kTile * kKeyRow + r * kValueRow + h * 16;
    auto read_values = [&](auto k_) {                    // 16 tokens
      constexpr int k = decltype(k_)::value;
#pragma unroll
      for (int d = 0; d < NB; ++d) vf[k % 2][d] = *reinterpret_cast<const i32x4*>(values + d * 32 * kValueRow + k * 32);
    };
    // (heads of 192 numbers: behind the last branch on scores, 512 queries over 8192 tokens 211 us, 214 from here; of 256
    // 279 and 272)
    constexpr bool kLate = D == 192;
    if constexpr (!kLate) read_values(std::integral_constant<int, 0>{});
    const bool all_seen = pages == 0x01010101u && token0 + kTile - 1 <= pos_first &&
                          (pos_last - token0 < window || token0 + kTile <= sinks);
    if (!all_seen) {
      // tokens that the row sees, of the tile's 64 a bit each, then those of the lane's half: bit 8 (v / 4) + v % 4 of seen
      uint64_t paged = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) paged |= ((pages >> (8 * i)) & 1u) ? 0xffffull << (16 * i) : 0ull;
      const uint64_t mask = paged & seen_tokens(pos, token0, window, sinks);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const uint32_t seen = uint32_t(mask >> (32 * n)) >> (4 * h);
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!(seen & (1u << (8 * (v / 4) + v % 4)))) s[n][v] = -__builtin_inff();
      }
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, s[n][v]);
    const uint32_t bits = __float_as_uint(top);
    const auto both = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
    top = fmaxf(unit.score(top) + kHeadroom, m);
    float ref = top == -__builtin_inff() ? 0.0f : top;
    if (__any(top > m)) {
      const float shrink = exp2_fast(m - ref);
      m = top;
      l *= shrink;
#pragma unroll
      for (int d = 0; d < NB; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[d][v] *= shrink;
      far = __any(ScoreScale::far(ref));
    }
    if (__builtin_expect(far, 0)) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) s[n][v] = unit.apart(s[n][v], ref);
      ref = 0.0f;
    }
    if constexpr (kLate) read_values(std::integral_constant<int, 0>{});
    // weights, four at a time; those of the second half between the products of the first
    i32x4 w[2][2];
    auto weigh = [&](auto n_, auto i_) {
      constexpr int n = decltype(n_)::value, i = decltype(i_)::value;
#pragma unroll
      for (int v = 4 * i; v < 4 * i + 4; ++v) {
        s[n][v] = exp2_fast(fmaf(s[n][v], unit.to_log2, -ref));
      }
#pragma unroll
      for (int v = 4 * i; v < 4 * i + 4; v += 2) w[n][i / 2][v / 2 % 4] = int32_t(pack_bf16x2(s[n][v], s[n][v + 1]));
      l = add_weights(w[n][i / 2][2 * i % 4], w[n][i / 2][2 * i % 4 + 1], l);
    };
    static_for<4>([&](auto i_) { weigh(std::integral_constant<int, 0>{}, i_); });
    static_for<4>([&](auto k_) {
      constexpr int k = decltype(k_)::value;
      if constexpr (k < 3) read_values(std::integral_constant<int, k + 1>{});
      static_for<NB>([&](auto d_) {
        constexpr int d = decltype(d_)::value, slot = k * NB + d;
        __builtin_amdgcn_sched_barrier(0);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[k % 2][d]),
                                                       __builtin_bit_cast(bf16x8, w[k / 2][k % 2]), o[d], 0, 0, 0);
        static_for<4>([&](auto i_) {
          if constexpr (decltype(i_)::value * NB / 2 == slot) weigh(std::integral_constant<int, 1>{}, i_);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
    });
    if (!tame) {
#pragma unroll 1
      for (int32_t token = token0; token < token0 + kTile && token < span.hi; ++token) {
        uint32_t entry, slot;
        a.cache.by_page.divmod(uint32_t(token), &entry, &slot);
        const int32_t id = table[entry];
        if (id < 0 || id >= a.cache.n_pages) continue;
        const uint8_t* const block = a.cache.block(id, int(head));
        const int32_t of = token - token0, mine = of / 8 * 4 + of % 4;       // which of a lane's 32 weights, in lanes of half of / 4 % 2
        float weight = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const uint32_t x = uint32_t(w[i / 16][i / 8 % 2][i / 2 % 4]);
          weight = i == mine ? __uint_as_float(i % 2 ? x & 0xffff0000u : x << 16) : weight;
        }
        weight = __shfl(weight, of / 4 % 2 * 32 + r);
        if (!sees(pos, token)) continue;
#pragma unroll
        for (int d = 0; d < NB; ++d) {
          const uint32_t byte = block[page * (D + NB) + (slot / 4 * NB + d) * 4 + slot % 4];
          if (byte < 253) continue;
          const float scaled = weight * mx4_scale(byte);
#pragma unroll
          for (int g = 0; g < 4; ++g) {                  // numbers 8 g + 4 h .. of the block
            const uint32_t x = reinterpret_cast<const uint16_t*>(block + page * (D / 2) + ((slot / 4 * (D / 8) + 4 * d + g) * 4 + slot % 4) * 4)[h];
            float f[4];
            mx4_decode2_f32<0>(x, 1.0f, f);
            mx4_decode2_f32<1>(x, 1.0f, f + 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[d][4 * g + j] += scaled * f[j];
          }
        }
      }
    }
  };

  if (threadIdx.x < S::kBufs) *reinterpret_cast<i32x4*>(lds_many + threadIdx.x * (S::kBuf + S::kMeta) + S::kBuf) = i32x4{0, 0, 0, 0};
  __syncthreads();
  if (begin < stop) {
    find(begin);
    load(begin);
    convert(lds_many);
    find(begin + 1);
    load(begin + 1);
    find(begin + 2);
    // With three buffers the barrier stands between the conversion of the next tile and the products of this one: a wave may be
    // ahead of another by almost a tile.  With two it stands behind the products, whose buffer the next conversion fills.
    if (S::kBufs == 2) __syncthreads();
    uint32_t buf = 0;
    for (int32_t i = begin; i < stop; ++i) {
      const uint32_t next = buf + (S::kBuf + S::kMeta) == S::kLds ? 0 : buf + (S::kBuf + S::kMeta);
      if (i + 1 < stop) {
        convert(lds_many + next);
        load(i + 2);
        find(i + 3);
      }
      if (S::kBufs == 3) __syncthreads();
      const int32_t token0 = span.token(i);
      const bool any_seen = active && token0 <= pos_last && (pos_first - (token0 + kTile - 1) < window || token0 < sinks);
      if (any_seen) compute(lds_many + buf, token0);
      if (S::kBufs == 2) __syncthreads();
      buf = next;
    }
  }

  const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[0]), __float_as_uint(l[0]), false, false);
  const float total = __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
  if (row >= rows) return;
  if (cut.parts == 1) {
    const float inv = total != 0.0f ? 1.0f / total : 0.0f;
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float x0 = o[d][4 * g] * inv, x1 = o[d][4 * g + 1] * inv, x2 = o[d][4 * g + 2] * inv, x3 = o[d][4 * g + 3] * inv;
        const int64_t dst = row_at + d * 32 + g * 8 + h * 4;
        if (a.out_dtype == GS_BF16)
          *reinterpret_cast<i32x2*>(static_cast<uint16_t*>(a.out) + dst) = i32x2{int32_t(pack_bf16x2(x0, x1)), int32_t(pack_bf16x2(x2, x3))};
        else
          *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + dst) = f32x4{x0, x1, x2, x3};
      }
  } else {
    float* const dst = a.partial + ((cut.base + part) * kRows + wave * 32 + r) * (D + kPartHead);
    if (h == 0) *reinterpret_cast<f32x2_t*>(dst) = f32x2_t{m, total};
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(dst + kPartHead + d * 32 + g * 8 + h * 4) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
  }
}

}  // namespace

}  // namespace gs
