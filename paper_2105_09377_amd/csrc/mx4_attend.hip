// Attention over a paged cache of microscaled 4-bit keys and values.
//
// A workgroup has 16 QT rows -- queries and heads that share the keys and values of one cache head -- and a part of
// the sequence; its four waves (eight where there is a compute unit for every workgroup) take tiles of 64 tokens in
// turn, each with a running maximum and sum, and are joined at the end; parts are joined by a second kernel.  Nothing
// passes through LDS on the way in: the cache's order is the one that the matrix unit wants.  With r = lane % 16,
// g = lane / 16:
//   scores: 16 tokens x 16 rows per product (16x16x32 bfloat16).  Lane (r, g) reads numbers g D/4 .. of the key of
//     token r of a run of 16, converts them to bfloat16 (exactly: e2m1 times a power of two) and multiplies them by the same
//     numbers of query row r.  It receives the scores of row r with tokens 4 g .. 4 g + 3 of the run.
//   output: rows are pieces of 8 numbers of the values, columns the 16 query rows, and the sum runs over the tokens whose
//     weights a lane already has: it reads piece r of those 4 tokens (16 bytes), converts, and pairs tokens by byte permutation.
//     Lane (r, g) receives numbers 8 (4 g + i) + j of row r.
// So a row's maximum, sum and correction are one register, the same for all of a lane's scores and results.
// Weights are rounded to bfloat16, results of floats too: in 32 bits their product with the values, which are exact in
// bfloat16, would be two.  The sum is that of the rounded weights.  In the norm, bfloat16 results are off by 0.0022 of themselves and by
// 0.0017, their own rounding, with weights of 32 bits.
// Many rows have a kernel of their own (mx4_attend_many.h).
//
// Bound by the reading of the cache, and by what a workgroup waits for before its first tile (lengths, table, codes,
// one behind the other): so there are as many workgroups as the chip has at a time, and sequences of different lengths
// are cut into parts of one length.  32 sequences of up to 8191 tokens (64 query heads on 8 of 128 numbers, 183 MB) 42
// us where they lie in the last-level cache in part, 44 from memory (4.1 TB/s), the joining of parts 5 of them (parts as
// many for each sequence 50; the same loads without the arithmetic 44 where this took 50); one sequence of 131072
// tokens (32 heads on 8, 143 MB) 35 and 36 us.  Codes are read with the streaming hint: with caches beyond the last-level
// cache 50 -> 45 us, within it up to 10 % slower, and a model's caches are beyond it.
#include "mx4_attend_many.h"

namespace gs {

namespace {

// Maximum and sum over the four lanes that have the same r.
__device__ __forceinline__ float max_over_g(float v) {
  uint32_t u = __float_as_uint(v);
  auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  u = __float_as_uint(v);
  p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float sum_over_g(float v) {
  uint32_t u = __float_as_uint(v);
  auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  u = __float_as_uint(v);
  p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// N dwords from an address aligned to 4 bytes (8 where N is even, 16 where it is a multiple of 4).
template <int N>
__device__ __forceinline__ void load_dwords(const uint8_t* p, uint32_t (&out)[N]) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const i32x4 v = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(p) + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) out[4 * i + j] = uint32_t(v[j]);
    }
  } else if constexpr (N % 2 == 0) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const i32x2 v = reinterpret_cast<const i32x2*>(p)[i];
      out[2 * i] = uint32_t(v[0]);
      out[2 * i + 1] = uint32_t(v[1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = reinterpret_cast<const uint32_t*>(p)[i];
  }
}

template <int D, int QT, int WV>
struct AttendShape {
  static constexpr int C = D / 32;                       // blocks of 32; dwords of a lane's quarter of a key
  static constexpr int KS = (C == 2 || C == 4) ? 1 : 2;  // scale bytes that this quarter has
  static constexpr int VP = (D / 8 + 15) / 16;           // passes over the pieces of the values, 16 at a time
  static constexpr int kRow = D + 4;                     // floats of a row while waves are joined
  static constexpr int kRows = 16 * QT;
  static constexpr size_t kLds = size_t(WV) * 16 * (kRow + 2) * 4;
};

template <int D, int QT, int WV>
__global__ void __launch_bounds__(WV * 64, QT == 1 ? (D <= 128 && WV == 4 ? 3 : 2) : 1) mx4_attend_kernel(Mx4AttendArgs a) {
  using S = AttendShape<D, QT, WV>;
  constexpr int C = S::C, KS = S::KS, VP = S::VP, kRows = S::kRows, kRow = S::kRow;
  extern __shared__ __attribute__((aligned(16))) float lds[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  // workgroup -> sequence, cache head and part; there is one row tile
  const int32_t rows = a.queries * a.group, row0 = 0, row1 = rows - 1;
  uint32_t b, head, part;
  Cut cut;
  if (a.slots) {
    const Shares all = shares_of(a, lane);
    const int32_t slot = int32_t(blockIdx.x / uint32_t(a.cache.heads));
    head = blockIdx.x - uint32_t(slot) * uint32_t(a.cache.heads);
    const uint64_t mine = __ballot(slot >= all.before && slot < all.before + all.parts);
    if (mine == 0) return;
    b = uint32_t(__builtin_ctzll(mine));
    cut.per = all.per;
    cut.parts = __builtin_amdgcn_readlane(all.parts, int(b));
    part = uint32_t(slot - __builtin_amdgcn_readlane(all.before, int(b)));
  } else {
    const uint32_t task = blockIdx.x / uint32_t(a.parts);
    part = blockIdx.x - task * uint32_t(a.parts);
    b = task / uint32_t(a.cache.heads);
    head = task - b * uint32_t(a.cache.heads);
  }
  const int32_t len = length_of(a, b);
  const Span span = span_of(a, len, row0, row1);
  if (!a.slots) {
    cut = cut_alike(a, span.total, 0);
    if (int32_t(part) >= cut.parts) return;
  }
  const int32_t begin = int32_t(part) * cut.per, stop = begin + cut.per < span.total ? begin + cut.per : span.total;

  // the rows' queries, as the scores' products want them, and positions
  i32x4 q[QT][C];
  int32_t pos[QT];
  const int64_t q_row = int64_t(a.cache.heads) * a.group * D;       // elements of one query position
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int32_t row = row0 + t * 16 + r;
    const int32_t i = row / a.group, h = row - i * a.group;
    const bool ok = row < rows;
    pos[t] = ok ? len - a.queries + i : -1;
    const uint16_t* src = static_cast<const uint16_t*>(a.q) + (int64_t(b) * a.queries + i) * q_row + (int64_t(head) * a.group + h) * D + g * (D / 4);
#pragma unroll
    for (int c = 0; c < C; ++c) q[t][c] = ok ? scaled_signs(*reinterpret_cast<const i32x4*>(src + 8 * c), a.scale) : i32x4{0, 0, 0, 0};
  }
  const int32_t pos_first = len - a.queries + row0 / a.group, pos_last = len - a.queries + row1 / a.group;
  const ScoreScale unit(a.scale);

  f32x4 o[QT][VP][8], l[QT];
  float m[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = -__builtin_inff();
    l[t] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < VP; ++p)
#pragma unroll
      for (int j = 0; j < 8; ++j) o[t][p][j] = f32x4{0, 0, 0, 0};
  }

  // Where the 4 runs of 16 tokens of a tile lie (wave-uniform).  Without branches: a run that has no page, or lies behind the last token that
  // a row sees, is read from another place of the cache, and its scores are set to -infinity.
  struct Place {
    const uint8_t* block[4];
    uint32_t slot[4];
    uint32_t pages;                  // bit n: run n has a page
    int32_t token;
  };
  const int32_t* table = a.table + int64_t(b) * a.width;
  const int32_t last_run = (span.hi - 1) & ~15;
  auto run_of = [&](int32_t i, int n) {
    const int32_t token = span.token(i < stop ? i : stop - 1) + 16 * n;
    return token < last_run ? token : last_run;
  };
  auto find = [&](int32_t i, int32_t (&ids)[4]) {
#pragma unroll
    for (int n = 0; n < 4; ++n) ids[n] = table[a.cache.by_page.div(uint32_t(run_of(i, n)))];
  };
  auto place = [&](int32_t i, const int32_t (&ids)[4]) {
    Place w;
    w.token = span.token(i);
    w.pages = 0;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint32_t run = uint32_t(run_of(i, n));
      w.slot[n] = run - a.cache.by_page.div(run) * uint32_t(a.cache.page);
      const bool there = ids[n] >= 0 && ids[n] < a.cache.n_pages;
      w.pages |= uint32_t(there) << n;
      w.block[n] = a.cache.block(there ? ids[n] : 0, int(head));
    }
    return w;
  };
  struct Keys {
    uint32_t k[4][C], scale[4][KS];
  };
  struct Values {
    i32x4 v[4][VP];
    uint32_t scale[4][VP];
  };
  const uint32_t page = uint32_t(a.cache.page);
  auto load_keys = [&](const Place& w, Keys& t) {
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      load_dwords<C>(w.block[n] + w.slot[n] * (D / 2) + uint32_t(r * (D / 2) + g * (D / 8)), t.k[n]);
      const uint8_t* ks = w.block[n] + page * D + w.slot[n] * C + uint32_t(r * C);
      t.scale[n][0] = ks[(C * g) / 4];
      if constexpr (KS == 2) t.scale[n][1] = ks[(C * g + C - 1) / 4];
    }
  };
  auto load_values = [&](const Place& w, Values& t) {
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int p = 0; p < VP; ++p) {
        const int piece = D / 8 - 16 * p >= 16 || 16 * p + r < D / 8 ? 16 * p + r : D / 8 - 1;
        const uint8_t* const codes = w.block[n] + page * (D / 2) + w.slot[n] * (D / 2) + uint32_t(g * (D * 2) + piece * 16);
        t.v[n][p] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(codes));
        t.scale[n][p] = *reinterpret_cast<const uint32_t*>(w.block[n] + page * (D + C) + w.slot[n] * C + uint32_t(g * (C * 4) + piece / 4 * 4));
      }
  };
  const int32_t window = a.window > 0 ? int32_t(a.window) : 1 << 30, sinks = int32_t(a.sinks);
  auto sees = [&](int32_t position, int32_t token) {
    return token <= position && (position - token < window || token < sinks);
  };

  // A tile: the next one's keys are requested once this one's are used up, and its values likewise, into the same registers.
  auto compute = [&](const Place& at, const Place& next, bool more, Keys& keys, Values& t) {
    // scores: s[row tile][run of 16 tokens]
    f32x4 s[QT][4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      float sc[KS];
#pragma unroll
      for (int c = 0; c < KS; ++c) sc[c] = mx4_scale(keys.scale[n][c]);
      i32x4 kv[C];
#pragma unroll
      for (int c = 0; c < C; ++c) kv[c] = mx4_decode8(keys.k[n][c], KS == 1 || (C * g + c) / 4 == (C * g) / 4 ? sc[0] : sc[KS - 1]);
#pragma unroll
      for (int u = 0; u < QT; ++u) {
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < C; ++c)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kv[c]), __builtin_bit_cast(bf16x8, q[u][c]), acc, 0, 0, 0);
        s[u][n] = acc;
      }
      __builtin_amdgcn_sched_barrier(0);               // (conversions ahead of their use cost registers)
    }
    if (more) load_keys(next, keys);
    const bool all_seen = at.pages == 15u && at.token + kTile - 1 <= pos_first && (pos_last - at.token < window || at.token + kTile <= sinks);
    // weights, as the products with the values want them: p[row tile][half of the tile]
    i32x4 w[QT][2];
    float ref[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
      if (!all_seen) {
        uint64_t paged = 0;
#pragma unroll
        for (int n = 0; n < 4; ++n) paged |= (at.pages >> n) & 1u ? 0xffffull << (16 * n) : 0ull;
        const uint64_t mask = (paged & seen_tokens(pos[u], at.token, window, sinks)) >> (4 * g);
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((mask >> (16 * n + i)) & 1u)) s[u][n][i] = -__builtin_inff();
      }
      float top = s[u][0][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[u][i / 4][i % 4]);
      top = fmaxf(unit.score(max_over_g(top)) + kHeadroom, m[u]);
      ref[u] = top == -__builtin_inff() ? 0.0f : top;
      if (__any(top > m[u])) {
        const float shrink = exp2_fast(m[u] - ref[u]);
        m[u] = top;
        l[u] *= shrink;
#pragma unroll
        for (int p = 0; p < VP; ++p)
#pragma unroll
          for (int j = 0; j < 8; ++j) o[u][p][j] *= shrink;
      }
    }
    bool far = false;                                  // (in one branch for all rows: one each 2 % more for 32 rows)
#pragma unroll
    for (int u = 0; u < QT; ++u) far = far || ScoreScale::far(ref[u]);
    if (__builtin_expect(__any(far), 0)) {
#pragma unroll
      for (int u = 0; u < QT; ++u) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[u][n][i] = unit.apart(s[u][n][i], ref[u]);
        ref[u] = 0.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < QT; ++u) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 x = s[u][2 * h + i / 2];
          const float low = fmaf(x[2 * i % 4], unit.to_log2, -ref[u]), high = fmaf(x[2 * i % 4 + 1], unit.to_log2, -ref[u]);
          w[u][h][i] = int32_t(pack_bf16x2(exp2_fast(low), exp2_fast(high)));
        }
#pragma unroll
      for (int n = 0; n < 4; ++n) l[u] = add_weights(w[u][n / 2][2 * n % 4], w[u][n / 2][2 * n % 4 + 1], l[u]);
    }
    // Scale bytes of 253 and more (2^126, 2^127, NaN) could make infinities or NaN of numbers, and those times a weight of
    // zero would spoil rows that do not see the token: their numbers are zero here and added one by one below.
    uint32_t wild = 0;
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int p = 0; p < VP; ++p) wild |= ((t.scale[n][p] & 0x7f7f7f7fu) + 0x03030303u) & t.scale[n][p];
    const bool tame = !__any((wild & 0x80808080u) != 0);
    if (!tame) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int p = 0; p < VP; ++p)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (((t.scale[n][p] >> (8 * j)) & 255u) >= 253u) {
              t.v[n][p][j] = 0;
              t.scale[n][p] = (t.scale[n][p] & ~(255u << (8 * j))) | 127u << (8 * j);
            }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int p = 0; p < VP; ++p) {
        i32x4 va[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {           // pairs of tokens of one run of 16
          uint32_t d[4][4];                              // [token][pair of numbers]
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t x = ((t.scale[2 * h + half][p] >> (8 * j)) & 255u) << 23;
            const i32x4 y = mx4_decode8(uint32_t(t.v[2 * h + half][p][j]), __uint_as_float(x > 0x00400000u ? x : 0x00400000u));
#pragma unroll
            for (int c = 0; c < 4; ++c) d[j][c] = uint32_t(y[c]);
          }
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              va[2 * c][2 * half + j] = int32_t(__builtin_amdgcn_perm(d[2 * j + 1][c], d[2 * j][c], 0x05040100u));
              va[2 * c + 1][2 * half + j] = int32_t(__builtin_amdgcn_perm(d[2 * j + 1][c], d[2 * j][c], 0x07060302u));
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int u = 0; u < QT; ++u)
            o[u][p][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va[j]), __builtin_bit_cast(bf16x8, w[u][h]),
                                                                 o[u][p][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    if (!tame) {
#pragma unroll 1
      for (int32_t token = at.token; token < at.token + kTile && token < span.hi; ++token) {
        uint32_t entry, slot;
        a.cache.by_page.divmod(uint32_t(token), &entry, &slot);
        const int32_t id = table[entry];
        if (id < 0 || id >= a.cache.n_pages) continue;
        const uint8_t* blk = a.cache.block(id, int(head));
        const int32_t of = token - at.token, mine = of / 16 * 4 + of % 4;     // which of a lane's 16 weights, in lanes of group of / 4 % 4
#pragma unroll
        for (int u = 0; u < QT; ++u) {
          float weight = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t x = uint32_t(w[u][i / 8][i / 2 % 4]);
            weight = i == mine ? __uint_as_float(i % 2 ? x & 0xffff0000u : x << 16) : weight;
          }
          weight = __shfl(weight, of / 4 % 4 * 16 + r);
#pragma unroll
          for (int p = 0; p < VP; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int piece = 16 * p + 4 * g + i;      // the pieces that the lane has results of
              if (piece >= D / 8 || !sees(pos[u], token)) continue;
              const uint32_t byte = blk[page * (D + C) + (slot / 4 * C + piece / 4) * 4 + slot % 4];
              if (byte < 253) continue;
              const uint32_t x = *reinterpret_cast<const uint32_t*>(blk + page * (D / 2) + ((slot / 4 * (D / 8) + piece) * 4 + slot % 4) * 4);
              const float scaled = weight * mx4_scale(byte);
              float f[8];
              mx4_decode2_f32<0>(x, 1.0f, f);
              mx4_decode2_f32<1>(x, 1.0f, f + 2);
              mx4_decode2_f32<2>(x, 1.0f, f + 4);
              mx4_decode2_f32<3>(x, 1.0f, f + 6);
#pragma unroll
              for (int j = 0; j < 8; ++j) o[u][p][j][i] += scaled * f[j];
            }
        }
      }
    }
  };

  if (begin + wave < stop) {
    int32_t i = begin + wave, ids[4];
    Keys keys;
    Values values;
    find(i, ids);
    Place at = place(i, ids);
    load_keys(at, keys);
    load_values(at, values);
    find(i + WV, ids);
    for (; i < stop; i += WV) {
      const bool more = i + WV < stop;
      const Place next = place(i + WV, ids);
      find(i + 2 * WV, ids);
      compute(at, next, more, keys, values);
      if (more) load_values(next, values);
      at = next;
    }
  }

  // join the waves, 16 rows at a time
  float* const my_o = lds + wave * 16 * kRow;
  float* const ml = lds + WV * 16 * kRow;            // [wave][row][2]
#pragma unroll
  for (int u = 0; u < QT; ++u) {
    const float sum = sum_over_g(l[u][0]);
    if (u) __syncthreads();
    if (g == 0) {
      ml[(wave * 16 + r) * 2] = m[u];
      ml[(wave * 16 + r) * 2 + 1] = sum;
    }
#pragma unroll
    for (int p = 0; p < VP; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int piece = 16 * p + 4 * g + i;
        if (D / 8 - 16 * p >= 16 || piece < D / 8)
#pragma unroll
          for (int j = 0; j < 8; j += 4)
            *reinterpret_cast<f32x4*>(my_o + r * kRow + piece * 8 + j) =
                f32x4{o[u][p][j][i], o[u][p][j + 1][i], o[u][p][j + 2][i], o[u][p][j + 3][i]};
      }
    __syncthreads();
    const int rr = threadIdx.x >> 4 & 15, d0 = (threadIdx.x & 15) * (D / 16);
    float top = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < WV; ++v) top = fmaxf(top, ml[(v * 16 + rr) * 2]);
    const float ref = top == -__builtin_inff() ? 0.0f : top;
    float total = 0, f[WV];
#pragma unroll
    for (int v = 0; v < WV; ++v) {
      f[v] = exp2_fast(ml[(v * 16 + rr) * 2] - ref);
      total += f[v] * ml[(v * 16 + rr) * 2 + 1];
    }
    float x[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
      x[d] = 0;
#pragma unroll
      for (int v = 0; v < WV; ++v) x[d] += f[v] * lds[(v * 16 + rr) * kRow + d0 + d];
    }
    const int32_t row = row0 + u * 16 + rr;
    if (threadIdx.x >= 256 || row >= rows) continue;     // (16 lanes to a row)
    if (cut.parts == 1) {
      const float inv = total != 0.0f ? 1.0f / total : 0.0f;
      const int32_t i = row / a.group, h = row - i * a.group;
      const int64_t dst = (int64_t(b) * a.queries + i) * q_row + (int64_t(head) * a.group + h) * D + d0;
#pragma unroll
      for (int d = 0; d < D / 16; d += 2) {
        if (a.out_dtype == GS_BF16)
          *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + dst + d) = pack_bf16x2(x[d] * inv, x[d + 1] * inv);
        else
          *reinterpret_cast<f32x2_t*>(static_cast<float*>(a.out) + dst + d) = f32x2_t{x[d] * inv, x[d + 1] * inv};
      }
    } else {
      const int64_t slot = int64_t(blockIdx.x) * kRows + u * 16 + rr;
      float* dst = a.partial + slot * (D + kPartHead);
      if (d0 == 0) *reinterpret_cast<f32x2_t*>(dst) = f32x2_t{top, total};
#pragma unroll
      for (int d = 0; d < D / 16; d += 2) *reinterpret_cast<f32x2_t*>(dst + kPartHead + d0 + d) = f32x2_t{x[d], x[d + 1]};
    }
  }
}

// Joins the parts of rows, D / 4 lanes to a row, four parts' loads under way at a time.  Up to 8 parts a workgroup has as many rows as
// it has lanes for; above, one row (SPLIT), whose parts are dealt to these groups of lanes and joined through LDS.
template <int D, int kRows, bool SPLIT>
__global__ void __launch_bounds__(256) mx4_attend_join_kernel(Mx4AttendArgs a, int32_t total_rows) {
  constexpr int LPR = D / 4, G = 256 / LPR;
  __shared__ f32x4 shared_x[SPLIT ? G : 1][LPR];
  __shared__ float shared_ml[SPLIT ? G : 1][2];
  const int group = threadIdx.x / LPR, d = threadIdx.x % LPR * 4;
  const int32_t at = SPLIT ? int32_t(blockIdx.x) : int32_t(blockIdx.x) * G + group;
  const int32_t rows = a.queries * a.group, row_tiles = (rows + kRows - 1) / kRows;
  const bool ok = at < total_rows && (SPLIT || group < G);
  const int32_t bh = ok ? int32_t(a.by_rows.div(uint32_t(at))) : 0, row = ok ? at - bh * rows : 0, row_tile = row / kRows;
  const int32_t b = int32_t(a.by_heads.div(uint32_t(bh))), head = bh - b * a.cache.heads;
  const int32_t row0 = row_tile * kRows, row1 = (row0 + kRows < rows ? row0 + kRows : rows) - 1;
  Cut cut;
  if (a.slots) {                     // (all lanes of a wave take part)
    const Shares all = shares_of(a, int(threadIdx.x & 63));
    cut.parts = __shfl(all.parts, b);
    cut.base = int64_t(__shfl(all.before, b)) * a.cache.heads + head;
    cut.stride = a.cache.heads;
  } else {
    cut = cut_alike(a, span_of(a, length_of(a, b), row0, row1).total, int64_t(bh) * row_tiles + row_tile);
  }
  if (!ok || cut.parts == 1) return;
  constexpr int64_t kResult = int64_t(kRows) * (D + kPartHead);
  const int64_t stride = cut.stride * kResult;
  const float* const src = a.partial + cut.base * kResult + (row - row0) * (D + kPartHead);
  float top = -__builtin_inff(), total = 0;
  f32x4 x = {0, 0, 0, 0};
  constexpr int kStep = SPLIT ? G : 1;
  if (group < G)
    for (int p0 = SPLIT ? group : 0; p0 < cut.parts; p0 += 4 * kStep) {
      f32x2_t ml[4];
      f32x4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i * kStep;
        ml[i] = f32x2_t{-__builtin_inff(), 0};
        v[i] = f32x4{0, 0, 0, 0};
        if (p < cut.parts) {
          ml[i] = *reinterpret_cast<const f32x2_t*>(src + p * stride);
          v[i] = *reinterpret_cast<const f32x4*>(src + p * stride + kPartHead + d);
        }
      }
      const float now = fmaxf(fmaxf(fmaxf(ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0])), top);
      const float ref = now == -__builtin_inff() ? 0.0f : now;
      const float shrink = exp2_fast(top - ref);
      top = now;
      total *= shrink;
      x *= shrink;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = exp2_fast(ml[i][0] - ref);
        total += f * ml[i][1];
        x += f * v[i];
      }
    }
  if constexpr (SPLIT) {
    if (group < G) {
      shared_x[group][d / 4] = x;
      if (d == 0) {
        shared_ml[group][0] = top;
        shared_ml[group][1] = total;
      }
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int i = 1; i < G; ++i) top = fmaxf(top, shared_ml[i][0]);
    const float ref = top == -__builtin_inff() ? 0.0f : top;
    total = 0;
    x = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const float f = exp2_fast(shared_ml[i][0] - ref);
      total += f * shared_ml[i][1];
      x += f * shared_x[i][d / 4];
    }
  }
  const float inv = total != 0.0f ? 1.0f / total : 0.0f;
  const int32_t i = int32_t(a.by_group.div(uint32_t(row))), h = row - i * a.group;
  const int64_t dst = ((int64_t(b) * a.queries + i) * a.cache.heads * a.group + int64_t(head) * a.group + h) * D + d;
  if (a.out_dtype == GS_BF16)
    *reinterpret_cast<i32x2*>(static_cast<uint16_t*>(a.out) + dst) =
        i32x2{int32_t(pack_bf16x2(x[0] * inv, x[1] * inv)), int32_t(pack_bf16x2(x[2] * inv, x[3] * inv))};
  else *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + dst) = x * inv;
}

// Row tiles of a workgroup and parts of a sequence, from what the host knows: the table's width stands for the lengths, which may be far
// shorter.  A table for 131072 tokens costs 8 sequences of 700 tokens 11.7 us where one for 700 costs 8.9 (two parts and their joining), 64 of
// 1000 20.9 and 15.4, 2048 queries of 2048 tokens 80 and 74 (rows that see different numbers of tokens in large workgroups).
void plan(Mx4AttendArgs* a) {
  const int64_t rows = int64_t(a->queries) * a->group;
  const bool wide = a->cache.dim > 128;
  // 256 rows per workgroup, one of them on a compute unit; 128, two of them, where most tokens are queries themselves,
  // so that row tiles differ in what they see, and there are few (2048 queries, 32 heads of 128 numbers on 8, 78.6 and
  // 69.6 us; 2 x 4096 of them 324 and 339; 2 x 512 over 4096 tokens 91 and 102).
  const bool uneven = a->width * a->cache.page <= 2 * int64_t(a->queries) && a->batch * a->cache.heads * ceil_div(rows, 256) <= 512;
  a->tiles = rows > 128 && !wide && !uneven ? 16 : rows > 32 ? 8 : rows > 16 ? 2 : 1;
  a->least = a->tiles >= 8 ? 4 : 8;
  a->slots = 0;
  const int64_t tasks = a->batch * a->cache.heads * ceil_div(rows, 16 * a->tiles), some = tasks > 0 ? tasks : 1;
  // workgroups that the chip has at a time
  const int64_t groups = a->tiles == 16 || (a->tiles == 8 && wide) || a->tiles == 2 ? 256 : a->tiles == 8 || wide ? 512 : 768;
  int64_t most = a->width * a->cache.page;
  if (a->window > 0) {
    const int64_t seen = a->window + a->queries + (a->sinks < most ? a->sinks : most) + 2 * kTile;
    most = seen < most ? seen : most;
  }
  const int64_t useful = ceil_div(ceil_div(most, kTile), a->least);
  int64_t parts = a->tiles >= 8 ? (groups + some / 2) / some : ceil_div(groups, some);
  parts = parts < useful ? parts : useful;
  parts = parts < kMaxParts ? parts : kMaxParts;
  // A second launch takes as long as two tiles of a wave that has a unit for itself, and as four where others share it: 8 sequences of 700 tokens (8
  // cache heads of 128 numbers) 8.7 us in one part, 11.4 in two, one of 1500 13.0 and 11.4; 64 of 1000 15.7 and 20.8.
  const int64_t few = tasks > 256 ? 16 : a->tiles == 1 && !wide ? 16 : 8;
  if (a->tiles <= 2 && ceil_div(most, kTile) <= few) parts = 1;
  a->parts = int32_t(parts > 1 ? parts : 1);
  // Lengths that differ are no reason to wait for the longest, where the sequences are few enough for a workgroup to look at all.
  if (a->parts > 1 && a->tiles <= 2 && a->batch <= 64 && groups / a->cache.heads > a->batch) {
    const int64_t slots = groups / a->cache.heads;
    a->slots = int32_t(slots < a->batch * useful ? slots : a->batch * useful);
  }
}
int64_t results_of(const Mx4AttendArgs& a) {     // workgroups
  if (a.slots) return int64_t(a.slots) * a.cache.heads;
  return a.batch * a.cache.heads * ceil_div(int64_t(a.queries) * a.group, 16 * a.tiles) * a.parts;
}
// Waves of a workgroup.  32 sequences of 500 tokens, 8 cache heads: 8.4 us with four, 7.9 with eight.
int waves_of(const Mx4AttendArgs& a) {
  if (a.tiles == 16) return 8;
  return a.tiles == 1 && results_of(a) <= 256 ? 8 : 4;
}
// Whether the parts of a row have a workgroup to join them.
bool joined_alone(const Mx4AttendArgs& a) { return a.slots ? a.slots / a.batch >= 8 : a.parts > 8; }

template <int D, int QT, int WV>
hipError_t launch(const Mx4AttendArgs& a, hipStream_t s) {
  constexpr bool kMany = QT >= 8;
  constexpr int kRows = 16 * QT;
  const int64_t rows = int64_t(a.queries) * a.group;
  const int64_t groups = results_of(a);
  const int64_t total_rows = a.batch * a.cache.heads * rows;
  if (groups > 0x7fffffff || total_rows > 0x7fffff00) return hipErrorInvalidValue;
  void (*kernel)(Mx4AttendArgs);
  size_t lds;
  if constexpr (kMany) {
    kernel = mx4_attend_many_kernel<D, WV>;
    lds = ManyShape<D, WV>::kLds;
  } else {
    kernel = mx4_attend_kernel<D, QT, WV>;
    lds = AttendShape<D, QT, WV>::kLds;
  }
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kernel, dim3(unsigned(groups)), dim3(WV * 64), lds, s, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.parts > 1) {
    constexpr int kJoined = 256 / (D / 4);                // rows of a workgroup
    const int32_t n = int32_t(total_rows);
    if (joined_alone(a)) hipLaunchKernelGGL((mx4_attend_join_kernel<D, kRows, true>), dim3(unsigned(n)), dim3(256), 0, s, a, n);
    else hipLaunchKernelGGL((mx4_attend_join_kernel<D, kRows, false>), dim3(unsigned(ceil_div(n, kJoined))), dim3(256), 0, s, a, n);
    e = hipGetLastError();
  }
  return e;
}
template <int D>
hipError_t launch_d(const Mx4AttendArgs& a, hipStream_t s) {
  if constexpr (D <= 128)
    if (a.tiles == 16) return launch<D, 16, 8>(a, s);
  if (a.tiles == 8) return launch<D, 8, 4>(a, s);
  if (a.tiles == 2) return launch<D, 2, 4>(a, s);
  return waves_of(a) == 4 ? launch<D, 1, 4>(a, s) : launch<D, 1, 8>(a, s);
}

}  // namespace

Mx4AttendPlan mx4_attend_plan(const Mx4AttendArgs& given) {
  Mx4AttendArgs a = given;
  plan(&a);
  return Mx4AttendPlan{16 * a.tiles, waves_of(a), a.parts, a.slots, a.parts > 1 && joined_alone(a)};
}

size_t mx4_attend_workspace(const Mx4AttendArgs& given) {
  Mx4AttendArgs a = given;
  plan(&a);
  if (a.parts == 1) return 0;
  return size_t(results_of(a) * 16 * a.tiles) * size_t(a.cache.dim + kPartHead) * 4;
}

hipError_t launch_mx4_attend(const Mx4AttendArgs& given, hipStream_t s) {
  Mx4AttendArgs a = given;
  plan(&a);
  if (a.batch == 0 || a.queries == 0 || a.group == 0) return hipSuccess;
  a.by_group = FastDiv::make(uint32_t(a.group));
  a.by_rows = FastDiv::make(uint32_t(a.queries) * uint32_t(a.group));
  a.by_heads = FastDiv::make(uint32_t(a.cache.heads));
  a.by_parts = FastDiv::make(uint32_t(a.parts));
  switch (a.cache.dim) {
    case 64: return launch_d<64>(a, s);
    case 96: return launch_d<96>(a, s);
    case 128: return launch_d<128>(a, s);
    case 192: return launch_d<192>(a, s);
    case 256: return launch_d<256>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace gs
