// Tiles of products of two operands of scaled 8-bit floats, moved global -> LDS without passing through registers.
//
// A slab is 128 bytes of K per row, one block: a 16x16x128 product takes 16 rows of each operand and gives the block's sums, which
// vector instructions, times the two scales, add to the results.  Rows are 128 bytes in LDS, their 16-byte columns exchanged by an
// XOR of the row so that lanes that are served together fall on different banks; lane (r = lane % 16, g = lane / 16) has columns
// g and g + 4 of row r of either operand (with 2 g and 2 g + 1 lanes 4 to 11 of one g meet those of the next on a bank: 4.3 cycles more a
// read).  w's rows are a lane's four results, x's rows the lanes, so that a lane needs one scale of
// x for each 16 rows; a wave's 128 rows of w or fewer have one scale where w is in blocks of 128 rows.  Scales come four slabs at a
// time, 16 bytes of a row.
//
// 8192 cubed 433 to 449 us in a graph, 2.5 PFLOP/s (451 to 465 among others), where the same without scales (gemm_nt_dma_kernel, which adds in the matrix unit)
// takes 423; 16384 rows of 16 experts with 4096 x 4096 287, 1.9 PFLOP/s, where they fill tiles, 309 to 318 drawn evenly.  What bounds them: the table
// of tiles in f8_dot.hip.
#pragma once

#include "f8_group.h"
#include "mx4_tile.h"

namespace gs {

namespace {

// (Eight neighbouring products are added together, cut to multiples of 2^-13 of the largest one's power of two: fewer bits than the fp32 in which
// eights and blocks are added, in this instruction and in 16x16x32 alike.  Products of 16-bit floats are not cut and take twice as long; the codes
// themselves are rounded to 2^-4.)
__device__ __forceinline__ f32x4 f8_mfma16(const i32x4 (&w)[2], const i32x4 (&x)[2]) {
  const i32x8 a = {w[0][0], w[0][1], w[0][2], w[0][3], w[1][0], w[1][1], w[1][2], w[1][3]};
  const i32x8 b = {x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}

// One wave's results, tot[m][n] being 16 x 16 of them, lane lane % 16 having row m0 + 16 m + lane % 16 and columns n0 + 16 n + 4 (lane / 16) ..
// + 3: staged 16 rows at a time in LDS of its own (16 rows of 16 NJ + 4 floats) and written 8 columns per lane.  `zero`: rows, a bit for each
// 16, of this lane's that are zero.
template <int MI, int NJ>
__device__ __forceinline__ void f8_write_back(const F8DotArgs& a, f32x4 (&tot)[MI][NJ], int64_t m0, int64_t m_end, int64_t n0, int64_t part, uint32_t zero,
                                              float* stage, int lane) {
  constexpr int WN = NJ * 16, RS = WN + 4, LPR = WN / 8, RPP = 64 / LPR, NP = 16 / RPP;
  static_assert(16 % RPP == 0 && NP >= 1, "whole rows per pass");
  const int cq = (lane % LPR) * 8, rsub = lane / LPR;
  const int64_t n = n0 + cq;
  static_for<MI>([&](auto m_) {
    constexpr int m = decltype(m_)::value;
    static_for<NJ>([&](auto n_) {
      constexpr int j = decltype(n_)::value;
      *reinterpret_cast<f32x4*>(stage + (lane & 15) * RS + j * 16 + 4 * (lane >> 4)) = (zero >> m) & 1 ? f32x4{0, 0, 0, 0} : tot[m][j];
    });
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const f32x4* src = reinterpret_cast<const f32x4*>(stage + (p * RPP + rsub) * RS + cq);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = src[e / 4][e % 4];
      if (a.relu)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaxf(x[e], 0.0f);
      const int64_t row = m0 + m * 16 + p * RPP + rsub;
      if (row >= m_end || n >= a.N) continue;
      const int64_t at = (part * a.M + row) * a.N + n;
      if (n + 8 <= a.N) {
        if (a.out_dtype == GS_BF16) {
          const i32x4 w = {int32_t(pack_bf16x2(x[0], x[1])), int32_t(pack_bf16x2(x[2], x[3])), int32_t(pack_bf16x2(x[4], x[5])), int32_t(pack_bf16x2(x[6], x[7]))};
          __builtin_nontemporal_store((i32x4_any2t)w, reinterpret_cast<i32x4_any2t*>(static_cast<uint16_t*>(a.out) + at));
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            *reinterpret_cast<i32x4_any4t*>(static_cast<float*>(a.out) + at + 4 * h) =
                i32x4{__float_as_int(x[4 * h]), __float_as_int(x[4 * h + 1]), __float_as_int(x[4 * h + 2]), __float_as_int(x[4 * h + 3])};
        }
      } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (n + e < a.N) {
            if (a.out_dtype == GS_BF16) static_cast<uint16_t*>(a.out)[at + e] = float_to_bf16_bits(x[e]);
            else static_cast<float*>(a.out)[at + e] = x[e];
          }
      }
    }
  });
}

// The part of a tile's slabs that a workgroup has, of `all`: whole fours.
__device__ __forceinline__ void f8_slabs_of(int all, int part, int parts, int* lo, int* hi) {
  const int fours = (all + 3) / 4, per = fours / parts, more = fours % parts;
  const int first = part * per + (part < more ? part : more), end = first + per + (part < more ? 1 : 0);
  *lo = first * 4;
  *hi = end * 4 < all ? end * 4 : all;
}

// (A closure that is called in several places would otherwise be left a function, and its registers be memory.)
#define GS_INLINE __attribute__((always_inline))

// W1: w has a scale for each row.
template <int BM, int BN, int WGM, int WGN, int NS, int SPREAD, bool W1, bool GROUPED>
__global__ void __launch_bounds__(WGM * WGN * 64, 2) f8_dot_tile_kernel(F8DotArgs a, uint32_t tiles_m, uint32_t tiles_n) {
  constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, MI = WM / 16, NJ = WN / 16;
  constexpr int XQ = BM / 8 / NW, YQ = BN / 8 / NW, VQ = XQ + YQ;  // transfers of values per wave and slab: 8 rows each
  static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BN % 64 == 0 && WN <= 128 && NJ % 2 == 0, "whole transfers");
  static_assert(NW % 2 == 0, "the exchange of columns must not depend on q");
  static_assert(NS >= 2 && NS <= 4, "two buffers of scales are enough");
  constexpr int kSX = (BM + 63) / 64, kSW = W1 ? BN / 64 : 1, kSAll = kSX + kSW, SQ = (kSAll + NW - 1) / NW;   // of scales, per four slabs: 64 rows each
  constexpr int kX = BM * 128, kBuf = (BM + BN) * 128, kSBuf = kSAll * 1024;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WGN, wn = wave % WGN;
  uint32_t tm, tn;
  F8Rows rows = {0, a.M, 0};
  int part = 0;
  if constexpr (GROUPED) {
    tiles_m = uint32_t(f8_group_tiles(a, BM));
    if (blockIdx.x >= tiles_m * tiles_n) return;
    mx4_tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, &tm, &tn);
    rows = f8_group_tile(a, tm, BM);
    if (rows.end <= rows.first) return;           // (only where offsets are written meanwhile, by a program's mistake)
  } else {
    const uint32_t tiles = tiles_m * tiles_n;
    part = int(blockIdx.x / tiles);
    mx4_tile_of(blockIdx.x - uint32_t(part) * tiles, tiles, tiles_m, tiles_n, &tm, &tn);
    rows.first = int64_t(tm) * BM;
  }
  const int64_t m0 = rows.first, n0 = int64_t(tn) * BN;
  const uint32_t row_bytes = uint32_t(a.K);
  int s, s_end;
  f8_slabs_of(int(a.K / kF8Block), part, GROUPED ? 1 : a.splits, &s, &s_end);
  const int s_first = s;

  // sources: a base per operand and slab, and an offset per lane and transfer; rows behind the end are the last row
  const int64_t w_scale_rows = W1 ? a.N : (a.N + 127) / 128;
  const uint8_t* const xb = GROUPED ? a.x : a.x + m0 * a.K;
  const uint8_t* const yb = a.w + (rows.expert * a.N + n0) * a.K;
  const int32_t m_last = int32_t(rows.end - m0 < BM ? rows.end - m0 : BM) - 1, n_last = int32_t(a.N - n0 < BN ? a.N - n0 : BN) - 1;
  const int lrow = lane / 8, lcol = ((lane % 8) ^ ((lrow / 2 + 4 * (wave & 1)) % 8)) * 16;    // (8 rows per transfer: row / 2 = 4 t + lrow / 2)
  auto x_row = [&](int32_t row) {                                  // of x (from xb on) for a row of the tile
    const int32_t r = row < m_last ? row : m_last;
    if constexpr (!GROUPED) return int64_t(r);
    const int64_t t = f8_x_row(a, m0 + r);
    return t < 0 ? int64_t(0) : t;
  };
  uint32_t xo[XQ], yo[YQ];
#pragma unroll
  for (int q = 0; q < XQ; ++q) xo[q] = uint32_t(x_row((wave + q * NW) * 8 + lrow)) * row_bytes + uint32_t(lcol);
#pragma unroll
  for (int q = 0; q < YQ; ++q) {
    const int32_t row = (wave + q * NW) * 8 + lrow;
    yo[q] = uint32_t(row < n_last ? row : n_last) * row_bytes + uint32_t(lcol);
  }
  // (with more waves than transfers of scales some are made twice, so that every wave counts the same number)
  const float* sp[SQ];
#pragma unroll
  for (int q = 0; q < SQ; ++q) {
    const int piece = (wave + q * NW) % kSAll;
    if (piece < kSX) {
      const int64_t row = x_row(piece * 64 + lane) + (GROUPED ? 0 : m0);
      sp[q] = a.xs + (a.x_rows == 1 ? row : row / 128) * a.pitch;
    } else {
      const int32_t r = (piece - kSX) * 64 + lane;
      const int64_t row = W1 ? n0 + (r < n_last ? r : n_last) : (n0 + (r * 128 < n_last ? r * 128 : n_last)) / 128;
      sp[q] = a.ws + (rows.expert * w_scale_rows + row) * a.pitch;
    }
  }

  const uint32_t lds0 = lds_addr_of(lds);
  auto issue_values = [&](int slab, int buf, auto idx_) GS_INLINE {
    constexpr int i = decltype(idx_)::value;
    const uint32_t base = lds0 + uint32_t(buf) * kBuf;
    if constexpr (i < XQ) lds_dma16_off(xb + int64_t(slab) * 128, xo[i], base + (wave + i * NW) * 1024);
    else lds_dma16_off(yb + int64_t(slab) * 128, yo[i - XQ], base + kX + (wave + (i - XQ) * NW) * 1024);
  };
  auto issue_scales = [&](int slab) GS_INLINE {                              // of the four slabs from this one on
    const uint32_t base = lds0 + NS * kBuf + uint32_t(((slab - s_first) / 4) & 1) * kSBuf;
#pragma unroll
    for (int q = 0; q < SQ; ++q) lds_dma16(sp[q] + slab, base + (wave + q * NW) % kSAll * 1024);
  };

  f32x4 tot[MI][NJ];
  static_for<MI>([&](auto m_) { static_for<NJ>([&](auto n_) { tot[decltype(m_)::value][decltype(n_)::value] = f32x4{0, 0, 0, 0}; }); });

  // fragment addresses in the buffer being read: columns g and g + 4 of row lane % 16
  const uint8_t *xa[2], *ya[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int col = (((lane >> 4) + 4 * c) ^ (((lane & 15) / 2) % 8)) * 16;
    xa[c] = lds + (wm * WM + (lane & 15)) * 128 + col;
    ya[c] = lds + kX + (wn * WN + (lane & 15)) * 128 + col;
  }
  const uint8_t* const sx = lds + NS * kBuf + (wm * WM + (lane & 15)) * 16;
  const uint8_t* const sw = lds + NS * kBuf + kSX * 1024 + (W1 ? (wn * WN + 4 * (lane >> 4)) * 16 : wn * WN / 128 * 16);

  i32x4 xf[MI][2], wf[2][2];
  float xs[MI];
  f32x4 wr[NJ];                       // W1: the scales of this lane's rows of w
  auto request_x = [&](auto m_) GS_INLINE {
    constexpr int m = decltype(m_)::value;
#pragma unroll
    for (int c = 0; c < 2; ++c) xf[m][c] = *reinterpret_cast<const i32x4*>(xa[c] + m * 16 * 128);
  };
  auto request_w = [&](auto n_) GS_INLINE {
    constexpr int n = decltype(n_)::value;
#pragma unroll
    for (int c = 0; c < 2; ++c) wf[n & 1][c] = *reinterpret_cast<const i32x4*>(ya[c] + n * 16 * 128);
  };
  float next_xs[MI], next_ws = 0.0f;
  f32x4 next_wr[NJ];
  auto request_scales = [&](int slab) GS_INLINE {
    const int at = (((slab - s_first) / 4) & 1) * kSBuf + (slab & 3) * 4;
    static_for<MI>([&](auto m_) { next_xs[decltype(m_)::value] = *reinterpret_cast<const float*>(sx + at + decltype(m_)::value * 256); });
    if constexpr (W1) {
      static_for<NJ>([&](auto n_) {
        constexpr int n = decltype(n_)::value;
#pragma unroll
        for (int e = 0; e < 4; ++e) next_wr[n][e] = *reinterpret_cast<const float*>(sw + at + n * 256 + e * 16);
      });
    } else {
      next_ws = *reinterpret_cast<const float*>(sw + at);
    }
  };
  auto take_scales = [&]() GS_INLINE {
    static_for<MI>([&](auto m_) { xs[decltype(m_)::value] = W1 ? next_xs[decltype(m_)::value] : next_xs[decltype(m_)::value] * next_ws; });
    if constexpr (W1) static_for<NJ>([&](auto n_) { wr[decltype(n_)::value] = next_wr[decltype(n_)::value]; });
  };
  // Products wait for their addition in a ring: that of a product follows the one R - 1 behind it, so that the vector unit never
  // waits for the matrix unit.
  constexpr int R = 3;
  f32x4 p[R];
  auto multiply = [&](auto t_) GS_INLINE {
    constexpr int t = decltype(t_)::value, n = t / MI, m = t % MI;
    p[t % R] = f8_mfma16(wf[n & 1], xf[m]);
  };
  auto add = [&](auto t_) GS_INLINE {
    constexpr int t = decltype(t_)::value, n = t / MI, m = t % MI;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (W1) tot[m][n][e] += xs[m] * wr[n][e] * p[t % R][e];
      else tot[m][n][e] += xs[m] * p[t % R][e];
    }
    asm volatile("" : "+v"(tot[m][n]));         // here, not behind the next branch: that would keep all of a slab's products
  };
  auto step = [&](auto t_) GS_INLINE {
    constexpr int t = decltype(t_)::value;
    multiply(t_);
    if constexpr (t >= R - 1) add(std::integral_constant<int, t - (R - 1)>{});
  };
  int buf = 0;
  using I0 = std::integral_constant<int, 0>;
  constexpr int kLast = (NJ - 1) * MI, kAll = NJ * MI;             // products in front of the last column's
  auto rest = [&]() GS_INLINE { static_for<R - 1>([&](auto i_) { add(std::integral_constant<int, kAll - (R - 1) + decltype(i_)::value>{}); }); };
  // What of a slab's transfers is requested as soon as its buffer is drained; the rest is requested SPREAD to a column of the slab
  // that follows: a wave waits while it requests, and where products take as long as transfers those of a burst would have them wait
  // together (256x256 tiles, four to a column: 8192 cubed 448 -> 439 us, 3000 cubed 42.6 -> 39.7).
  constexpr int kAtOnce = SPREAD > 0 && VQ > SPREAD * (NJ - 1) ? VQ - SPREAD * (NJ - 1) : SPREAD > 0 ? 0 : VQ;
  int drained = 0;
  auto columns = [&](auto rest_) GS_INLINE {    // all columns of a slab but the last; rest_: transfers are left to be requested
    static_for<NJ - 1>([&](auto n_) {
      constexpr int n = decltype(n_)::value;
      request_w(std::integral_constant<int, n + 1>{});
      __builtin_amdgcn_sched_barrier(0);
      static_for<(MI > SPREAD ? MI : SPREAD)>([&](auto m_) {
        constexpr int m = decltype(m_)::value, i = kAtOnce + n * SPREAD + m;
        if constexpr (m < MI) step(std::integral_constant<int, n * MI + m>{});
        if constexpr (m < SPREAD && i < VQ) {
          if (rest_) issue_values(s + NS - 1, drained, std::integral_constant<int, i>{});
          __builtin_amdgcn_sched_barrier(0);
        }
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // One slab that another follows.  ISSUE: slab s + NS exists and is requested.
  auto full_slab = [&](auto issue_, auto rest_) GS_INLINE {
    constexpr bool ISSUE = decltype(issue_)::value;
    columns(rest_);
    if constexpr (ISSUE) wait_vmem<(NS - 2) * VQ>();
    else wait_vmem<0>();
    lds_barrier_tracked();
    drained = buf;
    const bool wrap = buf + 1 == NS;
    buf = wrap ? 0 : buf + 1;
    const int d = wrap ? -(NS - 1) * kBuf : kBuf;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      xa[c] += d;
      ya[c] += d;
    }
    request_w(I0{});
    request_scales(s + 1);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (ISSUE)
      if (((s + NS - s_first) & 3) == 0) issue_scales(s + NS);
    static_for<(MI > kAtOnce ? MI : kAtOnce)>([&](auto i_) {
      constexpr int i = decltype(i_)::value;
      if constexpr (i < MI) {
        step(std::integral_constant<int, kLast + i>{});
        request_x(i_);
      }
      if constexpr (ISSUE && i < kAtOnce) issue_values(s + NS, drained, i_);
      __builtin_amdgcn_sched_barrier(0);
    });
    rest();
    take_scales();
    ++s;
  };

  if (s < s_end) {
    static_for<NS>([&](auto b_) {
      constexpr int b = decltype(b_)::value;
      if (s + b < s_end) {
        if constexpr (b == 0) issue_scales(s);
        static_for<VQ>([&](auto i_) { issue_values(s + b, b, i_); });
      }
    });
    asm volatile("" ::"s"(a.relu), "s"(a.M), "s"(a.N), "s"(a.out), "s"(a.out_dtype));   // not in the loop: scalar loads share a counter with LDS
    if (s + NS <= s_end) wait_vmem<(NS - 1) * VQ>();
    else wait_vmem<0>();
    lds_barrier_tracked();
    request_w(I0{});
    static_for<MI>([&](auto m_) { request_x(m_); });
    request_scales(s);
    take_scales();
    if (s + NS < s_end) full_slab(std::true_type{}, std::false_type{});
    while (s + NS < s_end) full_slab(std::true_type{}, std::true_type{});
    while (s + 1 < s_end) full_slab(std::false_type{}, s > s_first && s + NS - 1 < s_end);
    columns(s > s_first && s + NS - 1 < s_end);
    static_for<MI>([&](auto m_) { step(std::integral_constant<int, kLast + decltype(m_)::value>{}); });
    rest();
  }
  uint32_t zero = 0;
  if constexpr (GROUPED) {
#pragma unroll
    for (int m = 0; m < MI; ++m) {
      const int32_t row = wm * WM + m * 16 + (lane & 15);
      if (row <= m_last && f8_x_row(a, m0 + row) < 0) zero |= 1u << m;
    }
  }
  __syncthreads();
  f8_write_back<MI, NJ>(a, tot, m0 + wm * WM, rows.end, n0 + wn * WN, part, zero, reinterpret_cast<float*>(lds) + wave * 16 * (WN + 4), lane);
}

// Tiles of `size` rows, at most.
inline int64_t f8_most_tiles(const F8DotArgs& a, int64_t size) {
  return a.offsets ? a.M / size + (a.experts < a.M ? a.experts : a.M) : ceil_div(a.M, size);
}
template <int BM, int BN, int WGM, int WGN, int NS, int SPREAD, bool W1, bool GROUPED>
hipError_t launch_f8_tiles_as(const F8DotArgs& a, hipStream_t s) {
  constexpr int slabs = NS * (BM + BN) * 128 + 2 * 1024 * ((BM + 63) / 64 + (W1 ? BN / 64 : 1)), staging = WGM * WGN * 16 * (BN / WGN + 4) * 4;
  constexpr int bytes = slabs > staging ? slabs : staging;
  static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
  const int64_t tiles_m = f8_most_tiles(a, BM), tiles_n = ceil_div(a.N, BN);
  if (tiles_m * tiles_n > 0x00ffffff) return hipErrorInvalidValue;
  const auto kernel = f8_dot_tile_kernel<BM, BN, WGM, WGN, NS, SPREAD, W1, GROUPED>;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kernel, dim3(unsigned(tiles_m * tiles_n * a.splits)), dim3(WGM * WGN * 64), bytes, s, a, uint32_t(tiles_m), uint32_t(tiles_n));
  return hipGetLastError();
}
template <int BM, int BN, int WGM, int WGN, int NS, int SPREAD = 0>
hipError_t launch_f8_tiles(const F8DotArgs& a, hipStream_t s) {
  if (a.w_rows != 1)
    return a.offsets ? launch_f8_tiles_as<BM, BN, WGM, WGN, NS, SPREAD, false, true>(a, s) : launch_f8_tiles_as<BM, BN, WGM, WGN, NS, SPREAD, false, false>(a, s);
  // (scales for each row of w need more registers than the largest tile leaves)
  if constexpr (BM * BN > 128 * 256) return launch_f8_tiles<128, 256, 2, 4, 3>(a, s);
  else return a.offsets ? launch_f8_tiles_as<BM, BN, WGM, WGN, NS, SPREAD, true, true>(a, s) : launch_f8_tiles_as<BM, BN, WGM, WGN, NS, SPREAD, true, false>(a, s);
}

}  // namespace

}  // namespace gs
