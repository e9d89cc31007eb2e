// Tiles of products of bfloat16 rows with microscaled 4-bit weights, for more rows than mx4_dot_rows_kernel has tiles for.
//
// A slab is 128 numbers of K per row: 256 bytes of x, 64 bytes of codes (4 blocks) and 4 scale bytes, moved global -> LDS as they are;
// a wave converts the codes of its columns between the reading of a fragment and the products, exactly, so that LDS and memory carry
// 4 bits per weight.  Lane (r = lane % 32, h = lane / 32) has blocks 2 h and 2 h + 1 of its row, 8 numbers of them per 32x32x16
// product; x's 16-byte columns are read in the same order.  Columns of LDS rows are exchanged by an XOR of the row as in
// mx4_tile.h.  In the last slab, x behind K is replaced by zeros where it is read; blocks behind K have the slab's first codes and
// a scale of zero bytes.
//
// Bound by the products where tiles fill the chip (4096 x 8192 x 8192 in 128x256 tiles 506 us, 1.09 PFLOP/s), else by the slabs that
// one workgroup takes in turn, 0.46 us each in 32x128 and 64x64 tiles: then workgroups share a tile's slabs, and their parts are added by a second
// kernel (50 x 5000 x 4104 15.7 us alone, 11.7 by threes).  A slab's scales are a line of memory for each row: every one is requested once (by
// each wave that had room: 512 x 1024 x 16384 36.8 us against 32.9).
#pragma once

#include "mx4_tile.h"

namespace gs {

// The part of a tile's slabs that a workgroup has, of `all`.
struct Mx4Slabs {
  int first, end;
};
__device__ __forceinline__ Mx4Slabs mx4_slabs_of(int all, uint32_t part, uint32_t parts) {
  const int per = all / int(parts), more = all % int(parts), p = int(part);
  const int lo = p * per + (p < more ? p : more);
  return Mx4Slabs{lo, lo + per + (p < more ? 1 : 0)};
}

template <int BM, int BN, int WGM, int WGN, int NS>
__global__ void __launch_bounds__(WGM * WGN * 64) mx4_weight_tile_kernel(Mx4DotArgs a, int64_t ldx, uint32_t tiles_m, uint32_t tiles_n) {
  constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, MI = WM / 32, NJ = WN / 32;
  static_assert(BM % (4 * NW) == 0 && BN % 16 == 0 && NW % 4 == 0, "whole transfers");
  constexpr int XQ = BM / 4 / NW;                                  // transfers of x per wave and slab: 4 rows each
  constexpr int kWAll = BN / 16, WQ = kWAll / NW;                  // of codes: 16 rows each
  constexpr int kSAll = (BN + 63) / 64;                            // of scales: 64 rows each, in lines of their own, by the first waves
  static_assert(kSAll <= NW && kWAll % NW == 0, "one of scales at most, codes dealt evenly");
  constexpr int Q = XQ + WQ;                                       // of every wave; one more of the first kSAll
  constexpr int kX = BM * 256, kW = BN * 64, kBuf = kX + kW + kSAll * 256;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WGN, wn = wave % WGN;
  uint32_t tm, tn;
  const uint32_t tiles = tiles_m * tiles_n, part = blockIdx.x / tiles;
  mx4_tile_of(blockIdx.x - part * tiles, tiles, tiles_m, tiles_n, &tm, &tn);
  const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
  const int64_t nb = mx4_blocks(a.K), pitch = mx4_scale_pitch(a.K);
  const int nslab = int((a.K + 127) / 128);                        // of K; this workgroup has some of them
  const Mx4Slabs mine = mx4_slabs_of(nslab, part, uint32_t(a.splits));
  const int tail = int(a.K - int64_t(nslab - 1) * 128);            // numbers of the last slab
  const int x_tail = (tail + 7) / 8, w_tail = (tail + 31) / 32;    // in 16-byte columns (K is a multiple of 8)

  const uint8_t* const xb = static_cast<const uint8_t*>(a.x) + m0 * ldx * 2;
  const uint8_t* const wb = static_cast<const uint8_t*>(a.w) + n0 * nb * 16;
  const uint8_t* const sb = a.ws + n0 * pitch;
  const int32_t m_last = int32_t(a.M - m0 < BM ? a.M - m0 : BM) - 1, n_last = int32_t(a.N - n0 < BN ? a.N - n0 : BN) - 1;
  const int xcol = (lane & 15) ^ (4 * (wave & 3) + lane / 16);     // row % 16 = 4 (transfer % 4) + lane / 16
  const int wcol = (lane & 3) ^ ((lane / 16) & 3);                 // row / 4 % 4
  uint32_t xo[XQ], wo[WQ];
#pragma unroll
  for (int q = 0; q < XQ; ++q) {
    const int32_t row = (wave + q * NW) * 4 + lane / 16;
    xo[q] = uint32_t(row < m_last ? row : m_last) * uint32_t(ldx * 2) + uint32_t(xcol * 16);
  }
#pragma unroll
  for (int q = 0; q < WQ; ++q) {
    const int32_t row = (wave + q * NW) * 16 + lane / 4;
    wo[q] = uint32_t(row < n_last ? row : n_last) * uint32_t(nb * 16) + uint32_t(wcol * 16);
  }
  const bool has_scales = wave < kSAll;
  const int32_t scale_row = wave * 64 + lane;
  const uint32_t so = uint32_t(scale_row < n_last ? scale_row : n_last) * uint32_t(pitch);
  const uint32_t x_fix = xcol >= x_tail ? uint32_t(xcol * 16) : 0u, w_fix = wcol >= w_tail ? uint32_t(wcol * 16) : 0u;

  const uint32_t lds0 = lds_addr_of(lds);
  auto issue_one = [&](int slab, int buf, auto idx_) {
    constexpr int i = decltype(idx_)::value;
    const bool last = slab == nslab - 1;
    const uint32_t base = lds0 + uint32_t(buf) * kBuf;
    if constexpr (i < XQ) lds_dma16_off(xb + int64_t(slab) * 256, xo[i] - (last ? x_fix : 0u), base + (wave + i * NW) * 1024);
    else if constexpr (i < XQ + WQ)
      lds_dma16_off(wb + int64_t(slab) * 64, wo[i - XQ] - (last ? w_fix : 0u), base + kX + (wave + (i - XQ) * NW) * 1024);
    else if (has_scales) lds_dma4_off(sb + int64_t(slab) * 4, so, base + kX + kW + wave * 256);
  };
  auto wait_slabs = [&](auto slabs_) {                             // until at most so many slabs' transfers are under way
    constexpr int slabs = decltype(slabs_)::value;
    if (has_scales) wait_vmem<slabs*(Q + 1)>();
    else wait_vmem<slabs * Q>();
  };

  f32x16 acc[MI][NJ];
  static_for<MI>([&](auto m_) {
    static_for<NJ>([&](auto n_) {
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[decltype(m_)::value][decltype(n_)::value][v] = 0;
    });
  });

  const int r = lane & 31, h = lane >> 5;
  const uint32_t x_row = uint32_t((wm * WM + r) * 256), x_swz = uint32_t(r & 15);
  const uint32_t w_row = uint32_t(kX + (wn * WN + r) * 64), w_swz = uint32_t((r / 4) & 3);
  const uint32_t s_row = uint32_t(kX + kW + (wn * WN + r) * 4);

  i32x4 xf[2][MI], wf[2][NJ], raw[NJ][2];
  float sc[NJ][2];
  auto read_x = [&](const uint8_t* base, auto step_, auto set_) {
    constexpr int step = decltype(step_)::value, set = decltype(set_)::value;
#pragma unroll
    for (int m = 0; m < MI; ++m) xf[set][m] = *reinterpret_cast<const i32x4*>(base + x_row + m * 32 * 256 + ((8 * h + step) ^ x_swz) * 16);
  };
  auto decode = [&](auto step_, auto set_) {
    constexpr int step = decltype(step_)::value, set = decltype(set_)::value;
#pragma unroll
    for (int n = 0; n < NJ; ++n) wf[set][n] = mx4_decode8(uint32_t(raw[n][step / 4][step % 4]), sc[n][step / 4]);
  };
  auto products = [&](auto set_, auto i_) {
    constexpr int set = decltype(set_)::value, i = decltype(i_)::value, m = i / NJ, n = i % NJ;
    acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, xf[set][m]), __builtin_bit_cast(bf16x8, wf[set][n]), acc[m][n], 0, 0, 0);
  };
  uint32_t raw_sc[NJ];
  auto read_w = [&](const uint8_t* base) {
#pragma unroll
    for (int n = 0; n < NJ; ++n) {
      raw_sc[n] = *reinterpret_cast<const uint32_t*>(base + s_row + n * 32 * 4);
#pragma unroll
      for (int c = 0; c < 2; ++c) raw[n][c] = *reinterpret_cast<const i32x4*>(base + w_row + n * 32 * 64 + ((2 * h + c) ^ w_swz) * 16);
    }
  };
  auto scales = [&]() {
#pragma unroll
    for (int n = 0; n < NJ; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) sc[n][c] = mx4_scale((raw_sc[n] >> (16 * h + 8 * c)) & 255u);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  int s = mine.first, buf = 0;
  // One slab that another follows; ISSUE: slab s + NS exists and is requested once this one's buffer is drained.
  auto full_slab = [&](auto issue_) {
    constexpr bool ISSUE = decltype(issue_)::value;
    const uint8_t* const base = lds + buf * kBuf;
    static_for<7>([&](auto step_) {
      constexpr int step = decltype(step_)::value, set = step & 1;
      read_x(base, std::integral_constant<int, step + 1>{}, std::integral_constant<int, set ^ 1>{});
      __builtin_amdgcn_sched_barrier(0);
      decode(std::integral_constant<int, step + 1>{}, std::integral_constant<int, set ^ 1>{});
      static_for<MI * NJ>([&](auto i_) { products(std::integral_constant<int, set>{}, i_); });
    });
    if constexpr (ISSUE) wait_slabs(std::integral_constant<int, NS - 2>{});
    else wait_vmem<0>();
    lds_barrier_tracked();
    const int done = buf;
    buf = buf + 1 == NS ? 0 : buf + 1;
    read_w(lds + buf * kBuf);
    read_x(lds + buf * kBuf, I0{}, I0{});
    __builtin_amdgcn_sched_barrier(0);
    static_for<(MI * NJ > (ISSUE ? Q + 1 : 0) ? MI * NJ : Q + 1)>([&](auto i_) {
      constexpr int i = decltype(i_)::value;
      if constexpr (i < MI * NJ) products(I1{}, i_);
      if constexpr (ISSUE && i <= Q) issue_one(s + NS, done, i_);
      __builtin_amdgcn_sched_barrier(0);
    });
    scales();
    decode(I0{}, I0{});
    ++s;
  };

  static_for<NS>([&](auto b_) {
    constexpr int b = decltype(b_)::value;
    if (s + b < mine.end) static_for<Q + 1>([&](auto i_) { issue_one(s + b, b, i_); });
  });
  asm volatile("" ::"s"(a.relu), "s"(a.M), "s"(a.N), "s"(a.out), "s"(a.out_dtype));   // not in the loop: scalar loads share a counter with LDS
  if (s + NS <= mine.end) wait_slabs(std::integral_constant<int, NS - 1>{});
  else wait_vmem<0>();
  lds_barrier_tracked();
  read_w(lds);
  read_x(lds, I0{}, I0{});
  scales();
  decode(I0{}, I0{});
  while (s + NS < mine.end) full_slab(std::true_type{});
  while (s + 1 < mine.end) full_slab(std::false_type{});
  {
    const uint8_t* const base = lds + buf * kBuf;
    static_for<8>([&](auto step_) {
      constexpr int step = decltype(step_)::value, set = step & 1;
      if constexpr (step < 7) {
        read_x(base, std::integral_constant<int, step + 1>{}, std::integral_constant<int, set ^ 1>{});
        decode(std::integral_constant<int, step + 1>{}, std::integral_constant<int, set ^ 1>{});
      }
      const bool there = s + 1 < nslab || 8 * h + step < x_tail;
#pragma unroll
      for (int m = 0; m < MI; ++m)
        if (!there) xf[set][m] = i32x4{0, 0, 0, 0};
      static_for<MI * NJ>([&](auto i_) { products(std::integral_constant<int, set>{}, i_); });
    });
  }
  __syncthreads();
  mx4_write_back<MI, NJ>(a, acc, m0 + wm * WM, n0 + wn * WN, part, reinterpret_cast<float*>(lds) + wave * 32 * (WN + 4), lane);
}

// Rows of x are ldx numbers apart, a multiple of 8 that K does not exceed and whose last 8 may be partly zeros.
template <int BM, int BN, int WGM, int WGN, int NS>
hipError_t launch_mx4_weight_tiles(const Mx4DotArgs& a, int64_t ldx, hipStream_t s) {
  constexpr int slabs = NS * (BM * 256 + BN * 64 + (BN + 63) / 64 * 256), staging = WGM * WGN * 32 * (BN / WGN + 4) * 4;
  constexpr int bytes = slabs > staging ? slabs : staging;
  static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
  const int64_t tm = ceil_div(a.M, BM), tn = ceil_div(a.N, BN);
  if (tm * tn * a.splits > 0x0fffffff) return hipErrorInvalidValue;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(mx4_weight_tile_kernel<BM, BN, WGM, WGN, NS>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((mx4_weight_tile_kernel<BM, BN, WGM, WGN, NS>), dim3(unsigned(tm * tn * a.splits)), dim3(WGM * WGN * 64), bytes, s, a, ldx, uint32_t(tm), uint32_t(tn));
  return hipGetLastError();
}

}  // namespace gs
