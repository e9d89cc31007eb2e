// Tiles of products of two microscaled 4-bit operands, moved global -> LDS without passing through registers.
//
// A slab is 128 bytes of K per row: 8 blocks, 256 numbers, with 8 scale bytes.  Rows of values are 128 bytes in LDS, their
// 16-byte columns (one block each) exchanged by an XOR of the row so that the 32 rows that a matrix instruction reads fall on
// different banks; scales lie row after row.  One 32x32x64 product takes two blocks of 32 rows of each operand: lane (r = lane % 32,
// h = lane / 32) holds block 4 h + step of row r -- any assignment of K does, as long as both operands have the same -- so that a
// row's four scales of a lane are one dword, whose byte `step` the instruction selects.
//
// Where K ends inside a slab, the columns behind it are filled with the slab's first block; their scales are zero bytes in
// both operands, 2^-254 together, so that they add nothing.
//
// Bound by power where all compute units multiply (8192 cubed: 247 to 270 us over cards on random numbers, 4.1 to 4.4 PFLOP/s) and by the
// transfers.  Scales are a seventeenth of the bytes, but 8 per row and slab are a transfer instruction for 32 rows, each in a
// line of its own, and cost as much as half of the values (8192 cubed, an earlier state of this kernel: 319 us against 279 without them): where rows of scales are whole
// runs of 16 (PAIRED: K above a multiple of 512 by more than 256, or a multiple of it), those of two slabs come together.  Results are
// stored with the streaming hint (4096 cubed 39.5 -> 35.5 us, 2048 x 8192 x 8192 69.9 -> 63.2).
#pragma once

#include "mx4.h"

namespace gs {

typedef int32_t i32x8t __attribute__((ext_vector_type(8)));
typedef int32_t i32x4_any2t __attribute__((ext_vector_type(4), aligned(2)));
typedef int32_t i32x4_any4t __attribute__((ext_vector_type(4), aligned(4)));

// 4 bytes per lane, global -> LDS: lane i lands at lds_base + 4 i (see lds_dma16).
__device__ __forceinline__ void lds_dma4_off(const void* base, uint32_t byte_off, uint32_t lds_base) {
  const uint32_t lb = __builtin_amdgcn_readfirstlane(lds_base);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :: "v"(byte_off), "s"(base), "s"(lb) : "memory", "m0");
}

// The tile of a workgroup: each of the 8 XCDs (whose workgroups are every eighth) gets a compact region of the grid, in
// bands of 8 tile rows.
__device__ __forceinline__ void mx4_tile_of(uint32_t id, uint32_t count, uint32_t tiles_m, uint32_t tiles_n, uint32_t* tm, uint32_t* tn) {
  const uint32_t per = count / 8, rem = count % 8, x = id % 8;
  const uint32_t at = x * per + (x < rem ? x : rem) + id / 8;
  const uint32_t band = at / (8 * tiles_n), in = at - band * 8 * tiles_n;
  const uint32_t rows = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
  *tn = in / rows;
  *tm = band * 8 + (in - *tn * rows);
}

// One wave's results: 32x32 blocks whose lane has column lane % 32 and rows 8 (v / 4) + 4 (lane / 32) + v % 4, staged 32 rows at
// a time in LDS of its own (32 rows of 32 NJ + 4 floats) and written 8 columns per lane, into part `part` of the results.
template <int MI, int NJ>
__device__ __forceinline__ void mx4_write_back(const Mx4DotArgs& a, f32x16 (&acc)[MI][NJ], int64_t m0, int64_t n0, int64_t part, float* stage, int lane) {
  constexpr int WN = NJ * 32, RS = WN + 4, LPR = WN / 8, RPP = 64 / LPR, NP = 32 / RPP;
  const int cq = (lane % LPR) * 8, rsub = lane / LPR;
  const int64_t n = n0 + cq;
  static_for<MI>([&](auto m_) {
    constexpr int m = decltype(m_)::value;
    static_for<NJ>([&](auto n_) {
      constexpr int j = decltype(n_)::value;
#pragma unroll
      for (int v = 0; v < 16; ++v) stage[(8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * RS + j * 32 + (lane & 31)] = acc[m][j][v];
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
      const int64_t row = m0 + m * 32 + p * RPP + rsub;
      if (row >= a.M || n >= a.N) continue;
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

template <int BM, int BN, int WGM, int WGN, int NS, bool PAIRED>
__global__ void __launch_bounds__(WGM * WGN * 64) mx4_dot_tile_kernel(Mx4DotArgs a, uint32_t tiles_m, uint32_t tiles_n) {
  constexpr int NW = WGM * WGN, WM = BM / WGM, WN = BN / WGN, MI = WM / 32, NJ = WN / 32;
  constexpr int XQ = BM / 8 / NW, YQ = BN / 8 / NW;                // transfers of values per wave and slab: 8 rows each
  static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM % 64 == 0 && BN % 64 == 0, "whole transfers");
  static_assert(!PAIRED || NS % 2 == 0, "pairs of slabs");
  // transfers of scales, per slab or pair of slabs: 32 rows of 8 bytes, or 64 rows of 16
  constexpr int kSRow = PAIRED ? 16 : 8, kSRows = PAIRED ? 64 : 32, kSAll = (BM + BN) / kSRows, SQ = (kSAll + NW - 1) / NW;
  constexpr int VQ = XQ + YQ;
  // how many a wave may leave under way: those of the slabs behind the one that it waits for
  constexpr int kFirstWait = PAIRED ? (NS - 1) * VQ + (NS - 1) / 2 * SQ : (NS - 1) * (VQ + SQ);
  constexpr int kWait = PAIRED ? (NS - 2) * VQ + (NS - 2) / 2 * SQ : (NS - 2) * (VQ + SQ);
  constexpr int kX = BM * 128, kBuf = (BM + BN) * 128, kSBuf = (BM + BN) * kSRow, kSBufs = PAIRED ? NS / 2 + 1 : NS;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WGN, wn = wave % WGN;
  uint32_t tm, tn;
  mx4_tile_of(blockIdx.x, gridDim.x, tiles_m, tiles_n, &tm, &tn);
  const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
  const int64_t nb = mx4_blocks(a.K), pitch = mx4_scale_pitch(a.K);
  const int nslab = int(pitch / 8);
  const int tail = int(nb - int64_t(nslab - 1) * 8);                // blocks of the last slab

  // sources: a base per operand and slab, and an offset per lane and transfer; rows behind the end are the last row
  const uint8_t* const xb = static_cast<const uint8_t*>(a.x) + m0 * nb * 16;
  const uint8_t* const yb = static_cast<const uint8_t*>(a.w) + n0 * nb * 16;
  const uint8_t* const xsb = a.xs + m0 * pitch;
  const uint8_t* const ysb = a.ws + n0 * pitch;
  const int32_t m_last = int32_t(a.M - m0 < BM ? a.M - m0 : BM) - 1, n_last = int32_t(a.N - n0 < BN ? a.N - n0 : BN) - 1;
  const int lrow = lane / 8, lcol = ((lane % 8) ^ ((lrow / 2 + 4 * (wave & 1)) % 8)) * 16;    // (8 rows per transfer: row / 2 = 4 t + lrow / 2)
  static_assert(NW % 2 == 0, "the exchange of columns must not depend on q");
  uint32_t xo[XQ], yo[YQ], so[SQ];
#pragma unroll
  for (int q = 0; q < XQ; ++q) {
    const int32_t row = (wave + q * NW) * 8 + lrow;
    xo[q] = uint32_t(row < m_last ? row : m_last) * uint32_t(nb * 16) + uint32_t(lcol);
  }
#pragma unroll
  for (int q = 0; q < YQ; ++q) {
    const int32_t row = (wave + q * NW) * 8 + lrow;
    yo[q] = uint32_t(row < n_last ? row : n_last) * uint32_t(nb * 16) + uint32_t(lcol);
  }
  // (with more waves than transfers of scales some are made twice, so that every wave counts the same number)
#pragma unroll
  for (int q = 0; q < SQ; ++q) {
    const int32_t row = (wave + q * NW) % kSAll * kSRows + lane / (64 / kSRows), at = row < BM ? row : row - BM, last = row < BM ? m_last : n_last;
    so[q] = uint32_t(at < last ? at : last) * uint32_t(pitch) + uint32_t(PAIRED ? 0 : lane % 2 * 4);
  }
  const uint32_t tail_fix = lcol >= tail * 16 ? uint32_t(lcol) : 0u;

  const uint32_t lds0 = lds_addr_of(lds);
  auto issue_values = [&](int slab, int buf, auto idx_) {
    constexpr int i = decltype(idx_)::value;
    const uint32_t fix = slab == nslab - 1 ? tail_fix : 0u;
    const uint32_t base = lds0 + uint32_t(buf) * kBuf;
    if constexpr (i < XQ) lds_dma16_off(xb + int64_t(slab) * 128, xo[i] - fix, base + (wave + i * NW) * 1024);
    else lds_dma16_off(yb + int64_t(slab) * 128, yo[i - XQ] - fix, base + kX + (wave + (i - XQ) * NW) * 1024);
  };
  auto issue_scales = [&](int slab, int sbuf, auto idx_) {
    constexpr int i = decltype(idx_)::value;
    const int piece = (wave + i * NW) % kSAll;
    const uint8_t* src = (piece * kSRows < BM ? xsb : ysb) + int64_t(slab) * 8;
    const uint32_t dst = lds0 + NS * kBuf + uint32_t(sbuf) * kSBuf + piece * kSRows * kSRow;
    if constexpr (PAIRED) lds_dma16_off(src, so[i], dst);
    else lds_dma4_off(src, so[i], dst);
  };

  f32x16 acc[MI][NJ];
  static_for<MI>([&](auto m_) {
    static_for<NJ>([&](auto n_) {
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[decltype(m_)::value][decltype(n_)::value][v] = 0;
    });
  });

  // fragment addresses in buffer 0: block 4 h + step of row lane % 32
  const uint8_t *xa[4], *ya[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int col = ((4 * (lane >> 5) + s) ^ (((lane & 31) / 2) % 8)) * 16;
    xa[s] = lds + (wm * WM + (lane & 31)) * 128 + col;
    ya[s] = lds + kX + (wn * WN + (lane & 31)) * 128 + col;
  }
  const uint8_t* const xsa = lds + NS * kBuf + (wm * WM + (lane & 31)) * kSRow + (lane >> 5) * 4;
  const uint8_t* const ysa = lds + NS * kBuf + (BM + wn * WN + (lane & 31)) * kSRow + (lane >> 5) * 4;

  // The K loop: fragments of step k + 1 are requested in front of the products of step k; the barrier of a slab
  // sits in front of the products of its last step; transfers into the buffer just drained go between those.
  i32x4 fr[2][MI + NJ];
  int32_t sc[2][MI + NJ];             // scales of this slab and of the next
  auto request = [&](auto step_, auto set_) {
    constexpr int step = decltype(step_)::value, set = decltype(set_)::value;
#pragma unroll
    for (int m = 0; m < MI; ++m) fr[set][m] = *reinterpret_cast<const i32x4*>(xa[step] + m * 32 * 128);
#pragma unroll
    for (int n = 0; n < NJ; ++n) fr[set][MI + n] = *reinterpret_cast<const i32x4*>(ya[step] + n * 32 * 128);
  };
  auto request_scales = [&](int set, int sbuf, int odd) {
    const int at = sbuf * kSBuf + odd * 8;
#pragma unroll
    for (int m = 0; m < MI; ++m) sc[set][m] = *reinterpret_cast<const int32_t*>(xsa + at + m * 32 * kSRow);
#pragma unroll
    for (int n = 0; n < NJ; ++n) sc[set][MI + n] = *reinterpret_cast<const int32_t*>(ysa + at + n * 32 * kSRow);
  };
  auto product = [&](auto step_, auto set_, auto m_, auto n_) {
    constexpr int step = decltype(step_)::value, set = decltype(set_)::value, m = decltype(m_)::value, n = decltype(n_)::value;
    const i32x4 x = fr[set][m], y = fr[set][MI + n];
    const i32x8t x8 = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, y8 = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
    acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x8, y8, acc[m][n], 4, 4, step, sc[0][m], step, sc[0][MI + n]);
  };
  using I0 = std::integral_constant<int, 0>;
  int s = 0, buf = 0, sbuf = 0;       // the slab being multiplied, its buffer, that of its scales
  // One slab that another follows.  ISSUE: slab s + NS exists and is requested; ODD: s is odd (of interest where paired).
  auto full_slab = [&](auto issue_, auto odd_) {
    constexpr bool ISSUE = decltype(issue_)::value, ODD = decltype(odd_)::value;
    constexpr int TQ = ISSUE ? VQ + (PAIRED && ODD ? 0 : SQ) : 0;
    static_for<4>([&](auto step_) {
      constexpr int step = decltype(step_)::value, set = step & 1;
      if constexpr (step < 3) {
        request(std::integral_constant<int, step + 1>{}, std::integral_constant<int, set ^ 1>{});
        __builtin_amdgcn_sched_barrier(0);
        static_for<MI * NJ>([&](auto i_) {
          constexpr int i = decltype(i_)::value;
          product(step_, std::integral_constant<int, set>{}, std::integral_constant<int, i / NJ>{}, std::integral_constant<int, i % NJ>{});
        });
        __builtin_amdgcn_sched_barrier(0);
      } else {
        if constexpr (ISSUE) wait_vmem<kWait>();
        else wait_vmem<0>();
        lds_barrier_tracked();
        const int done = buf;
        const bool wrap = buf + 1 == NS;
        buf = wrap ? 0 : buf + 1;
        const int d = wrap ? -(NS - 1) * kBuf : kBuf;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          xa[k] += d;
          ya[k] += d;
        }
        // where the scales of slab s + NS go: unpaired, into the buffer just drained; paired, into the one that
        // the pair in front of this one had
        const int into = PAIRED ? (sbuf == 0 ? kSBufs - 1 : sbuf - 1) : done;
        if (!PAIRED || ODD) sbuf = sbuf + 1 == kSBufs ? 0 : sbuf + 1;
        request(I0{}, std::integral_constant<int, set ^ 1>{});
        request_scales(1, sbuf, PAIRED && !ODD);
        __builtin_amdgcn_sched_barrier(0);
        static_for<(MI * NJ > TQ ? MI * NJ : TQ)>([&](auto i_) {
          constexpr int i = decltype(i_)::value;
          if constexpr (i < MI * NJ) product(step_, std::integral_constant<int, set>{}, std::integral_constant<int, i / NJ>{}, std::integral_constant<int, i % NJ>{});
          if constexpr (i < TQ) {
            if constexpr (i < VQ) issue_values(s + NS, done, i_);
            else issue_scales(s + NS, into, std::integral_constant<int, i - VQ>{});
          }
          __builtin_amdgcn_sched_barrier(0);
        });
#pragma unroll
        for (int i = 0; i < MI + NJ; ++i) sc[0][i] = sc[1][i];
        ++s;
      }
    });
  };

  static_for<NS>([&](auto b_) {
    constexpr int b = decltype(b_)::value;
    if (b < nslab) {
      static_for<VQ>([&](auto i_) { issue_values(b, b, i_); });
      if constexpr (!PAIRED || b % 2 == 0) static_for<SQ>([&](auto i_) { issue_scales(b, PAIRED ? b / 2 : b, i_); });
    }
  });
  asm volatile("" ::"s"(a.relu), "s"(a.M), "s"(a.N), "s"(a.out), "s"(a.out_dtype));   // not in the loop: scalar loads share a counter with LDS
  if (nslab >= NS) wait_vmem<kFirstWait>();
  else wait_vmem<0>();
  lds_barrier_tracked();
  request(I0{}, I0{});
  request_scales(0, 0, 0);
  if constexpr (PAIRED) {             // (an even number of slabs, from an even one on)
    while (s + NS < nslab) {
      full_slab(std::true_type{}, std::false_type{});
      full_slab(std::true_type{}, std::true_type{});
    }
    static_for<NS - 1>([&](auto i_) {
      if (s + 1 < nslab) full_slab(std::false_type{}, std::integral_constant<bool, (decltype(i_)::value & 1) != 0>{});
    });
  } else {
    while (s + NS < nslab) full_slab(std::true_type{}, std::false_type{});
    while (s + 1 < nslab) full_slab(std::false_type{}, std::false_type{});
  }
  static_for<4>([&](auto step_) {
    constexpr int step = decltype(step_)::value, set = step & 1;
    if constexpr (step < 3) request(std::integral_constant<int, step + 1>{}, std::integral_constant<int, set ^ 1>{});
    static_for<MI * NJ>([&](auto i_) {
      constexpr int i = decltype(i_)::value;
      product(step_, std::integral_constant<int, set>{}, std::integral_constant<int, i / NJ>{}, std::integral_constant<int, i % NJ>{});
    });
  });
  __syncthreads();
  mx4_write_back<MI, NJ>(a, acc, m0 + wm * WM, n0 + wn * WN, 0, reinterpret_cast<float*>(lds) + wave * 32 * (WN + 4), lane);
}

template <int BM, int BN, int WGM, int WGN, int NS, bool PAIRED>
hipError_t launch_mx4_tiles_as(const Mx4DotArgs& a, hipStream_t s) {
  constexpr int slabs = NS * (BM + BN) * 128 + (PAIRED ? (NS / 2 + 1) * 16 : NS * 8) * (BM + BN), staging = WGM * WGN * 32 * (BN / WGN + 4) * 4;
  constexpr int bytes = slabs > staging ? slabs : staging;
  static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
  const int64_t tm = ceil_div(a.M, BM), tn = ceil_div(a.N, BN);
  if (tm * tn > 0x0fffffff) return hipErrorInvalidValue;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(mx4_dot_tile_kernel<BM, BN, WGM, WGN, NS, PAIRED>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((mx4_dot_tile_kernel<BM, BN, WGM, WGN, NS, PAIRED>), dim3(unsigned(tm * tn)), dim3(WGM * WGN * 64), bytes, s, a, uint32_t(tm), uint32_t(tn));
  return hipGetLastError();
}
template <int BM, int BN, int WGM, int WGN, int NS>
hipError_t launch_mx4_tiles(const Mx4DotArgs& a, hipStream_t s) {
  if constexpr (NS % 2 == 0)
    if (mx4_scale_pitch(a.K) % 16 == 0) return launch_mx4_tiles_as<BM, BN, WGM, WGN, NS, true>(a, s);
  return launch_mx4_tiles_as<BM, BN, WGM, WGN, NS, false>(a, s);
}

}  // namespace gs
