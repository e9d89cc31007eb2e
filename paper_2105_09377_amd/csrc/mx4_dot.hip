// Contractions with microscaled 4-bit operands:  out[m][n] = sum_k x[m][k] w[n][k],  w in blocks of 32 e2m1 numbers
// with a scale, x likewise (the matrix unit takes both with their scales: 16x16x128) or bfloat16 (w is converted
// in registers, exactly, and multiplied as bfloat16: 16x16x32).
//
// The order in which K is summed is free as long as both operands have the same one.  A unit is 8 blocks (256 of K)
// of 16 rows: lane (r = lane % 16, g = lane / 16) holds blocks 2 g and 2 g + 1 of row r, 32 consecutive bytes, and the
// two scale bytes beside each other.
#include "mx4_weight_tile.h"

namespace gs {

namespace {

__device__ __forceinline__ f32x4 mfma_mx4(const i32x4& a, const i32x4& b, const f32x4& c, int sa, int sb, std::integral_constant<int, 0>) {
  const i32x8t x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, sa, 0, sb);
}
__device__ __forceinline__ f32x4 mfma_mx4(const i32x4& a, const i32x4& b, const f32x4& c, int sa, int sb, std::integral_constant<int, 1>) {
  const i32x8t x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 1, sa, 1, sb);
}

typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));

// ---------------------------------------------------------------------------------------------
// Few rows of x: eight waves share a tile of 16 rows of x and 16 NT rows of w, the units of K dealt to them, their
// partial tiles added at the end in the order of the waves.  Everything goes from memory to registers, the next unit's
// loads in flight while one is multiplied: w is read once, and bound by that: one row with 8192 x 8192 weights 12.5 us,
// 2.9 TB/s from a standing start, 10.7 with weights that lie in the last-level cache (four units in flight 12.8, and
// lanes without a row of x switched off 11.8, where this took 11.9).
// ---------------------------------------------------------------------------------------------
constexpr int kRowWaves = 8;
template <bool XBF, int NT>
__global__ void __launch_bounds__(kRowWaves * 64) mx4_dot_rows_kernel(Mx4DotArgs a, uint32_t tiles_n) {
  constexpr int NW = kRowWaves;
  __shared__ f32x4 part[NW][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const uint32_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const int64_t m0 = int64_t(tm) * 16, n0 = int64_t(tn) * 16 * NT;
  const int64_t nb = mx4_blocks(a.K), pitch = mx4_scale_pitch(a.K);
  const int32_t units = int32_t(pitch / 8);

  // a lane's rows; those behind the end are the last one, and their results are not stored
  const uint8_t *wp[NT], *wsp[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t row = n0 + n * 16 + r < a.N ? n0 + n * 16 + r : a.N - 1;
    wp[n] = static_cast<const uint8_t*>(a.w) + row * nb * 16 + g * 32;
    wsp[n] = a.ws + row * pitch + g * 2;
  }
  const int64_t x_row = m0 + r < a.M ? m0 + r : a.M - 1;
  const uint8_t* const xp = static_cast<const uint8_t*>(a.x) + (XBF ? (x_row * a.K + g * 64) * 2 : x_row * nb * 16 + g * 32);
  const uint8_t* const xsp = XBF ? nullptr : a.xs + x_row * pitch + g * 2;

  f32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = f32x4{0, 0, 0, 0};

  constexpr int XP = XBF ? 8 : 2;          // 16-byte pieces of a lane's two blocks of x
  struct Unit {
    i32x4 w[NT][2], x[XP];
    uint32_t ws[NT], xs;
  };
  auto load = [&](int32_t u, Unit& t) {
    // blocks behind K are read as zeros
    const int64_t at = int64_t(u) * 8;
    const bool whole = at + 8 <= nb;       // (uniform)
    const int32_t left = int32_t(nb - at) - 2 * g;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      t.ws[n] = *reinterpret_cast<const uint16_t*>(wsp[n] + at);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        t.w[n][s] = i32x4{0, 0, 0, 0};
        if (whole || s < left) t.w[n][s] = *reinterpret_cast<const i32x4*>(wp[n] + at * 16 + s * 16);
      }
    }
    if constexpr (!XBF) {
      t.xs = *reinterpret_cast<const uint16_t*>(xsp + at);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        t.x[s] = i32x4{0, 0, 0, 0};
        if (whole || s < left) t.x[s] = *reinterpret_cast<const i32x4*>(xp + at * 16 + s * 16);
      }
    } else if (at * 32 + 256 <= a.K) {                    // (uniform)
#pragma unroll
      for (int c = 0; c < 8; ++c) t.x[c] = *reinterpret_cast<const i32x4_any2t*>(xp + at * 64 + c * 16);
    } else {
      const int64_t numbers = a.K - at * 32 - g * 64;     // of the lane's part of this row
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        t.x[c] = i32x4{0, 0, 0, 0};
        const uint16_t* src = reinterpret_cast<const uint16_t*>(xp + at * 64) + c * 8;
        if (c * 8 + 8 <= numbers) {
          t.x[c] = *reinterpret_cast<const i32x4_any2t*>(src);
        } else {
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (c * 8 + e < numbers) t.x[c][e / 2] |= int32_t(uint32_t(src[e]) << (16 * (e & 1)));
        }
      }
    }
  };
  auto multiply = [&](const Unit& t) {
    if constexpr (!XBF) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        acc[n] = mfma_mx4(t.w[n][0], t.x[0], acc[n], int(t.ws[n]), int(t.xs), std::integral_constant<int, 0>{});
        acc[n] = mfma_mx4(t.w[n][1], t.x[1], acc[n], int(t.ws[n]), int(t.xs), std::integral_constant<int, 1>{});
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float sc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) sc[n] = mx4_scale((t.ws[n] >> (8 * s)) & 255u);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const bf16x8 wv = __builtin_bit_cast(bf16x8, mx4_decode8(uint32_t(t.w[n][s][c]), sc[n]));
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, __builtin_bit_cast(bf16x8, t.x[4 * s + c]), acc[n], 0, 0, 0);
          }
      }
    }
  };
  if (wave < units) {
    Unit cur, next;
    load(wave, cur);
    int32_t u = wave;
    for (; u + NW < units; u += NW) {
      load(u + NW, next);
      multiply(cur);
      cur = next;
    }
    multiply(cur);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) part[wave][n][lane] = acc[n];
  __syncthreads();
  for (int t = wave; t < NT; t += NW) {
    f32x4 sum = part[0][t][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) sum += part[w][t][lane];
    const int64_t m = m0 + r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t n = n0 + t * 16 + 4 * g + e;
      if (m < a.M && n < a.N) store_result<float>(a.out, nullptr, a.out_dtype, m * a.N + n, sum[e], a.relu);
    }
  }
}

template <bool XBF, int NT>
hipError_t launch_rows(const Mx4DotArgs& a, hipStream_t s) {
  const int64_t tiles_m = ceil_div(a.M, 16), tiles_n = ceil_div(a.N, 16 * NT);
  if (tiles_m * tiles_n > 0x7fffffff || a.K >= (int64_t(1) << 38)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((mx4_dot_rows_kernel<XBF, NT>), dim3(unsigned(tiles_m * tiles_n)), dim3(kRowWaves * 64), 0, s, a, uint32_t(tiles_n));
  return hipGetLastError();
}

// Adds the parts of a sum over K, in their order: four results per lane.
__global__ void __launch_bounds__(256) mx4_dot_join_kernel(const float* parts, Mx4DotArgs a, int64_t total) {
  const int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= total) return;
  if (at + 4 <= total) {
    f32x4 sum = *reinterpret_cast<const f32x4_any4*>(parts + at);
    for (int p = 1; p < a.splits; ++p) sum += *reinterpret_cast<const f32x4_any4*>(parts + p * total + at);
    if (a.relu)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaxf(sum[e], 0.0f);
    if (a.out_dtype == GS_BF16)
      *reinterpret_cast<i32x2*>(static_cast<uint16_t*>(a.out) + at) = i32x2{int32_t(pack_bf16x2(sum[0], sum[1])), int32_t(pack_bf16x2(sum[2], sum[3]))};
    else *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = sum;
    return;
  }
  for (int64_t i = at; i < total; ++i) {
    float sum = parts[i];
    for (int p = 1; p < a.splits; ++p) sum += parts[p * total + i];
    store_result<float>(a.out, nullptr, a.out_dtype, i, sum, a.relu);
  }
}

// Rows of x, K numbers each, at rows of ldx numbers, zeros behind: what transfers of 16 bytes want.
__global__ void __launch_bounds__(256) mx4_pad_rows_kernel(const uint16_t* x, uint16_t* out, int64_t rows, int64_t K, int64_t ldx) {
  const int64_t pieces = ldx / 8, total = rows * pieces;
  for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < total; at += int64_t(gridDim.x) * 256) {
    const int64_t row = at / pieces, k = (at - row * pieces) * 8;
    const uint16_t* src = x + row * K + k;
    i32x4 v = {0, 0, 0, 0};
    if (k + 8 <= K) {
      v = *reinterpret_cast<const i32x4_any2t*>(src);
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (k + e < K) v[e / 2] |= int32_t(uint32_t(src[e]) << (16 * (e & 1)));
    }
    *reinterpret_cast<i32x4*>(out + row * ldx + k) = v;
  }
}

// How a product is done (times in us).
int64_t tiles(int64_t M, int64_t N, int bm, int bn) { return ceil_div(M, bm) * ceil_div(N, bn); }

// Tiles of bfloat16 rows with MX4 weights: what a slab of 128 of K takes a workgroup that has a compute unit for itself, and each of several
// that share one or follow each other on it (us).
struct WeightWay {
  Mx4DotWay way;
  int bm, bn;
  double alone, several;
};
constexpr WeightWay kWeightWays[] = {{kWeight32x128, 32, 128, 0.46, 0.43}, {kWeight64x64, 64, 64, 0.47, 0.43}, {kWeight64x128, 64, 128, 0.88, 0.58},
                                     {kWeight128x128, 128, 128, 1.15, 1.15}, {kWeight128x256, 128, 256, 1.72, 1.75}};
struct WeightChoice {
  Mx4DotWay way;
  int splits;
};
// The tile, and how many workgroups share one's sum over K (eight slabs each at least), by the time that they should
// take: the slabs of the busiest compute unit, or what all tiles read at 10 TB/s (200 x 4096 x 11000 in 256 64x64 tiles:
// 456 MB, 51 us), and where sums are shared 3 us for the second launch and the parts written and read, 8 bytes each at 4
// TB/s.  Times that it chooses between, measured: 100 x 8192 x 8192 34.6 in 64x64 tiles, 29.6 in 64x128 by fours, 29.4 in
// 128x128 by fours; 200 x 8192 x 8192 53.4 in 64x128, 47.4 by twos, 44.2 in 128x256 by fours; 100 x 5000 x 4104 16.9 in
// 64x64, 20.2 by twos; 256 x 5000 x 4104 28.6 in 64x128, 25.2 by threes; 300 x 11000 x 4096 62.9 in 128x128 by twos, 53.5
// in 64x64, 37.5 in 64x128; 20 x 16384 x 1024 7.0 in 32x128, 9.3 by twos; 17 x 8192 x 8192 in 32x128 25.8, 17.7, 13.7 and
// 15.3 alone, by twos, fours and eights; 2048 x 4096 x 4096 62.8 in 128x256, 73.9 in 128x128.
WeightChoice weight_choice(int64_t M, int64_t N, int64_t K) {
  const int32_t slabs = int32_t(ceil_div(K, 128));                 // (K is at most 2^22)
  WeightChoice best = {kWeight64x64, 1};
  double least = 1e30;
  for (const WeightWay& w : kWeightWays) {
    const int64_t count = tiles(M, N, w.bm, w.bn);
    const double read = double(count) * slabs * (w.bm * 256 + w.bn * 68) / 1e7, part = double(M) * double(N) * 8.0 / 4e6;
    // (more than four workgroups for each compute unit are no help)
    for (int32_t n = 1; n <= 16 && (n == 1 || (slabs / n >= 8 && count * n <= 1024)); ++n) {
      const int64_t on_one = (count * n + 255) / 256;
      double t = double((slabs + n - 1) / n) * (on_one == 1 ? w.alone : w.several * double(on_one));
      t = t > read ? t : read;
      if (n > 1) t += 3.0 + 0.2 * n + n * part;
      if (t < least) {
        least = t;
        best = {w.way, n};
      }
    }
  }
  return best;
}

}  // namespace

Mx4DotPlan plan_mx4_dot(bool xbf, int64_t M, int64_t N, int64_t K) {
  Mx4DotPlan p = {kRows1, 1, 0, false, 0, 0};
  // Up to 16 rows w is read once by the rows kernel.  Two blocks of 16 columns per wave where that leaves a workgroup for every
  // compute unit (1 x 8192 x 8192 bf16 10.0 against 11.7 with one; 1 x 4096 x 4096 6.1 against 4.7).  More rows, few tiles: the
  // waves of a workgroup share K, which a tile walks alone (MX4 100 x 700 x 5000 5.3 against 7.4 in 64x64 tiles, 40 x 300 x 16000
  // 8.9 / 16.4, 200 x 2000 x 1528 8.2 / 4.2).  bfloat16 rows stand in L2's way where K is long (100 x 700 x 5000 9.2 against 10.1 in
  // shared tiles, 40 x 300 x 16000 20.3 / 13.1).
  const int64_t t16x32 = tiles(M, N, 16, 32);
  p.way = M <= 16 ? (t16x32 >= 256 ? kRows2 : kRows1) : tiles(M, N, 16, 16) > 128 ? kRows2 : kRows1;
  if (M <= 16 || (t16x32 <= 256 && (!xbf || K <= 6144)) || K == 0 || K > (int64_t(1) << 22)) return p;
  const int64_t t64 = tiles(M, N, 64, 64), t128 = tiles(M, N, 128, 128);
  if (!xbf) {
    // 4096 cubed (256 tiles of 256x256) 39 in those, 47 in 128x128 and 71 in 64x64 tiles; 2048 cubed (64 of them, 256 of 128x128)
    // 17, 9.7 and 11.3; 1021 x 2000 x 1531 (128 of 128x128) 7.1 and 6.0.  Tiles that a compute unit has for itself are paid for
    // in latency: more slabs under way (64 x 8192 x 8192 11.3 with four, 18.4 with two), or, where those are few, more waves (2048
    // cubed 9.7 with eight waves, 10.5 with four; 512 x 8192 x 8192 27.8 and 26.3).  More 128x128 tiles than the chip has at a time, two
    // to a compute unit, are slower than fewer large ones (3000 cubed, 576 of them and 144 of 256x256, 32.4 and 25.6).
    if (tiles(M, N, 256, 256) >= 180 || t128 > 512) p.way = kTile256x256;
    else if (t128 > 256) p.way = kTile128x128;
    else if (t128 >= 192) p.way = K > 16 * 256 ? kTile128x128Long : kTile128x128Few;
    else p.way = t64 <= 256 ? kTile64x64Few : kTile64x64;
    return p;
  }
  p.pad = K % 8 != 0;
  p.ldx = round_up(K, 8);
  if (p.pad) p.pad_bytes = size_t(round_up(M * p.ldx * 2, 256));
  const WeightChoice c = weight_choice(M, N, K);
  p.way = c.way;
  if (c.splits > 1) {
    p.splits = c.splits;
    p.part_bytes = size_t(c.splits) * size_t(M) * size_t(N) * 4;
  }
  return p;
}

hipError_t launch_mx4_dot(const Mx4DotArgs& given, const Mx4DotPlan& p, void* workspace, hipStream_t s) {
  Mx4DotArgs a = given;
  if (a.M == 0 || a.N == 0) return hipSuccess;
  if (p.pad) {
    const int64_t pieces = a.M * (p.ldx / 8), groups = ceil_div(pieces, 256);
    hipLaunchKernelGGL(mx4_pad_rows_kernel, dim3(unsigned(groups < 4096 ? groups : 4096)), dim3(256), 0, s, static_cast<const uint16_t*>(a.x),
                       static_cast<uint16_t*>(workspace), a.M, a.K, p.ldx);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.x = workspace;
  }
  void* const parts = static_cast<uint8_t*>(workspace) + p.pad_bytes;
  Mx4DotArgs b = a;
  b.splits = p.splits;
  if (p.splits > 1) {
    b.out = parts;
    b.out_dtype = GS_F32;
    b.relu = 0;
  }
  hipError_t e = hipErrorInvalidValue;
  switch (p.way) {
    case kRows1: e = a.xs ? launch_rows<false, 1>(a, s) : launch_rows<true, 1>(a, s); break;
    case kRows2: e = a.xs ? launch_rows<false, 2>(a, s) : launch_rows<true, 2>(a, s); break;
    case kTile64x64Few: e = launch_mx4_tiles<64, 64, 2, 2, 4>(a, s); break;
    case kTile64x64: e = launch_mx4_tiles<64, 64, 2, 2, 2>(a, s); break;
    case kTile128x128Few: e = launch_mx4_tiles<128, 128, 2, 4, 4>(a, s); break;
    case kTile128x128Long: e = launch_mx4_tiles<128, 128, 2, 2, 4>(a, s); break;
    case kTile128x128: e = launch_mx4_tiles<128, 128, 2, 2, 2>(a, s); break;
    case kTile256x256: e = launch_mx4_tiles<256, 256, 2, 4, 2>(a, s); break;
    case kWeight32x128: e = launch_mx4_weight_tiles<32, 128, 1, 4, 3>(b, p.ldx, s); break;
    case kWeight64x64: e = launch_mx4_weight_tiles<64, 64, 2, 2, 3>(b, p.ldx, s); break;
    case kWeight64x128: e = launch_mx4_weight_tiles<64, 128, 2, 2, 2>(b, p.ldx, s); break;
    case kWeight128x128: e = launch_mx4_weight_tiles<128, 128, 2, 4, 3>(b, p.ldx, s); break;
    case kWeight128x256: e = launch_mx4_weight_tiles<128, 256, 2, 4, 3>(b, p.ldx, s); break;
  }
  if (e != hipSuccess || p.splits == 1) return e;
  b = a;
  b.splits = p.splits;
  const int64_t total = a.M * a.N;
  hipLaunchKernelGGL(mx4_dot_join_kernel, dim3(unsigned(ceil_div(total, 1024))), dim3(256), 0, s, static_cast<const float*>(parts), b, total);
  return hipGetLastError();
}

}  // namespace gs
