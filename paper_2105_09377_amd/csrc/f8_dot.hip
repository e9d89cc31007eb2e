// Contractions of scaled 8-bit floats:  out[m][n] = sum_b xs[m][b] ws[n][b] sum_{k in block b} x[m][k] w[n][k],  one matrix w for all rows, or
// one for every expert's.
//
// The matrix unit multiplies the 128 codes of a block (16x16x128: one instruction), into zeros; the block's sum, times the product of
// the two scales, is added to the result by vector instructions.  w is the operand whose rows become rows of a lane's results, x the one
// that becomes columns: a lane's results are all of one row of x, so that it needs one scale of x for each block.
#include "f8_tile.h"

namespace gs {

namespace {

// ---------------------------------------------------------------------------------------------
// Few rows: eight waves share a tile of 16 rows of x and 16 NT rows of w, the blocks of K dealt to them one by one, their partial
// tiles added at the end in the order of the waves.  Everything goes from memory to registers, the next block's loads in flight while
// one is multiplied.  Lane (r = lane % 16, g = lane / 16) has the 16-byte columns g and g + 4 of row r of a block, so that a load has
// 64 bytes of a row.
//
// Bound by w's reading: 1 x 8192 x 8192 from memory 13.9 us, 4.8 TB/s with the launch; 32 x 4 rows of 64 experts (2048 x 4096) 82 us, 5.6 TB/s.  Few
// registers, so many waves, are what carries it: four blocks at a time (16 bytes of scales, 158 registers) 16.2 and 144 us, three or four
// blocks under way 13.8 and 105.
// ---------------------------------------------------------------------------------------------
constexpr int kRowWaves = 8;
template <int NT, bool W1, bool GROUPED>
__global__ void __launch_bounds__(kRowWaves * 64, 2) f8_dot_rows_kernel(F8DotArgs a, uint32_t tiles_n) {
  constexpr int NW = kRowWaves, D = 2;
  static_assert(NT <= 8, "a tile's rows of w are in one block of 128");
  __shared__ f32x4 part[NW][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const uint32_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  F8Rows rows = {int64_t(tm) * 16, a.M, 0};
  if constexpr (GROUPED) {
    rows = f8_group_tile(a, tm, 16);
    if (rows.end <= rows.first) return;
  }
  const int64_t m0 = rows.first, n0 = int64_t(tn) * 16 * NT;
  const int64_t blocks = a.K / kF8Block;

  // a lane's rows; those behind the end are the last one, and their results are not stored
  const uint8_t* const w = a.w + rows.expert * a.N * a.K;
  const float* const ws = a.ws + rows.expert * (W1 ? a.N : (a.N + 127) / 128) * a.pitch;
  const uint8_t* wp[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t row = n0 + n * 16 + r < a.N ? n0 + n * 16 + r : a.N - 1;
    wp[n] = w + row * a.K + g * 16;
  }
  const float* wsp[W1 ? NT : 1][W1 ? 4 : 1];
  if constexpr (W1) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t row = n0 + n * 16 + 4 * g + e;
        wsp[n][e] = ws + (row < a.N ? row : a.N - 1) * a.pitch;
      }
  } else {
    wsp[0][0] = ws + n0 / 128 * a.pitch;
  }
  const int64_t m = m0 + r < rows.end ? m0 + r : rows.end - 1;
  const int64_t x_row = GROUPED ? f8_x_row(a, m) : m;
  const int64_t x_at = x_row < 0 ? 0 : x_row;
  const uint8_t* const xp = a.x + x_at * a.K + g * 16;
  const float* const xsp = a.xs + (a.x_rows == 1 ? x_at : x_at / 128) * a.pitch;

  f32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = f32x4{0, 0, 0, 0};
  struct Block {
    i32x4 w[NT][2], x[2];
    float xs, ws[W1 ? NT : 1][W1 ? 4 : 1];
  };
  auto load = [&](int64_t b, Block& t) __attribute__((always_inline)) {
    t.xs = xsp[b];
#pragma unroll
    for (int n = 0; n < (W1 ? NT : 1); ++n)
#pragma unroll
      for (int e = 0; e < (W1 ? 4 : 1); ++e) t.ws[n][e] = wsp[n][e][b];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      t.x[h] = *reinterpret_cast<const i32x4*>(xp + b * kF8Block + h * 64);
#pragma unroll
      for (int n = 0; n < NT; ++n) t.w[n][h] = *reinterpret_cast<const i32x4*>(wp[n] + b * kF8Block + h * 64);
    }
  };
  auto multiply = [&](const Block& t) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const f32x4 p = f8_mfma16(t.w[n], t.x);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[n][e] += t.xs * t.ws[W1 ? n : 0][W1 ? e : 0] * p[e];
    }
  };
  Block ring[D];
  static_for<D>([&](auto d_) {
    constexpr int d = decltype(d_)::value;
    if (wave + d * NW < blocks) load(wave + d * NW, ring[d]);
  });
  for (int64_t b = wave; b < blocks; b += D * NW) {
    static_for<D>([&](auto d_) {
      constexpr int d = decltype(d_)::value;
      if (b + d * NW < blocks) {
        multiply(ring[d]);
        if (b + (d + D) * NW < blocks) load(b + (d + D) * NW, ring[d]);
      }
    });
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) part[wave][n][lane] = acc[n];
  __syncthreads();
  for (int t = wave; t < NT; t += NW) {
    f32x4 sum = part[0][t][lane];
#pragma unroll
    for (int v = 1; v < NW; ++v) sum += part[v][t][lane];
    if (x_row < 0) sum = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t n = n0 + t * 16 + 4 * g + e;
      if (m0 + r < rows.end && n < a.N) store_result<float>(a.out, nullptr, a.out_dtype, (m0 + r) * a.N + n, sum[e], a.relu);
    }
  }
}

template <int NT, bool W1>
hipError_t launch_rows_as(const F8DotArgs& a, hipStream_t s) {
  const int64_t tiles_m = f8_most_tiles(a, 16), tiles_n = ceil_div(a.N, 16 * NT);
  if (tiles_m * tiles_n > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid(unsigned(tiles_m * tiles_n)), block(kRowWaves * 64);
  if (a.offsets) hipLaunchKernelGGL((f8_dot_rows_kernel<NT, W1, true>), grid, block, 0, s, a, uint32_t(tiles_n));
  else hipLaunchKernelGGL((f8_dot_rows_kernel<NT, W1, false>), grid, block, 0, s, a, uint32_t(tiles_n));
  return hipGetLastError();
}
template <int NT>
hipError_t launch_rows(const F8DotArgs& a, hipStream_t s) {
  return a.w_rows == 1 ? launch_rows_as<NT, true>(a, s) : launch_rows_as<NT, false>(a, s);
}

// Adds the SPLITS parts of a sum over K, in their order: four results per lane, whose parts are all under way together.
typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
template <int SPLITS>
__global__ void __launch_bounds__(256) f8_dot_join_kernel(const float* parts, F8DotArgs a, int64_t total) {
  const int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (at >= total) return;
  f32x4 part[SPLITS];
  if (at + 4 <= total) {
#pragma unroll
    for (int p = 0; p < SPLITS; ++p) part[p] = *reinterpret_cast<const f32x4_any4*>(parts + p * total + at);
  } else {
#pragma unroll
    for (int p = 0; p < SPLITS; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[p][e] = at + e < total ? parts[p * total + at + e] : 0.0f;
  }
  f32x4 sum = part[0];
#pragma unroll
  for (int p = 1; p < SPLITS; ++p) sum += part[p];
  if (a.relu)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = fmaxf(sum[e], 0.0f);
  if (at + 4 <= total) {
    if (a.out_dtype == GS_BF16)
      *reinterpret_cast<i32x2*>(static_cast<uint16_t*>(a.out) + at) = i32x2{int32_t(pack_bf16x2(sum[0], sum[1])), int32_t(pack_bf16x2(sum[2], sum[3]))};
    else *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = sum;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (at + e < total) store_result<float>(a.out, nullptr, a.out_dtype, at + e, sum[e], 0);
}

int64_t tiles(int64_t M, int64_t N, int bm, int bn) { return ceil_div(M, bm) * ceil_div(N, bn); }

// Tiles: what a launch of them takes to begin, a slab where a compute unit has one workgroup, and where several share it or follow each
// other on it, and what each of those that follow takes more (us).  All of them are bound by the transfers to LDS, 50 to 70 bytes per
// nanosecond and compute unit (80 where all slabs are in L2: the same kernels without products and fragments), until the largest tiles'
// products take as long: 8192 cubed 460 us before transfers were spread over columns (439), 386 without transfers behind the first slabs, 334 with nothing
// else.  (Lines requested into L2 by one workgroup of those that share them, two to eight slabs ahead: 472; six or eight slabs under way in place of four:
// 333 x 5000 x 4104 18.5 us, 18.0 with four in 64x128 tiles of four waves, 16.5 of eight.)
struct TileWay {
  F8DotWay way;
  int bm, bn;
  double begin, alone, several, next;
};
constexpr TileWay kTileWays[] = {{kF8Tile32x64, 32, 64, 1.5, 0.29, 0.205, 0.0},    {kF8Tile64x64, 64, 64, 1.5, 0.35, 0.27, 0.0},
                                 {kF8Tile64x128, 64, 128, 2.0, 0.47, 0.47, 0.0},   {kF8Tile128x128Few, 128, 128, 2.5, 0.64, 0.64, 2.0},
                                 {kF8Tile128x128, 128, 128, 2.5, 0.9, 0.57, 0.0},  {kF8Tile128x256, 128, 256, 3.0, 0.9, 1.03, 3.0},
                                 {kF8Tile256x256, 256, 256, 4.0, 1.35, 1.72, 4.0}};

}  // namespace

// Up to 16 rows, 8 of every expert that has some on average, w goes through registers (128 x 4 rows of 64 experts, 2048 x 4096, 106 us that way and 109 in
// 32x64 tiles; 256 x 4 154 and 108).  There two tiles of w to a workgroup, which then share x, where x has more than four rows and the chip
// stays full (16 x 8192 x 8192 17.1 us against 21.0 with one; 1 x 8192 x 8192 16.1 and 14.0).
// More rows: the tile, and how many workgroups share one's sum over K (eight slabs each on average, five at least), by the time that they should take: the slabs of the
// busiest compute unit and w read at 5.2 TB/s, the longer one and two fifths of the other; where sums are shared 3 us more for the second
// launch, and the parts written and read, 8 bytes each at 4.5 TB/s.  Times that it chooses between, measured: 64 x 8192 x 8192 24.7 in 64x64 tiles, 19.8 by twos, 39 in 128x128; 256 x 8192 x 8192 32.8 in
// 64x128, 39 in 64x64, 45 in 128x128; 512 x 8192 x 8192 46 in 128x128 with eight waves, 61 with four, 63 in 64x128; 1024 x 8192 x 8192 64 in 128x256, 68 in
// 128x128, 98 in 256x256; 2048 x 8192 x 8192 114 in 256x256, 126 in 128x256; 100 x 1000 x 8192 10.4 in 32x64 by fours, 16.4 alone; 4096 cubed 65 in
// 256x256, 71 in 128x256.  Experts: 512 rows of 64 (2048 x 4096) 109 in 32x64, 144 in
// 128x128; 8192 of them 153 in 128x256, 246 in 32x64; 16384 rows of 16 (4096 x 4096), drawn evenly, 319 in 256x256, 343 in 128x256.  What it chooses took a
// tenth longer than the best of these at most, with experts 22 %.
F8DotPlan plan_f8_dot(int64_t M, int64_t N, int64_t K, int64_t experts) {
  const int64_t matrices = experts < M ? experts : M;              // that have rows
  const double rows = experts ? double(M) / double(matrices > 0 ? matrices : 1) : double(M);
  F8DotPlan p = {rows > 4 && tiles(M, N, 16, 32) >= 256 ? kF8Rows2 : kF8Rows1, 1, 0};
  if (M == 0 || N == 0 || K == 0 || K > (int64_t(1) << 22) || rows <= (experts ? 8 : 16)) return p;
  const int32_t slabs = int32_t(K / kF8Block);
  const double read = 2.0 + double(experts ? matrices : 1) * double(N) * double(K) / 5.2e6, part = double(M) * double(N) * 8.0 / 4.5e6;
  double least = 1e30;
  for (const TileWay& w : kTileWays) {
    // (experts' rows fill their last tile by half)
    double down = experts ? double(matrices) * (rows / w.bm + 0.5 > 1.0 ? rows / w.bm + 0.5 : 1.0) : double(ceil_div(M, w.bm));
    const double count = down * double(ceil_div(N, w.bn));
    if (count > 1e7) continue;
    for (int32_t n = 1; n <= (experts ? 1 : 8) && (n == 1 || slabs / n >= 8); n *= 2) {
      const double on_one = double(int64_t(count * n + 255) / 256);
      const double each = n > 1 ? double(((slabs + 3) / 4 + n - 1) / n * 4) : double(slabs);
      double t = w.begin;
      if (on_one <= 1.0) t += each * (w.several > w.alone ? w.alone + (w.several - w.alone) * count * n / 256.0 : w.alone);
      else t += each * w.several * on_one + w.next * (on_one - 1.0);
      t = t > read ? t + 0.4 * read : read + 0.4 * t;
      if (n > 1) t += 3.0 + n * part;
      if (t < least) {
        least = t;
        p.way = w.way;
        p.splits = n;
      }
    }
  }
  p.part_bytes = p.splits > 1 ? size_t(p.splits) * size_t(M) * size_t(N) * 4 : 0;
  return p;
}

hipError_t launch_f8_dot(const F8DotArgs& given, const F8DotPlan& plan, void* workspace, hipStream_t s) {
  F8DotArgs a = given;
  if (a.M == 0 || a.N == 0) return hipSuccess;
  a.splits = plan.splits;
  F8DotArgs b = a;
  if (plan.splits > 1) {
    b.out = workspace;
    b.out_dtype = GS_F32;
    b.relu = 0;
  }
  // (rows of x that experts share are found by 32-bit offsets in tiles: beyond them w is read for every 16 rows, 4096 rows of 8 experts with 2048 x 8192
  // 786 us, 101 below)
  const bool far = a.offsets && a.K > 0 && a.x_count > int64_t(0xffffffffu) / a.K;
  hipError_t e = hipErrorInvalidValue;
  switch (far ? kF8Rows2 : plan.way) {
    case kF8Rows1: e = launch_rows<1>(b, s); break;
    case kF8Rows2: e = launch_rows<2>(b, s); break;
    case kF8Tile32x64: e = launch_f8_tiles<32, 64, 2, 2, 4>(b, s); break;
    case kF8Tile64x64: e = launch_f8_tiles<64, 64, 2, 2, 4>(b, s); break;
    case kF8Tile64x128: e = launch_f8_tiles<64, 128, 2, 4, 4>(b, s); break;
    case kF8Tile128x128Few: e = launch_f8_tiles<128, 128, 4, 2, 4>(b, s); break;
    case kF8Tile128x128: e = launch_f8_tiles<128, 128, 2, 2, 2>(b, s); break;
    case kF8Tile128x256: e = launch_f8_tiles<128, 256, 2, 4, 3>(b, s); break;
    case kF8Tile256x256: e = launch_f8_tiles<256, 256, 4, 2, 2, 4>(b, s); break;
  }
  if (e != hipSuccess || plan.splits == 1) return e;
  const int64_t total = a.M * a.N;
  if (ceil_div(total, 1024) > 0x7fffffff) return hipErrorInvalidValue;
  const auto join = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(ceil_div(total, 1024))), dim3(256), 0, s, static_cast<const float*>(workspace), a, total);
    return hipGetLastError();
  };
  return plan.splits == 2 ? join(f8_dot_join_kernel<2>) : plan.splits == 4 ? join(f8_dot_join_kernel<4>) : join(f8_dot_join_kernel<8>);
}

}  // namespace gs
