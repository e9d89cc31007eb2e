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
// Few rows: eight waves share a tile of 16 rows of x and 16 NT rows of w, the blocks of K dealt to them four at a time (16 bytes
// of a row's scales), their partial tiles added at the end in the order of the waves.  Everything goes from memory to registers.
// ---------------------------------------------------------------------------------------------
constexpr int kRowWaves = 8;
template <int NT, bool GROUPED>
__global__ void __launch_bounds__(kRowWaves * 64) f8_dot_rows_kernel(F8DotArgs a, uint32_t tiles_n) {
  constexpr int NW = kRowWaves, U = 4;
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
  const int64_t w_rows = (a.N + a.w_rows - 1) / a.w_rows;
  const uint8_t* const w = a.w + rows.expert * a.N * a.K;
  const float* const ws = a.ws + rows.expert * w_rows * a.pitch;
  const uint8_t* wp[NT];
  const float* wsp[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t row = n0 + n * 16 + r < a.N ? n0 + n * 16 + r : a.N - 1;
    wp[n] = w + row * a.K + g * 32;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t of = n0 + n * 16 + 4 * g + e < a.N ? n0 + n * 16 + 4 * g + e : a.N - 1;
      wsp[n][e] = ws + of / a.w_rows * a.pitch;
    }
  }
  const int64_t m = m0 + r < rows.end ? m0 + r : rows.end - 1;
  const int64_t x_row = GROUPED ? f8_x_row(a, m) : m;
  const int64_t x_at = x_row < 0 ? 0 : x_row;
  const uint8_t* const xp = a.x + x_at * a.K + g * 32;
  const float* const xsp = a.xs + x_at / a.x_rows * a.pitch;

  f32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = f32x4{0, 0, 0, 0};
  for (int64_t u = wave; u * U < blocks; u += NW) {
    const f32x4 xs = *reinterpret_cast<const f32x4*>(xsp + u * U);
#pragma unroll
    for (int b = 0; b < U; ++b) {
      if (u * U + b >= blocks) break;
      const int64_t at = (u * U + b) * kF8Block;
      i32x4 xv[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) xv[h] = *reinterpret_cast<const i32x4*>(xp + at + h * 16);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        i32x4 wv[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) wv[h] = *reinterpret_cast<const i32x4*>(wp[n] + at + h * 16);
        const f32x4 p = f8_mfma16(wv, xv);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] += xs[b] * wsp[n][e][u * U + b] * p[e];
      }
    }
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

// Tiles of `size` rows that experts' rows are cut into, at most.
int64_t most_tiles(const F8DotArgs& a, int64_t size) {
  return a.offsets ? a.M / size + (a.experts < a.M ? a.experts : a.M) : ceil_div(a.M, size);
}

template <int NT>
hipError_t launch_rows(const F8DotArgs& a, hipStream_t s) {
  const int64_t tiles_m = most_tiles(a, 16), tiles_n = ceil_div(a.N, 16 * NT);
  if (tiles_m * tiles_n > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid(unsigned(tiles_m * tiles_n)), block(kRowWaves * 64);
  if (a.offsets) hipLaunchKernelGGL((f8_dot_rows_kernel<NT, true>), grid, block, 0, s, a, uint32_t(tiles_n));
  else hipLaunchKernelGGL((f8_dot_rows_kernel<NT, false>), grid, block, 0, s, a, uint32_t(tiles_n));
  return hipGetLastError();
}

enum F8DotWay { kF8Rows, kF8Tile256x256, kF8Tile128x128, kF8Tile64x64 };

int64_t tiles(int64_t M, int64_t N, int bm, int bn) { return ceil_div(M, bm) * ceil_div(N, bn); }

}  // namespace

F8DotPlan plan_f8_dot(int64_t M, int64_t N, int64_t K, int64_t experts) {
  F8DotPlan p = {kF8Rows, 1, 0};
  if (K == 0 || K > (int64_t(1) << 22)) return p;
  const int64_t rows = experts ? ceil_div(M, experts) : M;     // of a matrix
  if (rows <= 16) return p;
  if (tiles(M, N, 256, 256) >= 180) p.way = kF8Tile256x256;
  else if (tiles(M, N, 128, 128) >= 192) p.way = kF8Tile128x128;
  else p.way = kF8Tile64x64;
  return p;
}

hipError_t launch_f8_dot(const F8DotArgs& given, const F8DotPlan& plan, void*, hipStream_t s) {
  F8DotArgs a = given;
  if (a.M == 0 || a.N == 0) return hipSuccess;
  a.splits = 1;
  // (rows of x that experts share are found by 32-bit offsets in tiles)
  const bool far = a.offsets && a.K > 0 && a.x_count > int64_t(0xffffffffu) / a.K;
  switch (far ? kF8Rows : plan.way) {
    case kF8Tile256x256: return launch_f8_tiles<256, 256, 4, 2, 2>(a, most_tiles(a, 256), s);
    case kF8Tile128x128: return launch_f8_tiles<128, 128, 2, 2, 2>(a, most_tiles(a, 128), s);
    case kF8Tile64x64: return launch_f8_tiles<64, 64, 2, 2, 4>(a, most_tiles(a, 64), s);
    default: return launch_rows<2>(a, s);
  }
}

}  // namespace gs
