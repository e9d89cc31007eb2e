// Contractions with microscaled 4-bit operands:  out[m][n] = sum_k x[m][k] w[n][k],  w in blocks of 32 e2m1 numbers
// with a scale, x likewise (the matrix unit takes both with their scales: 16x16x128) or bfloat16 (w is converted
// in registers, exactly, and multiplied as bfloat16: 16x16x32).
//
// The order in which K is summed is free as long as both operands have the same one.  A unit is 8 blocks (256 of K)
// of 16 rows: lane (r = lane % 16, g = lane / 16) holds blocks 2 g and 2 g + 1 of row r, 32 consecutive bytes, and the
// two scale bytes beside each other.
#include "mx4.h"

namespace gs {

namespace {

typedef int32_t i32x8v __attribute__((ext_vector_type(8)));
typedef int32_t i32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ f32x4 mfma_mx4(const i32x4& a, const i32x4& b, const f32x4& c, int sa, int sb, std::integral_constant<int, 0>) {
  const i32x8v x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, sa, 0, sb);
}
__device__ __forceinline__ f32x4 mfma_mx4(const i32x4& a, const i32x4& b, const f32x4& c, int sa, int sb, std::integral_constant<int, 1>) {
  const i32x8v x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 1, sa, 1, sb);
}

// ---------------------------------------------------------------------------------------------
// Few rows of x: NW waves share a tile of 16 MT rows of x and 16 NT rows of w, the units of K dealt to them, their
// partial tiles added at the end.  Everything is loaded where it is used: w is read once for each 16 MT rows of x.
// ---------------------------------------------------------------------------------------------
template <bool XBF, int MT, int NT, int NW>
__global__ void __launch_bounds__(NW * 64) mx4_dot_rows_kernel(Mx4DotArgs a, int64_t tiles_n) {
  __shared__ f32x4 part[NW][MT * NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int64_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const int64_t m0 = tm * 16 * MT, n0 = tn * 16 * NT;
  const int64_t nb = mx4_blocks(a.K), pitch = mx4_scale_pitch(a.K), units = pitch / 8;

  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0, 0, 0, 0};

  for (int64_t u = wave; u < units; u += NW) {
    i32x4 w[NT][2];
    uint32_t wsc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int64_t row = n0 + n * 16 + r;
      const bool ok = row < a.N;
      wsc[n] = ok ? *reinterpret_cast<const uint16_t*>(a.ws + row * pitch + u * 8 + 2 * g) : 0u;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int64_t blk = u * 8 + 2 * g + s;
        w[n][s] = ok && blk < nb ? static_cast<const i32x4*>(a.w)[row * nb + blk] : i32x4{0, 0, 0, 0};
      }
    }
    if constexpr (!XBF) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int64_t row = m0 + m * 16 + r;
        const bool ok = row < a.M;
        const uint32_t xsc = ok ? *reinterpret_cast<const uint16_t*>(a.xs + row * pitch + u * 8 + 2 * g) : 0u;
        i32x4 x[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int64_t blk = u * 8 + 2 * g + s;
          x[s] = ok && blk < nb ? static_cast<const i32x4*>(a.x)[row * nb + blk] : i32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          acc[m][n] = mfma_mx4(w[n][0], x[0], acc[m][n], int(wsc[n]), int(xsc), std::integral_constant<int, 0>{});
          acc[m][n] = mfma_mx4(w[n][1], x[1], acc[m][n], int(wsc[n]), int(xsc), std::integral_constant<int, 1>{});
        }
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int64_t k0 = (u * 8 + 2 * g + s) * 32;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          i32x4 wv[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n) wv[n] = mx4_decode8(uint32_t(w[n][s][c]), mx4_scale((wsc[n] >> (8 * s)) & 255u));
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const int64_t row = m0 + m * 16 + r, k = k0 + 8 * c;
            const uint16_t* src = static_cast<const uint16_t*>(a.x) + row * a.K + k;
            i32x4 x = {0, 0, 0, 0};
            if (row < a.M && k < a.K) {
              if (k + 8 <= a.K) {
                x = *reinterpret_cast<const i32x4_any2*>(src);
              } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                  if (k + e < a.K) x[e / 2] |= int32_t(uint32_t(src[e]) << (16 * (e & 1)));
              }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
              acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wv[n]), __builtin_bit_cast(bf16x8, x), acc[m][n], 0, 0, 0);
          }
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) part[wave][m * NT + n][lane] = acc[m][n];
  __syncthreads();
  for (int t = wave; t < MT * NT; t += NW) {
    f32x4 sum = part[0][t][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) sum += part[w][t][lane];
    const int64_t m = m0 + (t / NT) * 16 + r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t n = n0 + (t % NT) * 16 + 4 * g + e;
      if (m < a.M && n < a.N) store_result<float>(a.out, nullptr, a.out_dtype, m * a.N + n, sum[e], a.relu);
    }
  }
}

template <bool XBF, int MT, int NT, int NW>
hipError_t launch_rows(const Mx4DotArgs& a, hipStream_t s) {
  const int64_t tiles_m = ceil_div(a.M, 16 * MT), tiles_n = ceil_div(a.N, 16 * NT);
  if (tiles_m * tiles_n > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((mx4_dot_rows_kernel<XBF, MT, NT, NW>), dim3(unsigned(tiles_m * tiles_n)), dim3(NW * 64), 0, s, a, tiles_n);
  return hipGetLastError();
}

}  // namespace

size_t mx4_dot_workspace(bool, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx4_dot(const Mx4DotArgs& a, void*, hipStream_t s) {
  if (a.M == 0 || a.N == 0) return hipSuccess;
  return a.xs ? launch_rows<false, 4, 2, 4>(a, s) : launch_rows<true, 4, 2, 4>(a, s);
}

}  // namespace gs
