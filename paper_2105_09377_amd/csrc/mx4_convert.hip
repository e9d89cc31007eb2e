// Conversion to and from microscaled 4-bit floats: whole matrices, and tokens of a paged cache.
//
// A scale is the power of two of its block's largest magnitude, over 4 (the largest power of two of e2m1),
// so a block is read once, reduced over its 32 numbers, and written: 16 bytes of numbers per lane where they lie in rows, four (bfloat16) or
// eight (floats) neighbouring lanes per block, the maximum over them by lane exchanges; 8 numbers per lane of a cache's tokens.
//
// Bound by memory: n numbers of s bytes move n (s + 17/32).  16384 x 8190 floats quantised 104 us (5.8 TB/s), read back 89 (6.9 TB/s, part of
// the codes still in the last-level cache); 16384 x 8192 bfloat16 62 and 49 us.  Matrices are read and written with the streaming hint
// (without it 109 and 107, aligned rows); 4 x 4001 tokens of 8 x 128 numbers into the cache 21.7 us (3.8 TB/s), back 16.0.
#include "mx4.h"

namespace gs {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_plain(const void* p, int64_t i, std::integral_constant<int, GS_BF16>) {
  return bf16_bits_to_float(static_cast<const uint16_t*>(p)[i]);
}
__device__ __forceinline__ float load_plain(const void* p, int64_t i, std::integral_constant<int, GS_F32>) {
  return static_cast<const float*>(p)[i];
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));

// N numbers (8 or 4) of a row from element `at` on, zero beyond `left` of them.
template <int DT, int N>
__device__ __forceinline__ void load_numbers(const void* row, int64_t at, int64_t left, float (&x)[N]) {
  if (left >= N) {
    if constexpr (DT == GS_BF16) {
      static_assert(N == 8, "16 bytes");
      const i32x4 v = __builtin_nontemporal_load(reinterpret_cast<const i32x4_any2*>(static_cast<const uint16_t*>(row) + at));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(uint32_t(v[i]) << 16);
        x[2 * i + 1] = __uint_as_float(uint32_t(v[i]) & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int h = 0; h < N / 4; ++h) {
        const f32x4_any v = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(static_cast<const float*>(row) + at + 4 * h));
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * h + i] = v[i];
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = i < left ? load_plain(row, at + i, std::integral_constant<int, DT>{}) : 0.0f;
}

template <int DT, int N>
__device__ __forceinline__ void store_numbers(void* row, int64_t at, int64_t left, uint32_t w, float scale) {
  if constexpr (DT == GS_BF16) {
    static_assert(N == 8, "16 bytes");
    uint16_t* dst = static_cast<uint16_t*>(row) + at;
    const i32x4 v = mx4_decode8(w, scale);
    if (left >= 8) {
      __builtin_nontemporal_store((i32x4_any2)v, reinterpret_cast<i32x4_any2*>(dst));
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) dst[i] = uint16_t(uint32_t(v[i / 2]) >> (16 * (i & 1)));
    }
  } else {
    float* dst = static_cast<float*>(row) + at;
    float x[N];
    mx4_decode2_f32<0>(w, scale, x);
    mx4_decode2_f32<1>(w, scale, x + 2);
    if constexpr (N == 8) {
      mx4_decode2_f32<2>(w, scale, x + 4);
      mx4_decode2_f32<3>(w, scale, x + 6);
    }
    if (left >= N) {
#pragma unroll
      for (int h = 0; h < N / 4; ++h) __builtin_nontemporal_store((f32x4_any{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]}), reinterpret_cast<f32x4_any*>(dst + 4 * h));
    } else {
#pragma unroll
      for (int i = 0; i < N - 1; ++i)
        if (i < left) dst[i] = x[i];
    }
  }
}

// The scale byte of the block that 32 / N neighbouring lanes have.
template <int N>
__device__ __forceinline__ uint32_t block_scale_byte(const float (&x)[N]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    top = top > b ? top : b;
  }
  top = max_of_4_lanes(top);
  if constexpr (N == 4) {
    const uint32_t o = __builtin_amdgcn_mov_dpp(top, 0x141, 0xF, 0xF, true);       // the eight lanes in reverse
    top = top > o ? top : o;
  }
  return mx4_scale_byte(top);
}

// Pieces of 16 bytes of all rows' numbers, one after the other: a workgroup takes 256 P of them, a lane P that lie 256 apart, whose loads are
// all under way before the first is used.  What pieces cost in instructions counts (16384 x 8190 floats read back with 64-bit places 118 us):
// rows and places are counted in 32 bits where all numbers do (BIG: in 64), the first of a lane's from a division by multiplication, the others
// from it.
template <int DT>
constexpr int kNumbers = DT == GS_BF16 ? 8 : 4;
template <bool BIG>
struct Pieces {
  using Index = std::conditional_t<BIG, int64_t, uint32_t>;
  Index per_row, total;
  FastDiv by_row;
  // of pieces at, at + 256 ..; those behind the last are the first
  template <int P>
  __device__ void places(Index at, Index (&row)[P], Index (&piece)[P]) const {
    divide(at < total ? at : 0, &row[0], &piece[0]);
    const bool wide = per_row >= kThreads;               // (uniform)
#pragma unroll
    for (int p = 1; p < P; ++p) {
      if (wide) {
        const Index next = piece[p - 1] + kThreads;
        const bool same = next < per_row;
        row[p] = same ? row[p - 1] : row[p - 1] + 1;
        piece[p] = same ? next : next - per_row;
      } else {
        divide(at + p * kThreads < total ? at + p * kThreads : 0, &row[p], &piece[p]);
      }
      if (at + p * kThreads >= total) row[p] = piece[p] = 0;
    }
  }
  __device__ void divide(Index at, Index* row, Index* piece) const {
    if constexpr (BIG) {
      *row = at / per_row;
      *piece = at - *row * per_row;
    } else {
      by_row.divmod(at, row, piece);
    }
  }
};

// A row's pieces are counted up to whole runs of scale bytes, the padding written as zeros by the same lanes.
template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) mx4_quantize_kernel(Mx4ConvertArgs a, Pieces<BIG> n) {
  using Index = typename Pieces<BIG>::Index;
  constexpr int N = kNumbers<DT>;
  const Index cols = Index(a.cols), blocks = Index(mx4_blocks(a.cols)), pitch = Index(mx4_scale_pitch(a.cols));
  const Index base = Index(blockIdx.x) * (kThreads * P) + threadIdx.x;
  Index row[P], piece[P];
  float x[P][N];
  n.places(base, row, piece);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Index at = piece[p] * N;
    load_numbers<DT, N>(a.plain, int64_t(row[p] * cols + at), at + N <= cols ? N : at < cols ? int(cols - at) : 0, x[p]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const uint32_t byte = block_scale_byte<N>(x[p]);
    if (base + p * kThreads >= n.total) continue;
    const Index block = piece[p] / (kMx4Block / N);
    if (block < blocks) {
      float eight[8] = {};
#pragma unroll
      for (int i = 0; i < N; ++i) eight[i] = x[p][i];
      const Index to = row[p] * blocks * (kMx4Block / N) + piece[p];
      if constexpr (N == 8) static_cast<uint32_t*>(a.values)[to] = mx4_encode8(eight, byte);
      else static_cast<uint16_t*>(a.values)[to] = uint16_t(mx4_encode8(eight, byte));
    }
    if (piece[p] % (kMx4Block / N) == 0) static_cast<uint8_t*>(a.scales)[row[p] * pitch + block] = uint8_t(block < blocks ? byte : 0);
  }
}

template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) mx4_dequantize_kernel(Mx4ConvertArgs a, Pieces<BIG> n) {
  using Index = typename Pieces<BIG>::Index;
  constexpr int N = kNumbers<DT>;
  const Index cols = Index(a.cols), blocks = Index(mx4_blocks(a.cols)), pitch = Index(mx4_scale_pitch(a.cols));
  const Index base = Index(blockIdx.x) * (kThreads * P) + threadIdx.x;
  Index row[P], piece[P];
  uint32_t w[P], byte[P];
  n.places(base, row, piece);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Index from = row[p] * blocks * (kMx4Block / N) + piece[p];
    if constexpr (N == 8) w[p] = static_cast<const uint32_t*>(a.values)[from];
    else w[p] = static_cast<const uint16_t*>(a.values)[from];
    byte[p] = static_cast<const uint8_t*>(a.scales)[row[p] * pitch + piece[p] / (kMx4Block / N)];
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (base + p * kThreads >= n.total) continue;
    const Index at = piece[p] * N;
    store_numbers<DT, N>(a.plain, int64_t(row[p] * cols + at), at + N <= cols ? N : int(cols - at), w[p], mx4_scale(byte[p]));
  }
}

// Back into rows that do not all begin on 16 bytes: pieces are those of the result's memory, so that whole lines are written.  A piece may have
// numbers of two blocks; one with numbers of two rows is written number by number.  There are cols >= N numbers in a row, n.per_row of them.
template <int DT, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) mx4_dequantize_flat_kernel(Mx4ConvertArgs a, Pieces<BIG> n) {
  using Index = typename Pieces<BIG>::Index;
  constexpr int N = kNumbers<DT>;
  typedef uint32_t u32_any __attribute__((aligned(1)));
  typedef uint64_t u64_any __attribute__((aligned(1)));
  using Codes = std::conditional_t<N == 8, uint64_t, uint32_t>;
  using CodesAny = std::conditional_t<N == 8, u64_any, u32_any>;
  const Index cols = n.per_row, blocks = Index(mx4_blocks(a.cols)), pitch = Index(mx4_scale_pitch(a.cols)), most = blocks * 16 - sizeof(Codes);
  const Index base = (Index(blockIdx.x) * (kThreads * P) + threadIdx.x) * N;
  const uint8_t *const values = static_cast<const uint8_t*>(a.values), *const scales = static_cast<const uint8_t*>(a.scales);
  Index row[P], first[P];             // of the piece's first number
  uint32_t w[P], byte[P][2];
  int border[P];                      // numbers from here on are of the second block
#pragma unroll
  for (int p = 0; p < P; ++p) {
    n.divide(base + p * (kThreads * N) < n.total ? base + p * (kThreads * N) : 0, &row[p], &first[p]);
    const Index at = first[p] / 2 < most ? first[p] / 2 : most, last = first[p] + N <= cols ? first[p] + N - 1 : cols - 1;
    const Codes c = *reinterpret_cast<const CodesAny*>(values + (row[p] * blocks * 16 + at));
    w[p] = uint32_t(c >> (int(first[p] - 2 * at) * 4));
    byte[p][0] = scales[row[p] * pitch + first[p] / kMx4Block];
    byte[p][1] = scales[row[p] * pitch + last / kMx4Block];
    border[p] = int(last / kMx4Block * kMx4Block) - int(first[p]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Index number = base + p * (kThreads * N);
    if (number >= n.total) continue;
    if (first[p] + N > cols) {
#pragma unroll 1
      for (int i = 0; i < N && number + i < n.total; ++i) {
        const bool wraps = first[p] + i >= cols;
        const Index r = wraps ? row[p] + 1 : row[p], c = wraps ? first[p] + i - cols : first[p] + i;
        float pair[2];
        mx4_decode2_f32<0>(values[r * blocks * 16 + c / 2], mx4_scale(scales[r * pitch + c / kMx4Block]), pair);
        const float v = c % 2 ? pair[1] : pair[0];
        if constexpr (DT == GS_BF16) static_cast<uint16_t*>(a.plain)[number + i] = float_to_bf16_bits(v);
        else static_cast<float*>(a.plain)[number + i] = v;
      }
      continue;
    }
    const float s0 = mx4_scale(byte[p][0]), s1 = mx4_scale(byte[p][1]);
    if constexpr (DT == GS_BF16) {
      const i32x4 x0 = mx4_decode8(w[p], s0), x1 = mx4_decode8(w[p], s1);
      i32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t low = uint32_t(2 * i < border[p] ? x0[i] : x1[i]) & 0xffffu, high = uint32_t(2 * i + 1 < border[p] ? x0[i] : x1[i]) & 0xffff0000u;
        x[i] = int32_t(low | high);
      }
      __builtin_nontemporal_store(x, reinterpret_cast<i32x4*>(static_cast<uint16_t*>(a.plain) + number));
    } else {
      float x0[4], x1[4];
      mx4_decode2_f32<0>(w[p], s0, x0);
      mx4_decode2_f32<1>(w[p], s0, x0 + 2);
      mx4_decode2_f32<0>(w[p], s1, x1);
      mx4_decode2_f32<1>(w[p], s1, x1 + 2);
      f32x4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = i < border[p] ? x0[i] : x1[i];
      __builtin_nontemporal_store(x, reinterpret_cast<f32x4*>(static_cast<float*>(a.plain) + number));
    }
  }
}

enum Convert { kQuantize, kDequantize, kDequantizeFlat };
template <int DT, int P, bool BIG>
hipError_t launch_convert(const Mx4ConvertArgs& a, int64_t per_row, Convert what, hipStream_t s) {
  // (the flat kernel counts numbers, the others pieces)
  const bool flat = what == kDequantizeFlat;
  const int64_t total = flat ? a.rows * a.cols : a.rows * per_row, step = flat ? a.cols : per_row;
  const int64_t groups = ceil_div(total, kThreads * P * (flat ? kNumbers<DT> : 1));
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  using Index = typename Pieces<BIG>::Index;
  const Pieces<BIG> n{Index(step), Index(total), FastDiv::make(BIG ? 1u : uint32_t(step))};
  const dim3 grid{unsigned(groups)}, block(kThreads);
  if (what == kQuantize) hipLaunchKernelGGL((mx4_quantize_kernel<DT, P, BIG>), grid, block, 0, s, a, n);
  else if (what == kDequantize) hipLaunchKernelGGL((mx4_dequantize_kernel<DT, P, BIG>), grid, block, 0, s, a, n);
  else hipLaunchKernelGGL((mx4_dequantize_flat_kernel<DT, P, BIG>), grid, block, 0, s, a, n);
  return hipGetLastError();
}
// Four pieces per lane where that still leaves eight workgroups for every compute unit.
template <int DT>
hipError_t convert(const Mx4ConvertArgs& a, int64_t per_row, Convert what, hipStream_t s) {
  const int64_t total = a.rows * per_row;
  if (total == 0) return hipSuccess;
  if (total > (int64_t(1) << 30) / kNumbers<DT>) return launch_convert<DT, 4, true>(a, per_row, what, s);
  if (total >= int64_t(256) * 8 * 4 * kThreads) return launch_convert<DT, 4, false>(a, per_row, what, s);
  return launch_convert<DT, 1, false>(a, per_row, what, s);
}
// Rows of 16384 x 8190 floats, which begin on 8 bytes: 89 us, and 120 with pieces that begin where the rows do.
template <int DT>
hipError_t dequantize(const Mx4ConvertArgs& a, hipStream_t s) {
  constexpr int N = kNumbers<DT>;
  return convert<DT>(a, ceil_div(a.cols, N), a.cols % N == 0 || a.rows <= 1 || a.cols < 128 ? kDequantize : kDequantizeFlat, s);
}

// Tokens of a cache.  A token's place takes two loads, one behind the other (its sequence's first position, an entry of the table), so a lane has
// several tokens, whose loads are under way together.  Keys: lanes run over (batch, token, head, piece of 8 numbers), P of them each.
// Values: over (batch, four places, head, piece), whose codes are 16 bytes of the cache and whose scales are 4.
struct TokenDivs {
  FastDiv pieces, heads, steps;      // steps: tokens of a sequence, or fours of places
};
template <bool BIG>
__device__ __forceinline__ void split_item(int64_t at, const TokenDivs& by, int64_t pieces, int64_t heads, int64_t steps, uint32_t* piece, int* head, int64_t* b,
                                           int64_t* step) {
  if constexpr (BIG) {
    const int64_t r = at / pieces, s = r / heads;
    *piece = uint32_t(at - r * pieces);
    *head = int(r - s * heads);
    *b = s / steps;
    *step = s - *b * steps;
  } else {
    uint32_t r, s, of, seq, in;
    by.pieces.divmod(uint32_t(at), &r, piece);
    by.heads.divmod(r, &s, &of);
    by.steps.divmod(s, &seq, &in);
    *head = int(of);
    *b = seq;
    *step = in;
  }
}

template <int DT, bool WRITE, int P, bool BIG>
__device__ __forceinline__ void key_tokens(const Mx4TokenArgs& a, int64_t total, const TokenDivs& by) {
  const int64_t base = int64_t(blockIdx.x) * (kThreads * P) + threadIdx.x;
  float x[P][8];
  uint32_t piece[P];
  int head[P];
  int64_t b[P], pos[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const bool there = base + p * kThreads < total;
    const int64_t at = there ? base + p * kThreads : 0;
    int64_t t;
    split_item<BIG>(at, by, a.cache.dim / 8, a.cache.heads, a.tokens, &piece[p], &head[p], &b[p], &t);
    if constexpr (WRITE) load_numbers<DT, 8>(a.k, at * 8, 8, x[p]);
    // below 0: no place
    pos[p] = there && !(WRITE && a.counts && t >= a.counts[b[p]]) ? int64_t(a.first[b[p]]) + t : -1;
  }
  int32_t id[P];
  uint32_t slot[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    id[p] = -1;
    slot[p] = 0;
    if (pos[p] >= 0 && pos[p] < a.width * a.cache.page) {
      uint32_t entry;
      a.cache.by_page.divmod(uint32_t(pos[p]), &entry, &slot[p]);
      id[p] = a.table[b[p] * a.width + entry];
    }
  }
  uint32_t w[P], byte[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const bool placed = id[p] >= 0 && id[p] < a.cache.n_pages;
    uint8_t* const block = a.cache.block(placed ? id[p] : 0, head[p]);
    const uint32_t codes = a.cache.key(slot[p]) + piece[p] * 4, scale = a.cache.key_scale(slot[p], piece[p] / 4);
    if constexpr (WRITE) {
      byte[p] = block_scale_byte<8>(x[p]);
      if (!placed) continue;
      *reinterpret_cast<uint32_t*>(block + codes) = mx4_encode8(x[p], byte[p]);
      if (piece[p] % 4 == 0) block[scale] = uint8_t(byte[p]);
    } else {
      w[p] = 0;
      byte[p] = 127;
      if (!placed) continue;
      w[p] = *reinterpret_cast<const uint32_t*>(block + codes);
      byte[p] = block[scale];
    }
  }
  if constexpr (!WRITE) {
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (base + p * kThreads < total) store_numbers<DT, 8>(a.k, (base + p * kThreads) * 8, 8, w[p], mx4_scale(byte[p]));
  }
}

template <int DT, bool WRITE, bool BIG>
__device__ __forceinline__ void value_tokens(const Mx4TokenArgs& a, int64_t fours, const TokenDivs& by) {
  const int64_t at = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (at >= a.batch * fours * a.cache.heads * (a.cache.dim / 8)) return;      // (whole blocks)
  uint32_t piece;
  int head;
  int64_t b, four;
  split_item<BIG>(at, by, a.cache.dim / 8, a.cache.heads, fours, &piece, &head, &b, &four);
  const int64_t first = a.first[b], pos = first - (first & 3) + four * 4, t0 = pos - first;
  const int64_t number = ((b * a.tokens + t0) * a.cache.heads + head) * a.cache.dim + piece * 8, step = int64_t(a.cache.heads) * a.cache.dim;
  float x[4][8];
  if constexpr (WRITE) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool there = t0 + j >= 0 && t0 + j < a.tokens;
      load_numbers<DT, 8>(a.v, there ? number + j * step : 0, there ? 8 : 0, x[j]);
    }
  }
  int64_t count = a.tokens;
  if (WRITE && a.counts && a.counts[b] < count) count = a.counts[b];
  int32_t id = -1;
  uint32_t slot = 0;
  if (pos >= 0 && pos < a.width * a.cache.page) {        // (of all four: pages are multiples of 16)
    uint32_t entry;
    a.cache.by_page.divmod(uint32_t(pos), &entry, &slot);
    id = a.table[b * a.width + entry];
  }
  const bool placed = id >= 0 && id < a.cache.n_pages;
  uint8_t* const block = a.cache.block(placed ? id : 0, head);
  uint8_t *const codes = block + a.cache.value(slot, piece), *const scales = block + a.cache.value_scale(slot, piece / 4);
  if constexpr (WRITE) {
    uint32_t w[4], byte[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      byte[j] = block_scale_byte<8>(x[j]);
      w[j] = mx4_encode8(x[j], byte[j]);
    }
    if (!placed) return;
    if (t0 >= 0 && t0 + 4 <= count) {
      *reinterpret_cast<i32x4*>(codes) = i32x4{int32_t(w[0]), int32_t(w[1]), int32_t(w[2]), int32_t(w[3])};
      if (piece % 4 == 0) *reinterpret_cast<uint32_t*>(scales) = byte[0] | byte[1] << 8 | byte[2] << 16 | byte[3] << 24;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (t0 + j >= 0 && t0 + j < count) {
          reinterpret_cast<uint32_t*>(codes)[j] = w[j];
          if (piece % 4 == 0) scales[j] = uint8_t(byte[j]);
        }
    }
  } else {
    i32x4 w = {0, 0, 0, 0};
    uint32_t byte = 0x7f7f7f7fu;
    if (placed) {
      w = *reinterpret_cast<const i32x4*>(codes);
      byte = *reinterpret_cast<const uint32_t*>(scales);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (t0 + j >= 0 && t0 + j < a.tokens) store_numbers<DT, 8>(a.v, number + j * step, 8, uint32_t(w[j]), mx4_scale((byte >> (8 * j)) & 255u));
  }
}

template <int DT, bool WRITE, int P, bool BIG>
__global__ void __launch_bounds__(kThreads) mx4_tokens_kernel(Mx4TokenArgs a, int64_t keys, int64_t fours, TokenDivs by_tokens, TokenDivs by_fours) {
  if (blockIdx.y == 0) key_tokens<DT, WRITE, P, BIG>(a, keys, by_tokens);
  else value_tokens<DT, WRITE, BIG>(a, fours, by_fours);
}

template <int DT, bool WRITE, int P, bool BIG>
hipError_t launch_tokens_as(const Mx4TokenArgs& a, hipStream_t s) {
  const int64_t pieces = a.cache.dim / 8, keys = a.batch * a.tokens * a.cache.heads * pieces;
  const int64_t fours = ceil_div(a.tokens + 3, 4);       // of places, wherever the first token lies in one
  const int64_t key_groups = ceil_div(keys, kThreads * P), value_groups = ceil_div(a.batch * fours * a.cache.heads * pieces, kThreads);
  const int64_t groups = key_groups > value_groups ? key_groups : value_groups;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  const FastDiv by_pieces = FastDiv::make(uint32_t(pieces)), by_heads = FastDiv::make(uint32_t(a.cache.heads));
  const TokenDivs by_tokens{by_pieces, by_heads, FastDiv::make(BIG ? 1u : uint32_t(a.tokens))}, by_fours{by_pieces, by_heads, FastDiv::make(BIG ? 1u : uint32_t(fours))};
  hipLaunchKernelGGL((mx4_tokens_kernel<DT, WRITE, P, BIG>), dim3(unsigned(groups), 2), dim3(kThreads), 0, s, a, keys, fours, by_tokens, by_fours);
  return hipGetLastError();
}
// Four pieces of keys per lane where that still leaves four workgroups for every compute unit (4 x 4001 tokens of 8 x 128 numbers, keys and values with
// one per lane: 29.7 us, read back 20.8).
template <int DT, bool WRITE>
hipError_t launch_tokens_of(const Mx4TokenArgs& a, hipStream_t s) {
  const int64_t keys = a.batch * a.tokens * a.cache.heads * (a.cache.dim / 8);
  if (keys == 0) return hipSuccess;
  if (keys > 0x3fffffff) return launch_tokens_as<DT, WRITE, 4, true>(a, s);
  if (keys >= int64_t(256) * 4 * 4 * kThreads) return launch_tokens_as<DT, WRITE, 4, false>(a, s);
  return launch_tokens_as<DT, WRITE, 1, false>(a, s);
}
template <bool WRITE>
hipError_t launch_tokens(const Mx4TokenArgs& a, hipStream_t s) {
  return a.dtype == GS_BF16 ? launch_tokens_of<GS_BF16, WRITE>(a, s) : launch_tokens_of<GS_F32, WRITE>(a, s);
}

}  // namespace

hipError_t launch_mx4_quantize(const Mx4ConvertArgs& a, hipStream_t s) {
  const int64_t per_row = mx4_scale_pitch(a.cols) * kMx4Block;
  return a.dtype == GS_BF16 ? convert<GS_BF16>(a, per_row / 8, kQuantize, s) : convert<GS_F32>(a, per_row / 4, kQuantize, s);
}

hipError_t launch_mx4_dequantize(const Mx4ConvertArgs& a, hipStream_t s) {
  return a.dtype == GS_BF16 ? dequantize<GS_BF16>(a, s) : dequantize<GS_F32>(a, s);
}

hipError_t launch_mx4_append(const Mx4TokenArgs& a, hipStream_t s) { return launch_tokens<true>(a, s); }
hipError_t launch_mx4_read(const Mx4TokenArgs& a, hipStream_t s) { return launch_tokens<false>(a, s); }

}  // namespace gs
