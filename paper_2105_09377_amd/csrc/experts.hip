// Tokens dealt to experts: sorted by expert, spread out into rows, joined again with weights, and the gradient of the joining.
//
// Bound by memory where there are many tokens (rows are written and read once): 16384 tokens of 4096 bfloat16 numbers with 4 choices spread out in 106
// to 129 us and joined in 107, 5.2 to 6.3 TB/s, the gradient of the joining in 266, 4.5; by launches where there are few.  Nothing is added by
// atomics but counts, whose order does not show.
#include "f8.h"
#include "pieces.h"

namespace gs {

namespace {

// ---------------------------------------------------------------------------------------------
// Sorting: a stable sort by counting.  A workgroup has a run of the choices, each of its waves a part of that run.
// ---------------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024;
constexpr int kMaxExperts = 4096;
// 65536 choices of 128 experts 10.2 us (11.5 with 4096 choices to a workgroup, 17 with 512: all of them read all counts; 524288 of 512
// 34 in 128 workgroups, 53 in 256), 128 in one workgroup 3.5.
constexpr int kSortGroups = 128;     // at most
constexpr int kGroupKeys = 2048;     // at least, of a workgroup where there are several

// Adds v over the workgroup's threads up to and without this one; scratch: a number per wave.
__device__ __forceinline__ int32_t block_before(int32_t v, int32_t* scratch, int lane, int wave, int waves) {
  int32_t incl = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int32_t o = __shfl_up(incl, d);
    incl += lane >= d ? o : 0;
  }
  if (lane == 63) scratch[wave] = incl;
  __syncthreads();
  int32_t before = incl - v;
  for (int w = 0; w < waves; ++w) before += w < wave ? scratch[w] : 0;
  __syncthreads();
  return before;
}

__global__ void __launch_bounds__(kSortThreads) expert_count_kernel(ExpertSortArgs a, int32_t per_group) {
  __shared__ int32_t count[kMaxExperts];
  const int32_t ne = int32_t(a.n_experts);
  for (int e = threadIdx.x; e < ne; e += blockDim.x) count[e] = 0;
  __syncthreads();
  const int64_t lo = int64_t(blockIdx.x) * per_group, hi = lo + per_group < a.n ? lo + per_group : a.n;
  for (int64_t i = lo + threadIdx.x; i < hi; i += blockDim.x) {
    const int32_t e = a.experts[i];
    if (e >= 0 && e < ne) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < ne; e += blockDim.x) a.counts[int64_t(blockIdx.x) * ne + e] = count[e];
}

// ALONE: one workgroup has all choices.  bits: of the largest key, n_experts, which stands for choices that are dropped.
template <bool ALONE>
__global__ void __launch_bounds__(kSortThreads) expert_place_kernel(ExpertSortArgs a, int32_t per_group, int32_t per_wave, int bits, FastDiv by_choices,
                                                                     FastDiv by_experts) {
  extern __shared__ int32_t lds[];             // [waves][experts], then a number per wave and one, then two per expert
  const int32_t ne = int32_t(a.n_experts);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int32_t* const mine = lds + wave * ne;
  int32_t* const scratch = lds + waves * ne;
  int32_t* const totals = scratch + waves + 1;
  int32_t* const befores = totals + ne;        // of the workgroups in front of this one
  for (int i = threadIdx.x; i < waves * ne; i += blockDim.x) lds[i] = 0;
  if constexpr (!ALONE)
    for (int i = threadIdx.x; i < 2 * ne; i += blockDim.x) totals[i] = 0;
  __syncthreads();
  if constexpr (!ALONE) {
    // (whole workgroups' counts, a few of each thread's under way together)
    const int32_t all = int32_t(gridDim.x) * ne, mine_from = int32_t(blockIdx.x) * ne;
    for (int32_t i = threadIdx.x; i < all; i += blockDim.x) {
      const int32_t c = a.counts[i], e = i - int32_t(by_experts.div(uint32_t(i))) * ne;
      if (c == 0) continue;
      atomicAdd(&totals[e], c);
      if (i < mine_from) atomicAdd(&befores[e], c);
    }
  }
  const int64_t group_lo = int64_t(blockIdx.x) * per_group, group_hi = group_lo + per_group < a.n ? group_lo + per_group : a.n;
  const int64_t lo = group_lo + int64_t(wave) * per_wave, hi = lo + per_wave < group_hi ? lo + per_wave : group_hi;
  for (int64_t i = lo + lane; i < hi; i += 64) {
    const int32_t e = a.experts[i];
    if (e >= 0 && e < ne) atomicAdd(&mine[e], 1);
  }
  __syncthreads();
  // where every wave's rows of an expert begin
  int32_t done = 0;                            // rows of the experts in front
  for (int32_t e0 = 0; e0 < ne; e0 += blockDim.x) {
    const int32_t e = e0 + threadIdx.x;
    int32_t total = 0, before = 0;
    if (e < ne) {
      if constexpr (ALONE) {
        for (int w = 0; w < waves; ++w) total += lds[w * ne + e];
      } else {
        total = totals[e];
        before = befores[e];
      }
    }
    const int32_t at = done + block_before(total, scratch, lane, wave, waves);
    if (e < ne) {
      if (blockIdx.x == 0) a.offsets[e] = at;
      int32_t next = at + before;
      for (int w = 0; w < waves; ++w) {
        const int32_t c = lds[w * ne + e];
        lds[w * ne + e] = next;
        next += c;
      }
    }
    // all rows up to here: the last thread's
    if (threadIdx.x == blockDim.x - 1) scratch[waves] = at + total;
    __syncthreads();
    done = scratch[waves];
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[ne] = done;
  for (int64_t i = done + int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < a.n; i += int64_t(gridDim.x) * blockDim.x) a.tokens[i] = -1;
  // 64 choices at a time: a lane's rank among those of its expert, from a comparison bit by bit
  for (int64_t i0 = lo; i0 < hi; i0 += 64) {
    const int64_t i = i0 + lane;
    int32_t e = ne;
    if (i < hi) {
      const int32_t k = a.experts[i];
      e = k >= 0 && k < ne ? k : ne;
    }
    uint64_t same = ~0ull;
    for (int b = 0; b < bits; ++b) {
      const bool set = (e >> b) & 1;
      const uint64_t v = __ballot(set);
      same &= set ? v : ~v;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    int32_t place = -1;
    if (e < ne) place = mine[e] + rank;
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
    if (e < ne && rank == 0) mine[e] += __popcll(same);
    __threadfence_block();
    __builtin_amdgcn_wave_barrier();
    if (i < hi) {
      a.places[i] = place;
      if (place >= 0) a.tokens[place] = int32_t(by_choices.div(uint32_t(i)));
    }
  }
}

int sort_waves(int64_t n, int64_t n_experts) {
  int waves = 16;
  while (waves > 1 && waves * n_experts > 24 * 1024) waves /= 2;       // 96 KB of counts, and 32 more of the largest number of experts
  while (waves > 1 && int64_t(waves / 2) * 64 >= n) waves /= 2;        // (a wave for every 64 choices is enough)
  return waves;
}
int64_t sort_groups(int64_t n) {
  const int64_t g = ceil_div(n, kGroupKeys);
  return g < kSortGroups ? g : kSortGroups;
}

// ---------------------------------------------------------------------------------------------
// Rows.  Pieces of 16 bytes of a token, wherever rows begin.
// ---------------------------------------------------------------------------------------------
template <bool BIG>
__global__ void __launch_bounds__(kThreads) expert_split_kernel(ExpertRowsArgs a, int64_t row_bytes, Pieces<BIG> n) {
  using Index = typename Pieces<BIG>::Index;
  const Index at = Index(blockIdx.x) * kThreads + threadIdx.x;
  if (at >= n.total) return;
  Index token, piece;
  n.divide(at, &token, &piece);
  const int64_t byte = int64_t(piece) * 16, left = row_bytes - byte;
  const int32_t* const places = a.places + int64_t(token) * a.choices;
  uint8_t* const rows = static_cast<uint8_t*>(a.rows_out) + byte;
  const i32x4 v = load_16<true>(a.flat, int64_t(token) * row_bytes + byte, left);
  for (int64_t j = 0; j < a.choices; ++j) {
    const int32_t p = places[j];
    if (p >= 0 && p < a.count) store_16<1, false>(rows + int64_t(p) * row_bytes, left, v);
  }
}

// A lane has 8 numbers of a token's result; four choices' rows are under way together.
template <int DT, int OUT, bool BIG>
__global__ void __launch_bounds__(kThreads) expert_join_kernel(ExpertRowsArgs a, Pieces<BIG> n) {
  using Index = typename Pieces<BIG>::Index;
  const Index at = Index(blockIdx.x) * kThreads + threadIdx.x;
  if (at >= n.total) return;
  Index token, piece;
  n.divide(at, &token, &piece);
  const int64_t c = int64_t(piece) * 8, left = a.cols - c;
  const int32_t* const places = a.places + int64_t(token) * a.choices;
  const float* const weights = a.weights ? a.weights + int64_t(token) * a.choices : nullptr;
  float sum[8] = {};
  for (int64_t j0 = 0; j0 < a.choices; j0 += 4) {
    float x[4][8], w[4];
    bool there[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t k = j0 + j < a.choices ? j0 + j : a.choices - 1;
      const int32_t p = places[k];
      there[j] = j0 + j < a.choices && p >= 0 && p < a.count;
      w[j] = weights ? weights[k] : 1.0f;
      load_row_numbers<DT, 8>(a.rows, (there[j] ? int64_t(p) : 0) * a.cols + c, there[j] ? left : 0, x[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (there[j])
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += w[j] * x[j][i];
  }
  store_row_numbers<OUT, 8>(a.flat_out, int64_t(token) * a.cols + c, left, sum);
}

// WAVES waves have a token: its gradient, times their weights, into the rows of its choices, and its products with what those rows
// were; four choices at a time.
template <int DT, int WAVES, bool STREAM>
__global__ void __launch_bounds__(256) expert_join_grad_kernel(ExpertRowsArgs a) {
  constexpr int TOKENS = 4 / WAVES, T = WAVES * 64;
  __shared__ float part[4][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t token = int64_t(blockIdx.x) * TOKENS + wave / WAVES;
  if (WAVES == 1 && token >= a.tokens) return;
  const int t = threadIdx.x % T;
  const int32_t* const places = a.places + token * a.choices;
  const float* const weights = a.weights ? a.weights + token * a.choices : nullptr;
  const int64_t pieces = ceil_div(a.cols, 8);
  for (int64_t j0 = 0; j0 < a.choices; j0 += 4) {
    int64_t at[4];
    float w[4], dot[4] = {};
    bool there[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t k = j0 + j < a.choices ? j0 + j : a.choices - 1;
      const int32_t p = places[k];
      there[j] = j0 + j < a.choices && p >= 0 && p < a.count;
      at[j] = (there[j] ? int64_t(p) : 0) * a.cols;
      w[j] = weights ? weights[k] : 1.0f;
    }
    for (int64_t piece = t; piece < pieces; piece += T) {
      const int64_t c = piece * 8, left = a.cols - c;
      float g[8], x[4][8];
      load_row_numbers<DT, 8>(a.flat, token * a.cols + c, left, g);
#pragma unroll
      for (int j = 0; j < 4; ++j) load_row_numbers<DT, 8>(a.rows, at[j] + c, there[j] ? left : 0, x[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!there[j]) continue;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[i] = w[j] * g[i];
          dot[j] += g[i] * x[j][i];
        }
        store_row_numbers<DT, 8, STREAM>(a.rows_out, at[j] + c, left, y);
      }
    }
    if (!a.grad_weights) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int d = 32; d > 0; d /= 2) dot[j] += __shfl_xor(dot[j], d);
    if constexpr (WAVES > 1) {
      if (lane == 0)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[wave][j] = dot[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        dot[j] = part[0][j];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) dot[j] += part[v][j];
      }
      __syncthreads();
    }
    if (t == 0)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j0 + j < a.choices) a.grad_weights[token * a.choices + j0 + j] = there[j] ? dot[j] : 0.0f;
  }
}

template <typename F>
hipError_t by_pieces(int64_t rows, int64_t per_row, F&& launch) {
  const int64_t total = rows * per_row, groups = ceil_div(total, kThreads);
  if (total == 0) return hipSuccess;
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  if (total < (int64_t(1) << 30)) return launch(Pieces<false>{uint32_t(per_row), uint32_t(total), FastDiv::make(uint32_t(per_row))}, unsigned(groups));
  return launch(Pieces<true>{per_row, total, FastDiv::make(1u)}, unsigned(groups));
}

}  // namespace

size_t expert_sort_workspace(int64_t n, int64_t n_experts) {
  const int64_t groups = sort_groups(n);
  return groups <= 1 ? 0 : size_t(round_up(groups * n_experts * 4, 16));
}

hipError_t launch_expert_sort(const ExpertSortArgs& a, hipStream_t s) {
  if (a.n > (int64_t(1) << 30) || a.n_experts > kMaxExperts) return hipErrorInvalidValue;
  const int64_t groups = a.n ? sort_groups(a.n) : 1;
  const int32_t per_group = int32_t(ceil_div(ceil_div(a.n, groups), 64) * 64);
  const int waves = sort_waves(per_group, a.n_experts);
  const int32_t per_wave = int32_t(ceil_div(ceil_div(per_group, waves), 64) * 64);
  int bits = 1;
  while ((int64_t(1) << bits) <= a.n_experts) ++bits;
  const int lds = (waves * int(a.n_experts) + waves + 1 + (groups > 1 ? 2 * int(a.n_experts) : 0)) * 4;
  const FastDiv by_experts = FastDiv::make(uint32_t(a.n_experts > 0 ? a.n_experts : 1));
  const FastDiv by_choices = FastDiv::make(uint32_t(a.choices > 0 ? a.choices : 1));
  if (groups == 1) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(expert_place_kernel<true>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL((expert_place_kernel<true>), dim3(1), dim3(waves * 64), lds, s, a, per_group, per_wave, bits, by_choices, by_experts);
    return hipGetLastError();
  }
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(expert_place_kernel<false>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(expert_count_kernel, dim3(unsigned(groups)), dim3(kSortThreads), 0, s, a, per_group);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((expert_place_kernel<false>), dim3(unsigned(groups)), dim3(waves * 64), lds, s, a, per_group, per_wave, bits, by_choices, by_experts);
  return hipGetLastError();
}

hipError_t launch_expert_split(const ExpertRowsArgs& a, hipStream_t s) {
  const int64_t row_bytes = a.cols * int64_t(dtype_size(a.dtype));
  if (a.choices == 0) return hipSuccess;
  return by_pieces(a.tokens, ceil_div(row_bytes, 16), [&](auto n, unsigned groups) {
    hipLaunchKernelGGL((expert_split_kernel<std::is_same_v<decltype(n), Pieces<true>>>), dim3(groups), dim3(kThreads), 0, s, a, row_bytes, n);
    return hipGetLastError();
  });
}

hipError_t launch_expert_join(const ExpertRowsArgs& a, hipStream_t s) {
  return by_pieces(a.tokens, ceil_div(a.cols, 8), [&](auto n, unsigned groups) {
    constexpr bool BIG = std::is_same_v<decltype(n), Pieces<true>>;
    const dim3 grid(groups), block(kThreads);
    if (a.dtype == GS_BF16 && a.out_dtype == GS_BF16) hipLaunchKernelGGL((expert_join_kernel<GS_BF16, GS_BF16, BIG>), grid, block, 0, s, a, n);
    else if (a.dtype == GS_BF16) hipLaunchKernelGGL((expert_join_kernel<GS_BF16, GS_F32, BIG>), grid, block, 0, s, a, n);
    else if (a.out_dtype == GS_BF16) hipLaunchKernelGGL((expert_join_kernel<GS_F32, GS_BF16, BIG>), grid, block, 0, s, a, n);
    else hipLaunchKernelGGL((expert_join_kernel<GS_F32, GS_F32, BIG>), grid, block, 0, s, a, n);
    return hipGetLastError();
  });
}

hipError_t launch_expert_join_grad(const ExpertRowsArgs& a, hipStream_t s) {
  if (a.tokens == 0 || a.choices == 0) return hipSuccess;
  // A wave for a token, four of them where tokens are too few to fill the chip.
  const bool few = a.tokens < 2048;
  const int64_t groups = few ? a.tokens : ceil_div(a.tokens, 4);
  if (groups > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid{unsigned(groups)}, block(256);
  // Stores with the streaming hint where they fill whole pieces (16384 x 2 rows of 7168 bfloat16 numbers 222 us, 241 without; 8191 x 6 of 2050
  // 116 and 106).
  const bool stream = a.cols * int64_t(dtype_size(a.dtype)) % 16 == 0;
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
  if (a.dtype == GS_BF16) {
    if (few) stream ? launch(expert_join_grad_kernel<GS_BF16, 4, true>) : launch(expert_join_grad_kernel<GS_BF16, 4, false>);
    else stream ? launch(expert_join_grad_kernel<GS_BF16, 1, true>) : launch(expert_join_grad_kernel<GS_BF16, 1, false>);
  } else {
    if (few) stream ? launch(expert_join_grad_kernel<GS_F32, 4, true>) : launch(expert_join_grad_kernel<GS_F32, 4, false>);
    else stream ? launch(expert_join_grad_kernel<GS_F32, 1, true>) : launch(expert_join_grad_kernel<GS_F32, 1, false>);
  }
  return hipGetLastError();
}

}  // namespace gs
