// The plan that sorts a router's choices by expert, and the weighted sum of
// the experts' rows with its backward.  All HBM bound.
#include "sort.hpp"

namespace spr {

namespace {
constexpr int kRowThreads = 256;

__device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
  const bf16x8 x = *(const bf16x8*)p;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  bf16x8 x;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (bf16)v[j];
  *(bf16x8*)p = x;
}
}  // namespace

// One pass of the stable sort with a bin per expert; dropped choices are the
// last bin, whose start is offsets[E].
__global__ __launch_bounds__(kSortThreads) void experts_plan_kernel(SortPass p, int k, int* __restrict__ offsets,
                                                                    int* __restrict__ row_token,
                                                                    int* __restrict__ pos) {
  __shared__ SortLds s;
  sort_bases(s, p, offsets);
  sort_walk(s, p, [&](long i, int key, int place) {
    row_token[place] = key < p.limit ? (int)((unsigned)i / (unsigned)k) : -1;
    pos[i] = key < p.limit ? place : -1;
  });
}

// a workgroup per token, eight values a thread
__global__ __launch_bounds__(kRowThreads) void combine_fwd_kernel(const bf16* __restrict__ y,
                                                                  const int* __restrict__ pos,
                                                                  const float* __restrict__ weights, const bf16* add,
                                                                  bf16* out, long tokens, int k, int rows,
                                                                  int chunks) {
  for (long t = blockIdx.x; t < tokens; t += gridDim.x) {
    for (int c = threadIdx.x; c < chunks; c += kRowThreads) {
      float sum[8] = {};
      for (int j = 0; j < k; ++j) {
        const int p = pos[t * k + j];
        if ((unsigned)p >= (unsigned)rows) continue;
        const float w = weights ? weights[t * k + j] : 1.f;
        float v[8];
        load8(y + ((long)p * chunks + c) * 8, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, v[i], sum[i]);
      }
      const long at = (t * chunks + c) * 8;
      if (add) {
        float v[8];
        load8(add + at, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];
      }
      store8(out + at, sum);
    }
  }
}

// a wave per choice
__global__ __launch_bounds__(kRowThreads) void combine_bwd_kernel(const bf16* __restrict__ dout,
                                                                  const bf16* __restrict__ y,
                                                                  const int* __restrict__ pos,
                                                                  const float* __restrict__ weights,
                                                                  bf16* __restrict__ dy, float* __restrict__ dweights,
                                                                  long slots, int k, int rows, int chunks) {
  constexpr int kWaves = kRowThreads / 64;
  const int lane = threadIdx.x & 63;
  for (long i = (long)blockIdx.x * kWaves + (threadIdx.x >> 6); i < slots; i += (long)gridDim.x * kWaves) {
    const int p = pos[i];
    if ((unsigned)p >= (unsigned)rows) {
      if (dweights && lane == 0) dweights[i] = 0.f;
      continue;
    }
    const float w = weights ? weights[i] : 1.f;
    const bf16* d = dout + i / k * chunks * 8;
    float dot = 0.f;
    for (int c = lane; c < chunks; c += 64) {
      float g[8], o[8];
      load8(d + 8 * c, g);
      if (dweights) {
        float v[8];
        load8(y + ((long)p * chunks + c) * 8, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) dot = fmaf(v[j], g[j], dot);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = w * g[j];
      store8(dy + ((long)p * chunks + c) * 8, o);
    }
    if (dweights) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
      if (lane == 0) dweights[i] = dot;
    }
  }
}

size_t experts_plan_ws(int E, long slots) { return sort_hist_bytes(slots, E + 1); }

hipError_t launch_experts_plan(int E, int k, long slots, const int* experts, int* offsets, int* row_token, int* pos,
                               void* ws, hipStream_t st) {
  const int nb = sort_ranges(slots);
  const SortPass p = {experts, slots, sort_range_items(slots, nb), E, 0, sort_bits(E), E + 1, nb, (int*)ws};
  if (sort_counts(slots)) {
    ProfileScope ps("sort_count", st);
    hipLaunchKernelGGL(sort_count_kernel, dim3(nb), dim3(kSortThreads), 0, st, p);
  }
  ProfileScope ps("experts_plan", st);
  hipLaunchKernelGGL(experts_plan_kernel, dim3(nb), dim3(kSortThreads), 0, st, p, k, offsets, row_token, pos);
  return hipGetLastError();
}

hipError_t launch_combine_fwd(int tokens, int k, int rows, int width, const void* y, const int* pos,
                              const float* weights, const void* add, void* out, hipStream_t st) {
  if (tokens == 0) return hipSuccess;
  ProfileScope ps("experts_combine_fwd", st);
  hipLaunchKernelGGL(combine_fwd_kernel, dim3(grid_of(tokens, kRowThreads)), dim3(kRowThreads), 0, st, (const bf16*)y, pos,
                     weights, (const bf16*)add, (bf16*)out, (long)tokens, k, rows, width / 8);
  return hipGetLastError();
}

hipError_t launch_combine_bwd(int tokens, int k, int rows, int width, const void* dout, const void* y, const int* pos,
                              const float* weights, void* dy, float* dweights, hipStream_t st) {
  const long slots = (long)tokens * k;
  if (slots == 0) return hipSuccess;
  ProfileScope ps("experts_combine_bwd", st);
  hipLaunchKernelGGL(combine_bwd_kernel, dim3(grid_of((slots + 3) / 4, kRowThreads)), dim3(kRowThreads), 0, st,
                     (const bf16*)dout, (const bf16*)y, pos, weights, (bf16*)dy, dweights, slots, k, rows, width / 8);
  return hipGetLastError();
}

}  // namespace spr
