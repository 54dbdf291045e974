// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Forward: y[t] = s E[id_t], one read of the table row and one write.
// Backward: dE[v] += s sum of dy[t] over the tokens t of v.  The tokens are
// sorted stably by id (sort.hpp), so that a table row's tokens are one run of
// the sorted order, are added in token order and the row is read and written
// once; no atomics on values.
#include "sort.hpp"

namespace spr {

namespace {
constexpr int kEmbedThreads = 256;

template <typename T>
struct Vec8;  // eight values of a row
template <>
struct Vec8<bf16> {
  static __device__ __forceinline__ void load(const bf16* p, float (&v)[8]) {
    const bf16x8 x = *(const bf16x8*)p;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
  }
  static __device__ __forceinline__ void store(bf16* p, const float (&v)[8]) {
    bf16x8 x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (bf16)v[j];
    *(bf16x8*)p = x;
  }
};
template <>
struct Vec8<float> {
  static __device__ __forceinline__ void load(const float* p, float (&v)[8]) {
    const f32x4 a = ((const f32x4*)p)[0], b = ((const f32x4*)p)[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = a[j];
      v[j + 4] = b[j];
    }
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
    ((f32x4*)p)[0] = f32x4{v[0], v[1], v[2], v[3]};
    ((f32x4*)p)[1] = f32x4{v[4], v[5], v[6], v[7]};
  }
};
}  // namespace

// chunk c (eight values) of token t per thread
template <typename T>
__global__ __launch_bounds__(kEmbedThreads) void embed_fwd_kernel(const int* __restrict__ ids,
                                                                  const T* __restrict__ table, T* __restrict__ y,
                                                                  long tokens, int vocab, int chunks, float scale) {
  const long i = (long)blockIdx.x * kEmbedThreads + threadIdx.x;
  if (i >= tokens * chunks) return;
  const long t = i / chunks, c = i % chunks;
  const int id = ids[t];
  float v[8] = {};
  if ((unsigned)id < (unsigned)vocab) {
    Vec8<T>::load(table + ((long)id * chunks + c) * 8, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= scale;
  }
  Vec8<T>::store(y + 8 * i, v);
}

// one pass of the sort: keys and the tokens they belong to
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const int* __restrict__ keys,
                                                                  const int* __restrict__ tokens, long n, long per,
                                                                  int limit, int shift, int bins, int mask, int bits,
                                                                  int nb, const int* __restrict__ hist,
                                                                  int* __restrict__ keys_out,
                                                                  int* __restrict__ tokens_out) {
  __shared__ SortLds s;
  sort_bases(s, hist, bins, nb, blockIdx.x, nullptr);
  const long lo = blockIdx.x * per;
  sort_walk(s, keys, lo, min(n, lo + per), limit, shift, mask, bits, [&](long i, int key, int place) {
    keys_out[place] = key;
    tokens_out[place] = tokens ? tokens[i] : (int)i;
  });
}

// the thread of a run's first sorted token adds up one chunk of the run
template <typename T>
__global__ __launch_bounds__(kEmbedThreads) void embed_bwd_kernel(const int* __restrict__ keys,
                                                                  const int* __restrict__ order,
                                                                  const T* __restrict__ dy,
                                                                  float* __restrict__ dtable, long tokens, int vocab,
                                                                  int chunks, float scale) {
  const long i = (long)blockIdx.x * kEmbedThreads + threadIdx.x;
  if (i >= tokens * chunks) return;
  const long p = i / chunks, c = i % chunks;
  const int key = keys[p];
  if (key >= vocab || (p > 0 && keys[p - 1] == key)) return;
  float sum[8] = {};
  for (long q = p; q < tokens && keys[q] == key; ++q) {
    float v[8];
    Vec8<T>::load(dy + ((long)order[q] * chunks + c) * 8, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += v[j];
  }
  float* dst = dtable + ((long)key * chunks + c) * 8;
  float v[8];
  Vec8<float>::load(dst, v);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = fmaf(scale, sum[j], v[j]);
  Vec8<float>::store(dst, v);
}

namespace {
// workspace: two buffers of keys and tokens, then the histograms
struct EmbedWs {
  size_t item, hist, total;
};
EmbedWs embed_ws(long n) {
  EmbedWs w;
  w.item = ((size_t)n * 4 + 255) / 256 * 256;
  w.hist = 4 * w.item;
  w.total = w.hist + sort_hist_bytes(n, 1 << kSortRadixBits);
  return w;
}
}  // namespace

size_t embed_bwd_ws(long tokens, int vocab, int width) { return tokens == 0 ? 0 : embed_ws(tokens).total; }

hipError_t launch_embed_fwd(int dtype, int tokens, int vocab, int width, float scale, const int* ids,
                            const void* table, void* y, hipStream_t st) {
  const long n = (long)tokens * (width / 8);
  if (n == 0) return hipSuccess;
  ProfileScope ps("embed_fwd", st);
  const dim3 grid((unsigned)((n + kEmbedThreads - 1) / kEmbedThreads));
  if (dtype == 1)
    hipLaunchKernelGGL(embed_fwd_kernel<bf16>, grid, dim3(kEmbedThreads), 0, st, ids, (const bf16*)table, (bf16*)y,
                       (long)tokens, vocab, width / 8, scale);
  else
    hipLaunchKernelGGL(embed_fwd_kernel<float>, grid, dim3(kEmbedThreads), 0, st, ids, (const float*)table, (float*)y,
                       (long)tokens, vocab, width / 8, scale);
  return hipGetLastError();
}

hipError_t launch_embed_bwd(int dtype, int tokens, int vocab, int width, float scale, const int* ids, const void* dy,
                            float* dtable, void* ws, hipStream_t st) {
  const long n = tokens;
  if (n == 0) return hipSuccess;
  const EmbedWs w = embed_ws(n);
  char* base = (char*)ws;
  int* keys[2] = {(int*)base, (int*)(base + w.item)};
  int* order[2] = {(int*)(base + 2 * w.item), (int*)(base + 3 * w.item)};
  int* hist = (int*)(base + w.hist);
  const int nb = sort_ranges(n);
  const long per = sort_range_items(n, nb);
  const int* k_in = ids;
  const int* t_in = nullptr;
  int out = 0;
  {
    ProfileScope ps("embed_sort", st);
    for (int shift = 0, left = sort_bits(vocab); left > 0; left -= kSortRadixBits, shift += kSortRadixBits) {
      const int bits = left < kSortRadixBits ? left : kSortRadixBits, bins = 1 << bits, mask = bins - 1;
      hipLaunchKernelGGL(sort_count_kernel, dim3(nb), dim3(kSortThreads), 0, st, k_in, n, per, vocab, shift, bins,
                         mask, hist);
      hipLaunchKernelGGL(embed_sort_kernel, dim3(nb), dim3(kSortThreads), 0, st, k_in, t_in, n, per, vocab, shift,
                         bins, mask, bits, nb, hist, keys[out], order[out]);
      k_in = keys[out];
      t_in = order[out];
      out ^= 1;
    }
  }
  ProfileScope ps("embed_bwd", st);
  const long m = n * (width / 8);
  const dim3 grid((unsigned)((m + kEmbedThreads - 1) / kEmbedThreads));
  if (dtype == 1)
    hipLaunchKernelGGL(embed_bwd_kernel<bf16>, grid, dim3(kEmbedThreads), 0, st, k_in, t_in, (const bf16*)dy, dtable,
                       n, vocab, width / 8, scale);
  else
    hipLaunchKernelGGL(embed_bwd_kernel<float>, grid, dim3(kEmbedThreads), 0, st, k_in, t_in, (const float*)dy,
                       dtable, n, vocab, width / 8, scale);
  return hipGetLastError();
}

}  // namespace spr
