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
  for (long i = (long)blockIdx.x * kEmbedThreads + threadIdx.x; i < tokens * chunks;
       i += (long)gridDim.x * kEmbedThreads) {
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
}

// Up to kFewTokens tokens: no sort and one launch.  The wave of a token and 512
// columns holds all ids, four a lane; where the token is its id's first, it adds
// up the rows of all of the id's tokens in order, eight at a time.
constexpr int kFewTokens = 256;

template <typename T>
__global__ __launch_bounds__(kEmbedThreads) void embed_few_kernel(const int* __restrict__ ids,
                                                                  const T* __restrict__ dy, float* dtable, int tokens,
                                                                  int vocab, int chunks, int slabs, float scale) {
  constexpr int kWaves = kEmbedThreads / 64;
  const int lane = threadIdx.x & 63;
  for (long wave = (long)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
       wave < (long)tokens * slabs; wave += (long)gridDim.x * kWaves) {
    const int t = (int)wave / slabs, chunk = (int)wave % slabs * 64 + lane;
    const int id = ids[t];
    if ((unsigned)id >= (unsigned)vocab) continue;
    const bool in = chunk < chunks;
    float* dst = dtable + ((long)id * chunks + chunk) * 8;
    float old[8] = {}, sum[8] = {};
    if (in) Vec8<float>::load(dst, old);
    unsigned long long same[kFewTokens / 64];
#pragma unroll
    for (int c = 0; c < kFewTokens / 64; ++c) {
      const int j = 64 * c + lane;
      same[c] = __ballot(j < tokens && ids[min(j, tokens - 1)] == id);
    }
    // the next of the id's tokens, or -1
    auto next = [&]() -> int {
      int at = -1;
#pragma unroll
      for (int c = kFewTokens / 64 - 1; c >= 0; --c)
        if (same[c] != 0) at = 64 * c + __builtin_ctzll(same[c]);
#pragma unroll
      for (int c = 0; c < kFewTokens / 64; ++c)
        if (at >= 0 && at >> 6 == c) same[c] &= same[c] - 1;
      return at;
    };
    int row = next();
    if (row != t) continue;  // an earlier token's wave does it
    while (row >= 0) {
      float v[8][8] = {};
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (row >= 0) {
          if (in) Vec8<T>::load(dy + ((long)row * chunks + chunk) * 8, v[q]);
          row = next();
        }
      }
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[q][j];
    }
    if (!in) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) old[j] = fmaf(scale, sum[j], old[j]);
    Vec8<float>::store(dst, old);
  }
}

// Up to kRankTokens tokens: a token's place is the number of keys that sort
// before it, counted by 32 lanes.  One launch, where a radix pass takes two.
// Whole call of width 1024, us, by counting / in radix passes: 4096 tokens 23 /
// 31, 8192 31 / 39, 12000 46 / 44.  (Eight lanes a token: 32 and 51.)
constexpr int kRankTokens = 8192, kRankLanes = 32, kRankThreads = 1024;
static_assert(kRankTokens >= kSortSelfCount, "a sort in radix passes has its counts in a launch of their own");

__global__ __launch_bounds__(kRankThreads) void embed_rank_kernel(const int* __restrict__ ids, int tokens, int vocab,
                                                                  int* __restrict__ keys_out,
                                                                  int* __restrict__ tokens_out) {
  __shared__ __attribute__((aligned(16))) unsigned keys[kRankTokens];
  // whole rounds of 4 keys a lane; the places behind the last token sort last
  const int round = 4 * kRankLanes, padded = (tokens + round - 1) / round * round;
#pragma unroll 4
  for (int i = threadIdx.x; i < padded; i += kRankThreads)
    keys[i] = i < tokens ? (unsigned)sort_key(ids[i], vocab) : 0xffffffffu;
  __syncthreads();
  const int mine = blockIdx.x * (kRankThreads / kRankLanes) + threadIdx.x / kRankLanes, part = threadIdx.x % kRankLanes;
  if (mine >= tokens) return;
  const unsigned key = keys[mine];
  // smaller keys, and equal ones of earlier quads; then those of its own quad
  int before = 0;
#pragma unroll 4
  for (int j = 4 * part; j < padded; j += round) {
    const uint4 k = *(const uint4*)(keys + j);
    const unsigned bound = key + (j + 4 <= mine);
    before += (k.x < bound) + (k.y < bound) + (k.z < bound) + (k.w < bound);
  }
  if (part < mine % 4) before += keys[mine / 4 * 4 + part] == key;
#pragma unroll
  for (int o = 1; o < kRankLanes; o <<= 1) before += __shfl_xor(before, o);
  if (part == 0) {
    keys_out[before] = (int)key;
    tokens_out[before] = mine;
  }
}

// one pass of the sort: keys and the tokens they belong to
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(SortPass p, const int* __restrict__ tokens,
                                                                  int* __restrict__ keys_out,
                                                                  int* __restrict__ tokens_out) {
  __shared__ SortLds s;
  sort_bases(s, p, nullptr);
  sort_walk(s, p, [&](long i, int key, int place) {
    keys_out[place] = key;
    tokens_out[place] = tokens ? tokens[i] : (int)i;
  });
}

// Sums of runs (the sorted tokens of one id).  A wave takes `len` consecutive
// sorted tokens, a span, and 512 columns (eight a lane), so that a frequent id's
// run is shared by many waves.  A run that lies inside the span is added to its
// table row at once; the part of one that began before it goes to head[span], the
// part of one that begins here and goes on to tail[span], and embed_join adds
// those up in order.  Per element that is the order of the tokens within a span,
// then of the spans.  HBM bound: a row of dy is read once, a row of the table read
// and written once, a part (at most two a span) written and read once.
// 28672 tokens x 4096 of log-uniform ids: 124 us (4.7 TB/s; one thread a run and
// chunk 1.9 ms).
constexpr int kAhead = 4;

template <typename T>
__global__ __launch_bounds__(kEmbedThreads) void embed_runs_kernel(const int* __restrict__ keys,
                                                                   const int* __restrict__ order,
                                                                   const T* __restrict__ dy, float* dtable,
                                                                   float* __restrict__ head, float* __restrict__ tail,
                                                                   int tokens, int vocab, int chunks, int slabs,
                                                                   int len, float scale) {
  const long wave = (long)blockIdx.x * (kEmbedThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long span = wave / slabs;
  const int lane = threadIdx.x & 63, chunk = (int)(wave % slabs) * 64 + lane;
  const long p0 = span * len;
  if (p0 >= tokens) return;
  const int n = (int)min((long)len, tokens - p0);
  // lane q holds the span's q-th key and token
  int key = vocab, token = 0;
  if (lane < n) {
    key = keys[p0 + lane];
    token = order[p0 + lane];
  }
  const int behind = p0 + len < tokens ? keys[p0 + len] : vocab, before = p0 > 0 ? keys[p0 - 1] : vocab;
  auto key_at = [&](int q) { return __builtin_amdgcn_readlane(key, q); };
  const bool in = chunk < chunks;
  float sum[8] = {};
  float v[kAhead][8];
  auto fetch = [&](int q, float (&to)[8]) {
    const int t = __builtin_amdgcn_readlane(token, q);
    if (in) Vec8<T>::load(dy + ((long)t * chunks + chunk) * 8, to);
  };
#pragma unroll
  for (int q = 0; q < kAhead; ++q)
    if (q < n && key_at(q) < vocab) fetch(q, v[q]);
  bool first = true;  // of the run that the sum holds: it begins the span
  for (int q0 = 0; q0 < n; q0 += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int q = q0 + u;
      if (q >= n) break;
      const int k = key_at(q);
      if (k >= vocab) return;  // dropped tokens are the last ones
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[u][j];
      if (q + kAhead < n && key_at(q + kAhead) < vocab) fetch(q + kAhead, v[u]);
      const int next = q + 1 < n ? key_at(q + 1) : behind;
      if (next == k && q + 1 < n) continue;
      if (in) {
        if (first && before == k) {
          Vec8<float>::store(head + (span * chunks + chunk) * 8, sum);
        } else if (next == k) {
          Vec8<float>::store(tail + (span * chunks + chunk) * 8, sum);
        } else {
          float* dst = dtable + ((long)k * chunks + chunk) * 8;
          float old[8];
          Vec8<float>::load(dst, old);
#pragma unroll
          for (int j = 0; j < 8; ++j) old[j] = fmaf(scale, sum[j], old[j]);
          Vec8<float>::store(dst, old);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] = 0.f;
      first = false;
    }
  }
}

// The runs that cross spans: the wave of the span where one begins adds its
// tail and the heads of the spans up to its end, eight at a time.  A chain of
// dependent loads: the first head and the table's row are read while the run's
// end is looked for (eight heads ahead would read more than most runs have: 25 us
// instead of 12 at 28672 tokens x 4096).
__global__ __launch_bounds__(kEmbedThreads) void embed_join_kernel(const int* __restrict__ keys, float* dtable,
                                                                   const float* __restrict__ head,
                                                                   const float* __restrict__ tail, int tokens,
                                                                   int vocab, int chunks, int slabs, int len,
                                                                   float scale) {
  const long wave = (long)blockIdx.x * (kEmbedThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long span = wave / slabs, p0 = span * len;
  const int lane = threadIdx.x & 63, chunk = (int)(wave % slabs) * 64 + lane;
  if (p0 + len >= tokens) return;
  const int before = keys[p0 > 0 ? p0 - 1 : 0], at = keys[p0], k = keys[p0 + len - 1], next = keys[p0 + len];
  // a run begins here and goes on
  if ((k >= vocab) | (next != k) | ((p0 > 0) & (at == k) & (before == k))) return;
  const long spans = ((long)tokens + len - 1) / len;
  const bool in = chunk < chunks;
  float* dst = dtable + ((long)k * chunks + chunk) * 8;
  float sum[8] = {}, old[8] = {}, one[8] = {};
  if (in) {
    Vec8<float>::load(tail + (span * chunks + chunk) * 8, sum);
    Vec8<float>::load(head + ((span + 1) * chunks + chunk) * 8, one);
    Vec8<float>::load(dst, old);
  }
  // the run's last span: the first one behind this that does not hold it whole
  // and go on, found 64 spans at a time
  long end = span;
  for (long s = span + 1;; s += 64) {
    const long mine = s + lane;
    const bool on = mine + 1 < spans && keys[mine * len + len - 1] == k && keys[mine * len + len] == k;
    const unsigned long long off = __ballot(!on);
    if (off != 0) {
      end = s + __builtin_ctzll(off);
      break;
    }
  }
  if (!in) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] += one[j];
  for (long s = span + 2; s <= end; s += 8) {
    float v[8][8] = {};
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (s + q <= end) Vec8<float>::load(head + ((s + q) * chunks + chunk) * 8, v[q]);
#pragma unroll
    for (int q = 0; q < 8; ++q)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[q][j];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) old[j] = fmaf(scale, sum[j], old[j]);
  Vec8<float>::store(dst, old);
}

namespace {
// Tokens of a span: a power of two that leaves about 4096 waves (four a SIMD),
// from 8 to the 64 that a wave holds keys of.  Short spans cross more runs, whose
// parts are written and read again; long ones leave CUs idle.  Whole call, us,
// with 2048 / 4096 / 8192 waves as the aim, width 4096: 28672 tokens 179 / 163 /
// 178, 8192 tokens 80 / 65 / 68, 28672 tokens of 500 ids 91 / 84 / 95.
int embed_span(long n, long slabs) {
  int len = 8;
  while (len < 64 && 2 * len * 4096L <= n * slabs) len *= 2;
  return len;
}
// workspace: two buffers of keys and tokens, the histograms, then the parts of
// runs that cross spans (more than kFewTokens tokens are several spans)
struct EmbedWs {
  size_t item, hist, head, tail, total;
};
EmbedWs embed_ws(long n, long width) {
  const int len = embed_span(n, (width / 8 + 63) / 64);
  EmbedWs w;
  w.item = ((size_t)n * 4 + 255) / 256 * 256;
  w.hist = 4 * w.item;
  w.head = w.hist + (sort_hist_bytes(n, 1 << kSortRadixBits) + 255) / 256 * 256;
  const size_t part = (size_t)((n + len - 1) / len) * width * 4;
  w.tail = w.head + part;
  w.total = w.tail + part;
  return w;
}
}  // namespace

size_t embed_bwd_ws(long tokens, int vocab, int width) {
  return tokens <= kFewTokens ? 0 : embed_ws(tokens, width).total;
}

hipError_t launch_embed_fwd(int dtype, int tokens, int vocab, int width, float scale, const int* ids,
                            const void* table, void* y, hipStream_t st) {
  const long n = (long)tokens * (width / 8);
  if (n == 0) return hipSuccess;
  ProfileScope ps("embed_fwd", st);
  const dim3 grid(grid_of((n + kEmbedThreads - 1) / kEmbedThreads, kEmbedThreads));
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
  if (n <= kFewTokens) {
    ProfileScope ps("embed_few", st);
    const int few_slabs = (width / 8 + 63) / 64;
    const dim3 few_grid(grid_of((n * few_slabs + kEmbedThreads / 64 - 1) / (kEmbedThreads / 64), kEmbedThreads));
    if (dtype == 1)
      hipLaunchKernelGGL(embed_few_kernel<bf16>, few_grid, dim3(kEmbedThreads), 0, st, ids, (const bf16*)dy, dtable,
                         tokens, vocab, width / 8, few_slabs, scale);
    else
      hipLaunchKernelGGL(embed_few_kernel<float>, few_grid, dim3(kEmbedThreads), 0, st, ids, (const float*)dy, dtable,
                         tokens, vocab, width / 8, few_slabs, scale);
    return hipGetLastError();
  }
  const EmbedWs w = embed_ws(n, width);
  char* base = (char*)ws;
  int* keys[2] = {(int*)base, (int*)(base + w.item)};
  int* order[2] = {(int*)(base + 2 * w.item), (int*)(base + 3 * w.item)};
  int* hist = (int*)(base + w.hist);
  const int nb = sort_ranges(n);
  const long per = sort_range_items(n, nb);
  const int* k_in = ids;
  const int* t_in = nullptr;
  int out = 0;
  if (n <= kRankTokens) {
    ProfileScope ps("embed_rank", st);
    constexpr int per_block = kRankThreads / kRankLanes;
    hipLaunchKernelGGL(embed_rank_kernel, dim3((tokens + per_block - 1) / per_block), dim3(kRankThreads), 0, st, ids,
                       tokens, vocab, keys[0], order[0]);
    k_in = keys[0];
    t_in = order[0];
  }
  for (int shift = 0, left = n <= kRankTokens ? 0 : sort_bits(vocab); left > 0; left -= kSortRadixBits, shift += kSortRadixBits) {
    const int bits = left < kSortRadixBits ? left : kSortRadixBits;
    const SortPass p = {k_in, n, per, vocab, shift, bits, 1 << bits, nb, hist};
    {
      ProfileScope ps("sort_count", st);
      hipLaunchKernelGGL(sort_count_kernel, dim3(nb), dim3(kSortThreads), 0, st, p);
    }
    ProfileScope ps("embed_sort", st);
    hipLaunchKernelGGL(embed_sort_kernel, dim3(nb), dim3(kSortThreads), 0, st, p, t_in, keys[out], order[out]);
    k_in = keys[out];
    t_in = order[out];
    out ^= 1;
  }
  const int chunks = width / 8, slabs = (chunks + 63) / 64, len = embed_span(n, slabs);
  float* head = (float*)(base + w.head);
  float* tail = (float*)(base + w.tail);
  const long waves = (n + len - 1) / len * slabs;
  const dim3 grid((unsigned)((waves + kEmbedThreads / 64 - 1) / (kEmbedThreads / 64)));
  {
    ProfileScope ps("embed_runs", st);
    if (dtype == 1)
      hipLaunchKernelGGL(embed_runs_kernel<bf16>, grid, dim3(kEmbedThreads), 0, st, k_in, t_in, (const bf16*)dy,
                         dtable, head, tail, tokens, vocab, chunks, slabs, len, scale);
    else
      hipLaunchKernelGGL(embed_runs_kernel<float>, grid, dim3(kEmbedThreads), 0, st, k_in, t_in, (const float*)dy,
                         dtable, head, tail, tokens, vocab, chunks, slabs, len, scale);
  }
  {
    ProfileScope ps("embed_join", st);
    hipLaunchKernelGGL(embed_join_kernel, grid, dim3(kEmbedThreads), 0, st, k_in, dtable, head, tail, tokens, vocab,
                       chunks, slabs, len, scale);
  }
  return hipGetLastError();
}

}  // namespace spr
