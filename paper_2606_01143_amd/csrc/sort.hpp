// Stable counting sort of int32 keys on the device, one digit of a pass at a
// time: positions of the keys in (key, index) order, the same every run.
//
// A pass cuts the items into nb equal ranges, one per workgroup.  sort_count
// writes each range's histogram; sort_place adds up the histograms before its
// own (all smaller digits, and its digit in earlier ranges) and then walks its
// range 256 items at a time: a wave's equal digits are matched with one ballot
// per bit, their counts per wave go through LDS, and the running start of each
// digit moves on.  Only integer counts are added atomically, so no result
// depends on an order of execution.
#pragma once

#include "launch.hpp"

namespace spr {

constexpr int kSortThreads = 256, kSortWaves = kSortThreads / 64;
constexpr int kSortMaxBins = 1025;   // 1024 experts and the dropped choices
constexpr int kSortRadixBits = 9;    // a pass of a longer key
constexpr int kSortMaxRanges = 64;

// keys outside [0, limit) sort last, as `limit`
__device__ __forceinline__ int sort_key(int id, int limit) { return (unsigned)id < (unsigned)limit ? id : limit; }

inline int sort_ranges(long n) {
  const long r = (n + 1023) / 1024;
  return (int)(r < 1 ? 1 : r > kSortMaxRanges ? kSortMaxRanges : r);
}
inline long sort_range_items(long n, int nb) { return ((n + nb - 1) / nb + kSortThreads - 1) / kSortThreads * kSortThreads; }
inline int sort_bits(long top) {  // bits of keys 0 .. top
  int b = 1;
  while (b < 31 && (top >> b) != 0) ++b;
  return b;
}
inline size_t sort_hist_bytes(long n, int bins) { return (size_t)sort_ranges(n) * bins * 4; }

__global__ __launch_bounds__(kSortThreads) static void sort_count_kernel(const int* __restrict__ keys, long n,
                                                                         long per, int limit, int shift, int bins,
                                                                         int mask, int* __restrict__ hist) {
  __shared__ int cnt[kSortMaxBins];
  for (int i = threadIdx.x; i < bins; i += kSortThreads) cnt[i] = 0;
  __syncthreads();
  const long lo = blockIdx.x * per, hi = min(n, lo + per);
  for (long i = lo + threadIdx.x; i < hi; i += kSortThreads) atomicAdd(&cnt[(sort_key(keys[i], limit) >> shift) & mask], 1);
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) hist[(long)blockIdx.x * bins + i] = cnt[i];
}

struct SortLds {
  int base[kSortMaxBins];
  int wave[kSortWaves][kSortMaxBins];
  int scan[kSortThreads];
};

// base[b] = items with a smaller digit, plus those of digit b in earlier
// ranges; returns after a barrier.  starts != null: the digits' starts over
// all ranges, bins entries, written by the first workgroup.
__device__ __forceinline__ void sort_bases(SortLds& s, const int* __restrict__ hist, int bins, int nb, int block,
                                           int* starts) {
  // thread t owns bins [t * per, (t + 1) * per)
  const int per = (bins + kSortThreads - 1) / kSortThreads;
  int sum = 0;
  for (int q = 0; q < per; ++q) {
    const int b = threadIdx.x * per + q;
    if (b < bins) {
      int all = 0, before = 0;
      for (int r = 0; r < nb; ++r) {
        const int c = hist[(long)r * bins + b];
        all += c;
        before += r < block ? c : 0;
      }
      s.base[b] = before;
      s.wave[0][b] = all;
      sum += all;
    }
  }
  s.scan[threadIdx.x] = sum;
  __syncthreads();
  for (int o = 1; o < kSortThreads; o <<= 1) {
    const int v = threadIdx.x >= o ? s.scan[threadIdx.x - o] : 0;
    __syncthreads();
    s.scan[threadIdx.x] += v;
    __syncthreads();
  }
  int start = threadIdx.x ? s.scan[threadIdx.x - 1] : 0;
  for (int q = 0; q < per; ++q) {
    const int b = threadIdx.x * per + q;
    if (b < bins) {
      const int all = s.wave[0][b];
      s.base[b] += start;
      if (starts != nullptr && block == 0) starts[b] = start;
      start += all;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kSortWaves * kSortMaxBins; i += kSortThreads) (&s.wave[0][0])[i] = 0;
  __syncthreads();
}

// Calls put(i, key, place) for every item i of [lo, hi) with its place in
// the sorted order; every thread of the workgroup takes part.
template <typename Put>
__device__ __forceinline__ void sort_walk(SortLds& s, const int* __restrict__ keys, long lo, long hi, int limit,
                                          int shift, int mask, int bits, Put put) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const unsigned long long below = (1ull << lane) - 1;
  for (long at = lo; at < hi; at += kSortThreads) {
    const long i = at + threadIdx.x;
    const bool in = i < hi;
    const int key = in ? sort_key(keys[i], limit) : 0;
    const int digit = (key >> shift) & mask;
    unsigned long long same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
      const bool one = (digit >> b) & 1;
      const unsigned long long m = __ballot(one);
      same &= one ? m : ~m;
    }
    const int rank = __popcll(same & below);
    const bool first = in && rank == 0;
    if (first) s.wave[w][digit] = __popcll(same);
    __syncthreads();
    if (in) {
      int place = s.base[digit] + rank;
      for (int q = 0; q < w; ++q) place += s.wave[q][digit];
      put(i, key, place);
    }
    __syncthreads();
    if (first) {
      atomicAdd(&s.base[digit], __popcll(same));
      s.wave[w][digit] = 0;
    }
    __syncthreads();
  }
}

}  // namespace spr
