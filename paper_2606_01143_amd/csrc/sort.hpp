// Stable counting sort of int32 keys on the device, one digit of a pass at a
// time: positions of the keys in (key, index) order, the same every run.
//
// A pass cuts the items into equal ranges, one per workgroup.  A range's places
// need the counts of all items, and of those before it: sort_count writes each
// range's histogram first, or, of up to 4096 items, every workgroup counts all
// of them itself and the launch is saved.  (Of 28672 items too, a pass took 20
// us instead of 12: the counting's conflicts in LDS.)  The placing kernel walks
// its range 1024 items at a time: a wave's equal digits are matched with one
// ballot per bit, their counts are summed over the sixteen waves through LDS,
// and the running start of each digit moves on.  Only integer counts are added
// atomically, so no result depends on an order of execution.
//
// Latency bound.  28672 keys below 128000, two passes of nine bits: 23 us (with
// 256 threads a workgroup 40).
#pragma once

#include "launch.hpp"

namespace spr {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSortMaxBins = 1025;   // 1024 experts and the dropped choices
constexpr int kSortRadixBits = 9;    // a pass of a longer key
constexpr int kSortMaxRanges = 64;
constexpr long kSortSelfCount = 4096;  // items that every workgroup counts for itself

// keys outside [0, limit) sort last, as `limit`
__device__ __forceinline__ int sort_key(int id, int limit) { return (unsigned)id < (unsigned)limit ? id : limit; }

inline int sort_ranges(long n) {
  const long r = (n + kSortThreads - 1) / kSortThreads;
  return (int)(r < 1 ? 1 : r > kSortMaxRanges ? kSortMaxRanges : r);
}
inline bool sort_counts(long n) { return n > kSortSelfCount; }  // sort_count runs first
inline long sort_range_items(long n, int nb) { return ((n + nb - 1) / nb + kSortThreads - 1) / kSortThreads * kSortThreads; }
inline int sort_bits(long top) {  // bits of keys 0 .. top
  int b = 1;
  while (b < 31 && (top >> b) != 0) ++b;
  return b;
}
inline size_t sort_hist_bytes(long n, int bins) { return sort_counts(n) ? (size_t)sort_ranges(n) * bins * 4 : 0; }

// One digit of the keys.
struct SortPass {
  const int* keys;
  long n, per;  // items, and those of a range
  int limit, shift, bits, bins, ranges;
  int* hist;    // [ranges][bins]
  __device__ __forceinline__ int digit(int key) const { return (key >> shift) & ((1 << bits) - 1); }
};

static __global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass p) {
  __shared__ int cnt[kSortMaxBins];
  for (int i = threadIdx.x; i < p.bins; i += kSortThreads) cnt[i] = 0;
  __syncthreads();
  const long lo = blockIdx.x * p.per, hi = min(p.n, lo + p.per);
  for (long i = lo + threadIdx.x; i < hi; i += kSortThreads) atomicAdd(&cnt[p.digit(sort_key(p.keys[i], p.limit))], 1);
  __syncthreads();
  for (int i = threadIdx.x; i < p.bins; i += kSortThreads) p.hist[(long)blockIdx.x * p.bins + i] = cnt[i];
}

struct SortLds {
  int base[kSortMaxBins], total[kSortMaxBins];
  int wave[kSortWaves * kSortMaxBins];
  int scan[kSortWaves];
};

// base[b] = items with a smaller digit, plus those of digit b in earlier
// ranges.  starts != null: the digits' starts over all ranges, written by the
// first workgroup.  Every thread of the workgroup takes part; ends in a barrier.
__device__ __forceinline__ void sort_bases(SortLds& s, const SortPass& p, int* starts) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, bins = p.bins;
  for (int i = t; i < bins; i += kSortThreads) s.base[i] = s.total[i] = 0;
  __syncthreads();
  if (p.n <= kSortSelfCount) {
    // base: items before this range; total: the others, and then all
    const int n = (int)p.n, lo = (int)(blockIdx.x * p.per);
#pragma unroll 4
    for (int i = t; i < n; i += kSortThreads) atomicAdd((i < lo ? s.base : s.total) + p.digit(sort_key(p.keys[i], p.limit)), 1);
    __syncthreads();
    for (int i = t; i < bins; i += kSortThreads) s.total[i] += s.base[i];
  } else {
    // threads beyond one per bin share the ranges
    const int groups = max(1, kSortThreads / bins), block = blockIdx.x;
    for (int i = t; i < groups * bins; i += kSortThreads) {
      const int b = i % bins;
      int all = 0, before = 0;
#pragma unroll 8
      for (int r = i / bins; r < p.ranges; r += groups) {
        const int c = p.hist[r * bins + b];
        all += c;
        before += r < block ? c : 0;
      }
      atomicAdd(&s.total[b], all);
      atomicAdd(&s.base[b], before);
    }
  }
  __syncthreads();
  const int mine = t < bins ? s.total[t] : 0;
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 63) s.scan[w] = upto;
  __syncthreads();
  int start = upto - mine;
  for (int q = 0; q < w; ++q) start += s.scan[q];
  if (t < bins) {
    s.base[t] += start;
    if (starts != nullptr && blockIdx.x == 0) starts[t] = start;
  }
  if (t == kSortThreads - 1 && bins > kSortThreads) {  // the one bin beyond the threads
    s.base[kSortThreads] += start + mine;
    if (starts != nullptr && blockIdx.x == 0) starts[kSortThreads] = start + mine;
  }
  __syncthreads();
}

// Calls put(i, key, place) for every item i of this workgroup's range with its
// place in the sorted order; every thread of the workgroup takes part.
template <typename Put>
__device__ __forceinline__ void sort_walk(SortLds& s, const SortPass& p, Put put) {
  const int t = threadIdx.x, lane = t & 63, bins = p.bins;
  int* counts = s.wave + (t >> 6) * bins;
  const unsigned long long below = (1ull << lane) - 1;
  const long lo = blockIdx.x * p.per, hi = min(p.n, lo + p.per);
  for (long at = lo; at < hi; at += kSortThreads) {
    const long i = at + t;
    const bool in = i < hi;
    const int key = in ? sort_key(p.keys[i], p.limit) : 0, digit = p.digit(key);
    for (int q = t; q < kSortWaves * bins; q += kSortThreads) s.wave[q] = 0;
    unsigned long long same = __ballot(in);
    for (int b = 0; b < p.bits; ++b) {
      const bool one = (digit >> b) & 1;
      const unsigned long long m = __ballot(one);
      same &= one ? m : ~m;
    }
    const int rank = __popcll(same & below);
    __syncthreads();
    if (in && rank == 0) counts[digit] = __popcll(same);
    __syncthreads();
    for (int b = t; b < bins; b += kSortThreads) {
      int run = s.base[b];
#pragma unroll
      for (int q = 0; q < kSortWaves; ++q) {
        const int c = s.wave[q * bins + b];
        s.wave[q * bins + b] = run;
        run += c;
      }
      s.base[b] = run;
    }
    __syncthreads();
    if (in) put(i, key, counts[digit] + rank);
    __syncthreads();
  }
}

}  // namespace spr
