// Per-head RMS norm with gain and rotary embedding of queries and keys in one
// pass, forward and backward.
//
// Row x (one head of one token, d values), r = 1 / sqrt(mean(x^2) + eps):
//   z_j = x_j g_j r;  y = R z, pairs (j, j + d/2) turned by the token's angle.
//   dz = R^T dy;  dx_j = r g_j dz_j - x_j r^3 mean(g dz x);
//   dg_j = sum over rows of dz_j x_j r.
// The backward forms r again from the row it reads anyway, so the forward
// keeps nothing.  Sums, norms and angles are fp32 (the angle's reduction fp64).
#include <math.h>

#include <algorithm>

#include "launch.hpp"

namespace spr {

namespace {
constexpr int kHeadThreads = 256, kHeadWaves = kHeadThreads / 64;
constexpr int kMaxPairs = 2;  // pairs of a lane: head_dim / 2 <= 128

// sum over the wave, the same in every lane
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// cos and sin of position pos at frequency theta^(-2 j / d), as turns: the
// angle's whole turns are dropped in fp64, the rest is exact in its last bits
// at any int32 position
__device__ __forceinline__ float2 head_angle(double pos, int j, const HeadArgs& a) {
  const double turns = pos * exp2((double)j * a.log2_step) * (0.5 / M_PI);
  float sn, cs;
  sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
  return make_float2(cs, sn);
}
__device__ __forceinline__ double head_pos(const HeadArgs& a, long t) {
  return (double)a.pos0 + (a.positions ? (double)a.positions[t] : (double)t);
}
}  // namespace

// ------------------------------------------------ any head dim and alignment
// A wave per row; lane l has the pairs l and l + 64.
template <typename T>
__global__ __launch_bounds__(kHeadThreads) void head_norm_rope_fwd_kernel(HeadArgs a) {
  const int lane = threadIdx.x & 63, heads = a.hq + a.hkv, half = a.d / 2;
  const long rows = (long)a.tokens * heads;
  for (long row = (long)blockIdx.x * kHeadWaves + (threadIdx.x >> 6); row < rows; row += (long)gridDim.x * kHeadWaves) {
    const long t = row / heads;
    const int h = (int)(row % heads);
    const bool is_q = h < a.hq;
    const int hh = is_q ? h : h - a.hq;
    const T* x = is_q ? (const T*)a.q + t * a.q_stride + (long)hh * a.d : (const T*)a.k + t * a.k_stride + (long)hh * a.d;
    T* y = is_q ? (T*)a.yq + (t * a.hq + hh) * a.d : (T*)a.yk + (t * a.hkv + hh) * a.d;
    const T* g = (const T*)(is_q ? a.gain_q : a.gain_k);
    float u[kMaxPairs], v[kMaxPairs], ss = 0.f;
#pragma unroll
    for (int c = 0; c < kMaxPairs; ++c) {
      const int j = lane + 64 * c;
      u[c] = j < half ? to_f32(x[j]) : 0.f;
      v[c] = j < half ? to_f32(x[j + half]) : 0.f;
      ss = fmaf(u[c], u[c], fmaf(v[c], v[c], ss));
    }
    const float r = rsqrtf(wave_sum(ss) / (float)a.d + a.eps);
    const double pos = head_pos(a, t);
#pragma unroll
    for (int c = 0; c < kMaxPairs; ++c) {
      const int j = lane + 64 * c;
      if (j < half) {
        const float2 w = head_angle(pos, j, a);
        const float p = u[c] * r * to_f32(g[j]), q = v[c] * r * to_f32(g[j + half]);
        y[j] = from_f32<T>(p * w.x - q * w.y);
        y[j + half] = from_f32<T>(q * w.x + p * w.y);
      }
    }
  }
}

// Waves take rows in turn; a lane's gain gradients of its pairs stay in
// registers and the workgroup's sum goes to part[block][q or k][d].
template <typename T>
__global__ __launch_bounds__(kHeadThreads) void head_norm_rope_bwd_kernel(HeadArgs a) {
  __shared__ float red[kHeadWaves][2][2 * kMaxPairs * 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, heads = a.hq + a.hkv, half = a.d / 2;
  const long rows = (long)a.tokens * heads;
  float dg[2][2 * kMaxPairs] = {};
  for (long row = (long)blockIdx.x * kHeadWaves + w; row < rows; row += (long)gridDim.x * kHeadWaves) {
    const long t = row / heads;
    const int h = (int)(row % heads);
    const bool is_q = h < a.hq;
    const int hh = is_q ? h : h - a.hq;
    const T* x =
        is_q ? (const T*)a.q + t * a.q_stride + (long)hh * a.d : (const T*)a.k + t * a.k_stride + (long)hh * a.d;
    const T* dy = is_q ? (const T*)a.dyq + (t * a.hq + hh) * a.d : (const T*)a.dyk + (t * a.hkv + hh) * a.d;
    T* dx = is_q ? (T*)a.dq + t * a.dq_stride + (long)hh * a.d : (T*)a.dk + t * a.dk_stride + (long)hh * a.d;
    const T* g = (const T*)(is_q ? a.gain_q : a.gain_k);
    const double pos = head_pos(a, t);
    float xv[2 * kMaxPairs], dz[2 * kMaxPairs], gz[2 * kMaxPairs], ss = 0.f, dot = 0.f;
#pragma unroll
    for (int c = 0; c < kMaxPairs; ++c) {
      const int j = lane + 64 * c, i = 2 * c;
      xv[i] = xv[i + 1] = dz[i] = dz[i + 1] = gz[i] = gz[i + 1] = 0.f;
      if (j < half) {
        xv[i] = to_f32(x[j]);
        xv[i + 1] = to_f32(x[j + half]);
        const float2 cs = head_angle(pos, j, a);
        const float p = to_f32(dy[j]), q = to_f32(dy[j + half]);
        dz[i] = p * cs.x + q * cs.y;
        dz[i + 1] = q * cs.x - p * cs.y;
        gz[i] = dz[i] * to_f32(g[j]);
        gz[i + 1] = dz[i + 1] * to_f32(g[j + half]);
      }
#pragma unroll
      for (int b = i; b < i + 2; ++b) {
        ss = fmaf(xv[b], xv[b], ss);
        dot = fmaf(gz[b], xv[b], dot);
      }
    }
    const float r = rsqrtf(wave_sum(ss) / (float)a.d + a.eps);
    const float k3 = r * (r * (r * (wave_sum(dot) / (float)a.d)));  // r^3 alone can pass the range
#pragma unroll
    for (int c = 0; c < kMaxPairs; ++c) {
      const int j = lane + 64 * c, i = 2 * c;
      if (j < half) {
        dx[j] = from_f32<T>(r * gz[i] - k3 * xv[i]);
        dx[j + half] = from_f32<T>(r * gz[i + 1] - k3 * xv[i + 1]);
      }
#pragma unroll
      for (int b = i; b < i + 2; ++b) {
        const float add = dz[b] * xv[b] * r;
        dg[0][b] += is_q ? add : 0.f;
        dg[1][b] += is_q ? 0.f : add;
      }
    }
  }
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int b = 0; b < 2 * kMaxPairs; ++b) red[w][s][b * 64 + lane] = dg[s][b];
  __syncthreads();
  // value b * 64 + lane of red is column lane + 64 (b / 2) (+ d/2 for odd b)
  for (int i = threadIdx.x; i < 2 * a.d; i += kHeadThreads) {
    const int s = i / a.d, col = i % a.d, j = col % half;
    const int at = (2 * (j / 64) + (col >= half)) * 64 + j % 64;
    float sum = 0.f;
    for (int q = 0; q < kHeadWaves; ++q) sum += red[q][s][at];
    a.part[(long)blockIdx.x * 2 * a.d + i] = sum;
  }
}

// ------------------------------------------------ rows of 16-byte chunks
// Head dims that are a multiple of 16, with 16-byte rows: a wave takes a token
// at a time (or a share of its heads, where there are few tokens).  A head's row
// is held by G lanes (a power of two, d / 16 of them used), eight values of
// either half each, so that a pair's two values meet in one lane; the row's sums
// take log2 G shuffles.  The token's angles are formed once, one pair a lane,
// and shared by its heads through LDS; the frequencies once a wave.  The next
// rows are loaded before the present ones are worked on.
// HBM bound: 8192 tokens x 36 heads x 128 forward 28.5 us (5.3 TB/s; one wave a
// row 117 us), 18474 tokens backward 108 us (4.5 TB/s; 315 us).
namespace {
template <typename T>
struct Chunk;
template <>
struct Chunk<bf16> {
  bf16x8 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *(const bf16x8*)p; }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (bf16)0.f;
  }
  __device__ __forceinline__ float at(int j) const { return (float)v[j]; }
  static __device__ __forceinline__ void store(bf16* p, const float (&x)[8]) {
    bf16x8 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = (bf16)x[j];
    *(bf16x8*)p = o;
  }
};
template <>
struct Chunk<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = ((const f32x4*)p)[0];
    b = ((const f32x4*)p)[1];
  }
  __device__ __forceinline__ void zero() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float at(int j) const { return j < 4 ? a[j] : b[j - 4]; }
  static __device__ __forceinline__ void store(float* p, const float (&x)[8]) {
    ((f32x4*)p)[0] = f32x4{x[0], x[1], x[2], x[3]};
    ((f32x4*)p)[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
};

template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// A lane's place in its wave's rows and what it needs of every token.
template <typename T, int G>
struct RowLane {
  static constexpr int kHeads = 64 / G;  // heads a wave holds at once
  int lane, c, col, half;                // chunk of either half, its first column
  bool used;
  double turns[kMaxPairs];               // of the pairs lane and lane + 64, per position
  float cs[8], sn[8];
  __device__ __forceinline__ RowLane(const HeadArgs& a) {
    lane = threadIdx.x & 63;
    c = lane % G;
    col = 8 * c;
    half = a.d / 2;
    used = col < half;
#pragma unroll
    for (int q = 0; q < kMaxPairs; ++q) turns[q] = exp2((double)(lane + 64 * q) * a.log2_step) * (0.5 / M_PI);
  }
  // the angles of token t, through the wave's own LDS
  __device__ __forceinline__ void angles(const HeadArgs& a, long t, float2* shared) {
    const double pos = head_pos(a, t);
    __builtin_amdgcn_wave_barrier();  // the last token's have been read
#pragma unroll
    for (int q = 0; q < kMaxPairs; ++q) {
      if (64 * q < half) {
        const double n = pos * turns[q];
        float s, k;
        sincospif((float)(2.0 * (n - rint(n))), &s, &k);
        if (lane + 64 * q < half) shared[lane + 64 * q] = make_float2(k, s);
      }
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 v = shared[used ? col + j : 0];
      cs[j] = v.x;
      sn[j] = v.y;
    }
  }
};

// both halves' chunks of a row
template <typename T>
struct Pair {
  Chunk<T> lo, hi;
  __device__ __forceinline__ void load(const T* row, int col, int half, bool used) {
    lo.zero();
    hi.zero();
    if (used) {
      lo.load(row + col);
      hi.load(row + col + half);
    }
  }
};

// A token's heads in rounds of 64 / G, q's before k's; a unit is a token's share
// [part * per, ..) of them.  A wave's units lie `stride` apart, and it walks
// their rounds as one sequence.
struct Cursor {
  long u;
  int r;
};
template <int G>
struct Walk {
  int nq, n, per, parts;
  long units, stride;
  __device__ __forceinline__ Walk(const HeadArgs& a, int parts_) {
    constexpr int H = 64 / G;
    nq = (a.hq + H - 1) / H;
    n = nq + (a.hkv + H - 1) / H;
    parts = parts_;
    per = (n + parts - 1) / parts;
    units = (long)a.tokens * parts;
    stride = (long)gridDim.x * kHeadWaves;
  }
  __device__ __forceinline__ int lo(long u) const { return (int)(u % parts) * per; }
  __device__ __forceinline__ bool ends(const Cursor& c) const { return c.u >= units; }
  __device__ __forceinline__ Cursor after(const Cursor& c) const {
    if (c.r + 1 < min(lo(c.u) + per, n)) return {c.u, c.r + 1};
    return {c.u + stride, lo(c.u + stride)};
  }
};
// the rows of a cursor's round: heads of q or of k
struct Round {
  bool is_q;
  long t;
  int first, heads;
};
template <int G>
__device__ __forceinline__ Round round_at(const HeadArgs& a, const Walk<G>& w, const Cursor& c) {
  const bool is_q = c.r < w.nq;
  return {is_q, c.u / w.parts, (is_q ? c.r : c.r - w.nq) * (64 / G), is_q ? a.hq : a.hkv};
}
}  // namespace

template <typename T, int G>
__global__ __launch_bounds__(kHeadThreads) void head_rows_fwd_kernel(HeadArgs a, int parts) {
  __shared__ float2 shared[kHeadWaves][64 * kMaxPairs];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Walk<G> walk(a, parts);
  Cursor cur = {(long)blockIdx.x * kHeadWaves + w, 0};
  if (walk.ends(cur)) return;
  cur.r = walk.lo(cur.u);
  const int lane = threadIdx.x & 63, half = a.d / 2, col = lane % G * 8;
  auto fetch = [&](const Cursor& c, Pair<T>& x) {
    const Round r = round_at<G>(a, walk, c);
    const int h = r.first + lane / G;
    const T* token = r.is_q ? (const T*)a.q + r.t * a.q_stride : (const T*)a.k + r.t * a.k_stride;
    x.load(token + h * a.d, col, half, col < half && h < r.heads);
  };
  Pair<T> x, ahead, gq, gk;
  fetch(cur, x);
  gq.load((const T*)a.gain_q, col, half, col < half);
  gk.load((const T*)a.gain_k, col, half, col < half);
  RowLane<T, G> l(a);
  for (bool begins = true;;) {
    const Cursor next = walk.after(cur);
    const bool more = !walk.ends(next);
    if (more) fetch(next, ahead);
    const Round r = round_at<G>(a, walk, cur);
    if (begins) l.angles(a, r.t, shared[w]);
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(x.lo.at(j), x.lo.at(j), fmaf(x.hi.at(j), x.hi.at(j), ss));
    const float rs = rsqrtf(group_sum<G>(ss) / (float)a.d + a.eps);
    const int h = r.first + lane / G;
    if (col < half && h < r.heads) {
      const Pair<T>& g = r.is_q ? gq : gk;
      T* y = (r.is_q ? (T*)a.yq : (T*)a.yk) + (r.t * r.heads + h) * a.d + col;
      float p[8], q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u0 = x.lo.at(j) * rs * g.lo.at(j), u1 = x.hi.at(j) * rs * g.hi.at(j);
        p[j] = u0 * l.cs[j] - u1 * l.sn[j];
        q[j] = u1 * l.cs[j] + u0 * l.sn[j];
      }
      Chunk<T>::store(y, p);
      Chunk<T>::store(y + half, q);
    }
    if (!more) break;
    begins = next.u != cur.u;
    x = ahead;
    cur = next;
  }
}

template <typename T, int G>
__global__ __launch_bounds__(kHeadThreads) void head_rows_bwd_kernel(HeadArgs a, int parts) {
  __shared__ float2 shared[kHeadWaves][64 * kMaxPairs];
  __shared__ float red[kHeadWaves][2][2 * 64 * kMaxPairs];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Walk<G> walk(a, parts);
  Cursor cur = {(long)blockIdx.x * kHeadWaves + w, 0};
  cur.r = walk.lo(cur.u);
  const int lane = threadIdx.x & 63, half = a.d / 2, col = lane % G * 8;
  auto fetch = [&](const Cursor& c, Pair<T>& x, Pair<T>& y) {
    const Round r = round_at<G>(a, walk, c);
    const int h = r.first + lane / G;
    const bool used = col < half && h < r.heads;
    const T* token = r.is_q ? (const T*)a.q + r.t * a.q_stride : (const T*)a.k + r.t * a.k_stride;
    x.load(token + h * a.d, col, half, used);
    y.load((r.is_q ? (const T*)a.dyq : (const T*)a.dyk) + (r.t * r.heads + h) * a.d, col, half, used);
  };
  Pair<T> x, y, ahead_x, ahead_y, gq, gk;
  bool more = !walk.ends(cur);
  if (more) fetch(cur, x, y);
  gq.load((const T*)a.gain_q, col, half, col < half);
  gk.load((const T*)a.gain_k, col, half, col < half);
  RowLane<T, G> l(a);
  float dgq[16] = {}, dgk[16] = {};
  for (bool begins = true; more;) {
    const Cursor next = walk.after(cur);
    more = !walk.ends(next);
    if (more) fetch(next, ahead_x, ahead_y);
    const Round r = round_at<G>(a, walk, cur);
    if (begins) l.angles(a, r.t, shared[w]);
    const Pair<T>& g = r.is_q ? gq : gk;
    float ss = 0.f, dot = 0.f, d0[8], d1[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      d0[j] = y.lo.at(j) * l.cs[j] + y.hi.at(j) * l.sn[j];
      d1[j] = y.hi.at(j) * l.cs[j] - y.lo.at(j) * l.sn[j];
      ss = fmaf(x.lo.at(j), x.lo.at(j), fmaf(x.hi.at(j), x.hi.at(j), ss));
      dot = fmaf(d0[j] * g.lo.at(j), x.lo.at(j), fmaf(d1[j] * g.hi.at(j), x.hi.at(j), dot));
    }
    const float rs = rsqrtf(group_sum<G>(ss) / (float)a.d + a.eps);
    const float k3 = rs * (rs * (rs * (group_sum<G>(dot) / (float)a.d)));  // rs^3 alone can pass the range
    const int h = r.first + lane / G;
    if (col < half && h < r.heads) {
      T* dx = (r.is_q ? (T*)a.dq + r.t * a.dq_stride : (T*)a.dk + r.t * a.dk_stride) + h * a.d + col;
      float p[8], q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        p[j] = rs * (g.lo.at(j) * d0[j]) - k3 * x.lo.at(j);
        q[j] = rs * (g.hi.at(j) * d1[j]) - k3 * x.hi.at(j);
      }
      Chunk<T>::store(dx, p);
      Chunk<T>::store(dx + half, q);
      auto add = [&](float (&dg)[16]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          dg[j] = fmaf(d0[j] * x.lo.at(j), rs, dg[j]);
          dg[8 + j] = fmaf(d1[j] * x.hi.at(j), rs, dg[8 + j]);
        }
      };
      if (r.is_q)
        add(dgq);
      else
        add(dgk);
    }
    begins = next.u != cur.u;
    x = ahead_x;
    y = ahead_y;
    cur = next;
  }
  // gain gradients: over the wave's heads, then over the workgroup's waves
#pragma unroll
  for (int j = 0; j < 16; ++j) {
#pragma unroll
    for (int o = G; o < 64; o <<= 1) {
      dgq[j] += __shfl_xor(dgq[j], o);
      dgk[j] += __shfl_xor(dgk[j], o);
    }
    if (lane < G && col < half) {
      red[w][0][col + j % 8 + (j < 8 ? 0 : half)] = dgq[j];
      red[w][1][col + j % 8 + (j < 8 ? 0 : half)] = dgk[j];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.d; i += kHeadThreads) {
    float sum = 0.f;
    for (int q = 0; q < kHeadWaves; ++q) sum += red[q][i / a.d][i % a.d];
    a.part[(long)blockIdx.x * 2 * a.d + i] = sum;
  }
}

// dgain (+)= the sum of part over its blocks: 16 columns of the 2 d a workgroup,
// 64 interleaved slices of the blocks, added in a fixed order
__global__ __launch_bounds__(1024) void head_gain_sum_kernel(const float* __restrict__ part, int blocks, int d,
                                                             float* __restrict__ dgq, float* __restrict__ dgk,
                                                             int overwrite) {
  __shared__ float red[64][17];
  const int c = threadIdx.x & 15, s = threadIdx.x >> 4, i = blockIdx.x * 16 + c;
  float sum = 0.f;
  if (i < 2 * d)
#pragma unroll 8
    for (int b = s; b < blocks; b += 64) sum += part[(long)b * 2 * d + i];
  red[s][c] = sum;
  __syncthreads();
  for (int o = 32; o > 0; o >>= 1) {
    if (s < o) red[s][c] += red[s + o][c];
    __syncthreads();
  }
  if (s != 0 || i >= 2 * d) return;
  float* dst = i < d ? dgq + i : dgk + i - d;
  *dst = overwrite ? red[0][c] : *dst + red[0][c];
}

namespace {
// Workgroups of the backward, whose gain-gradient partials the workspace holds:
// four waves each, a row a wave at least, and as many as the chip holds at once
// by the row kernels' registers (167 a lane in bf16: three on each of 256 CUs;
// 203 in fp32: two), because all waves get the same work.  18474 tokens of 36
// heads x 128, us, at 512 / 768 / 1024 / 2048: bf16 109 / 108 / 121 / 110, fp32
// 200 / 219 / 200 / 204.
constexpr long kHeadBwdBlocks = 768;
long head_bwd_blocks(long rows) { return std::max(1L, std::min(kHeadBwdBlocks, (rows + kHeadWaves - 1) / kHeadWaves)); }

// 16-byte chunks everywhere: what the row kernels read and write as such
bool by_chunks(const HeadArgs& a, int es) {
  const uintptr_t bits = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.dq | (uintptr_t)a.dk |
                         (uintptr_t)a.gain_q | (uintptr_t)a.gain_k |
                         (uintptr_t)((a.q_stride | a.k_stride | a.dq_stride | a.dk_stride) * es);
  return a.d % 16 == 0 && bits % 16 == 0;
}
// lanes of a row: a power of two that holds d / 16 chunk pairs
int row_lanes(int d) {
  int g = 1;
  while (16 * g < d) g *= 2;
  return g;
}
// Shares of a token's heads: one while there are waves enough (four thousand,
// four a SIMD), else up to one per round of heads, so that a few tokens still
// use the chip.
int head_parts(const HeadArgs& a) {
  const int heads = 64 / row_lanes(a.d);
  const int rounds = (a.hq + heads - 1) / heads + (a.hkv + heads - 1) / heads;
  const long want = a.tokens > 0 ? 4096 / a.tokens : 1;
  const int parts = (int)std::max(1L, std::min((long)rounds, want)), per = (rounds + parts - 1) / parts;
  return (rounds + per - 1) / per;  // no empty share
}

// the instantiation for the head dim's lanes per row
template <typename T, bool BWD>
void launch_rows(const HeadArgs& a, unsigned blocks, int parts, hipStream_t st) {
#define SPR_ROWS(G)                                                                                              \
  case G:                                                                                                        \
    if (BWD)                                                                                                     \
      hipLaunchKernelGGL((head_rows_bwd_kernel<T, G>), dim3(blocks), dim3(kHeadThreads), 0, st, a, parts);       \
    else                                                                                                         \
      hipLaunchKernelGGL((head_rows_fwd_kernel<T, G>), dim3(blocks), dim3(kHeadThreads), 0, st, a, parts);       \
    break
  switch (row_lanes(a.d)) {
    SPR_ROWS(1);
    SPR_ROWS(2);
    SPR_ROWS(4);
    SPR_ROWS(8);
    SPR_ROWS(16);
  }
#undef SPR_ROWS
}
}  // namespace

size_t head_norm_rope_bwd_ws(long rows, int d) { return (size_t)head_bwd_blocks(rows) * 2 * d * 4; }

hipError_t launch_head_norm_rope_fwd(int dtype, const HeadArgs& a, hipStream_t st) {
  const long rows = (long)a.tokens * (a.hq + a.hkv);
  if (rows == 0) return hipSuccess;
  ProfileScope ps("head_norm_rope_fwd", st);
  if (by_chunks(a, dtype == 1 ? 2 : 4)) {
    const int parts = head_parts(a);
    const long units = (long)a.tokens * parts, blocks = std::min(1024L, (units + kHeadWaves - 1) / kHeadWaves);
    if (dtype == 1)
      launch_rows<bf16, false>(a, (unsigned)blocks, parts, st);
    else
      launch_rows<float, false>(a, (unsigned)blocks, parts, st);
    return hipGetLastError();
  }
  const dim3 grid(grid_of((rows + kHeadWaves - 1) / kHeadWaves, kHeadThreads));
  if (dtype == 1)
    hipLaunchKernelGGL(head_norm_rope_fwd_kernel<bf16>, grid, dim3(kHeadThreads), 0, st, a);
  else
    hipLaunchKernelGGL(head_norm_rope_fwd_kernel<float>, grid, dim3(kHeadThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_head_norm_rope_bwd(int dtype, const HeadArgs& a, float* dgain_q, float* dgain_k, bool overwrite,
                                     hipStream_t st) {
  const long rows = (long)a.tokens * (a.hq + a.hkv);
  if (rows == 0 && !overwrite) return hipSuccess;
  long blocks = rows > 0 ? head_bwd_blocks(rows) : 0;  // no tokens: the gains' gradient is zero
  if (rows > 0) {
    ProfileScope ps("head_norm_rope_bwd", st);
    if (by_chunks(a, dtype == 1 ? 2 : 4)) {
      const int parts = head_parts(a);
      // never more waves than units: an idle wave's partial would be read for nothing
      blocks = std::max(1L, std::min(blocks, ((long)a.tokens * parts + kHeadWaves - 1) / kHeadWaves));
      if (dtype != 1) blocks = std::min(blocks, 512L);
      if (dtype == 1)
        launch_rows<bf16, true>(a, (unsigned)blocks, parts, st);
      else
        launch_rows<float, true>(a, (unsigned)blocks, parts, st);
    } else if (dtype == 1) {
      hipLaunchKernelGGL(head_norm_rope_bwd_kernel<bf16>, dim3((unsigned)blocks), dim3(kHeadThreads), 0, st, a);
    } else {
      hipLaunchKernelGGL(head_norm_rope_bwd_kernel<float>, dim3((unsigned)blocks), dim3(kHeadThreads), 0, st, a);
    }
  }
  ProfileScope ps("head_gain_sum", st);
  hipLaunchKernelGGL(head_gain_sum_kernel, dim3((2 * a.d + 15) / 16), dim3(1024), 0, st, a.part, (int)blocks, a.d,
                     dgain_q, dgain_k, overwrite ? 1 : 0);
  return hipGetLastError();
}

}  // namespace spr
