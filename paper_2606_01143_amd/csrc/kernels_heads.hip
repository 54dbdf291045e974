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

// One wave per row; lane l has the pairs l and l + 64.
template <typename T>
__global__ __launch_bounds__(kHeadThreads) void head_norm_rope_fwd_kernel(HeadArgs a) {
  const int lane = threadIdx.x & 63, heads = a.hq + a.hkv, half = a.d / 2;
  const long row = (long)blockIdx.x * kHeadWaves + (threadIdx.x >> 6);
  if (row >= (long)a.tokens * heads) return;
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
    const float k3 = r * r * r * (wave_sum(dot) / (float)a.d);
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

// dgain (+)= the sum of part over its blocks, in block order within sixteen
// interleaved slices; 64 columns of the 2 d per workgroup
__global__ __launch_bounds__(1024) void head_gain_sum_kernel(const float* __restrict__ part, int blocks, int d,
                                                             float* __restrict__ dgq, float* __restrict__ dgk,
                                                             int overwrite) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
  float sum = 0.f;
  if (i < 2 * d)
    for (int b = w; b < blocks; b += 16) sum += part[(long)b * 2 * d + i];
  red[w][lane] = sum;
  __syncthreads();
  if (w != 0 || i >= 2 * d) return;
  sum = 0.f;
  for (int q = 0; q < 16; ++q) sum += red[q][lane];
  float* dst = i < d ? dgq + i : dgk + i - d;
  *dst = overwrite ? sum : *dst + sum;
}

namespace {
// workgroups of the backward: four waves each, a row a wave at least, and
// enough of them to fill the chip eight waves deep per SIMD
constexpr long kHeadBwdBlocks = 2048;
long head_bwd_blocks(long rows) { return std::max(1L, std::min(kHeadBwdBlocks, (rows + kHeadWaves - 1) / kHeadWaves)); }
}  // namespace

size_t head_norm_rope_bwd_ws(long rows, int d) { return (size_t)head_bwd_blocks(rows) * 2 * d * 4; }

hipError_t launch_head_norm_rope_fwd(int dtype, const HeadArgs& a, hipStream_t st) {
  const long rows = (long)a.tokens * (a.hq + a.hkv);
  if (rows == 0) return hipSuccess;
  ProfileScope ps("head_norm_rope_fwd", st);
  const dim3 grid((unsigned)((rows + kHeadWaves - 1) / kHeadWaves));
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
  const unsigned blocks = (unsigned)head_bwd_blocks(rows);
  {
    ProfileScope ps("head_norm_rope_bwd", st);
    if (dtype == 1)
      hipLaunchKernelGGL(head_norm_rope_bwd_kernel<bf16>, dim3(blocks), dim3(kHeadThreads), 0, st, a);
    else
      hipLaunchKernelGGL(head_norm_rope_bwd_kernel<float>, dim3(blocks), dim3(kHeadThreads), 0, st, a);
  }
  ProfileScope ps("head_gain_sum", st);
  hipLaunchKernelGGL(head_gain_sum_kernel, dim3((2 * a.d + 63) / 64), dim3(1024), 0, st, a.part, (int)blocks, a.d,
                     dgain_q, dgain_k, overwrite ? 1 : 0);
  return hipGetLastError();
}

}  // namespace spr
