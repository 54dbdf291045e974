// The norms around a block of a decoder layer, the block's gate and the scaled
// residual in one pass, and activations kept in 8 bits.
//   p = f r_f g_post,  h = a x + b gate p,  n = h r_h g_pre
// Both directions read each tensor once and write each once: HBM bound.  A row
// stays in its threads' registers between its sums and its outputs, eight values a
// thread (two chunks of eight past 8192 columns).  The forward has a row a workgroup;
// a workgroup of the backward holds as many rows at once as fill 512 threads.
// Measured, 28672 rows of 4096 bf16: residual, norm and an 8-bit copy 184 us (5.8
// TB/s); norms on both sides and a gate 181 us, backward 277 us (5.1 TB/s); 2048
// columns from 8 bits, 17543 rows, backward 80-85 us (4.4 TB/s; half its
// instructions turn bytes into fp32) and 5 us for the columns' sums.
// 1024 threads leave a thread 128 registers, and the backward's column sums spill some
// there: 34 of fp32 rows from 4104 columns (4096 rows of 8192: 189 us where the bytes
// take 164), 103 of fp32 and 6 of bf16 rows past 8192 columns (4096 rows of 8200: 396 and
// 129 us, 164 and 82).
#include "act8.hpp"
#include "launch.hpp"

namespace spr {

namespace {

// eight consecutive values of a row as loaded: T, or 8 bits and their exponent
// (forget(): what was formed of it is formed again, not kept in registers)
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16> : Act8Chunk {
  __device__ __forceinline__ void zero() { raw = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(raw)); }
  __device__ __forceinline__ void load(const void* p, size_t at) { Act8Chunk::load(p, nullptr, at, 0, false); }
  __device__ __forceinline__ void load(const void* p, const uint8_t* e, size_t at, size_t block) {
    Act8Chunk::load(p, e, at, block, e != nullptr);
  }
};
template <>
struct Raw8<float> {
  u32x4 a, b;
  __device__ __forceinline__ void zero() { a = b = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(a), "+v"(b)); }
  __device__ __forceinline__ void load(const void* p, size_t at) {
    a = ((const u32x4*)((const float*)p + at))[0];
    b = ((const u32x4*)((const float*)p + at))[1];
  }
  __device__ __forceinline__ void load(const void* p, const uint8_t* e, size_t at, size_t block) {
    if (e == nullptr) return load(p, at);
    Act8Chunk c;
    c.load(p, e, at, block, true);
    a = c.raw;
  }
  __device__ __forceinline__ void values(float (&v)[8], bool small) const {
    if (small) {
      Act8Chunk c;
      c.raw = a;
      c.values(v, true);
      return;
    }
    const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
  }
};

__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) { store_bf16x8(p, v); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  ((f32x4*)p)[0] = f32x4{v[0], v[1], v[2], v[3]};
  ((f32x4*)p)[1] = f32x4{v[4], v[5], v[6], v[7]};
}

// over a wave: rows of 16 lanes in registers, the four rows through scalars
__device__ __forceinline__ float wave_total(float v) {
  v += __uint_as_float(dpp<kXor1>(__float_as_uint(v)));
  v += __uint_as_float(dpp<kXor2>(__float_as_uint(v)));
  v += __uint_as_float(dpp<kHalfMirror>(__float_as_uint(v)));
  v += __uint_as_float(dpp<kMirror>(__float_as_uint(v)));
  const int b = (int)__float_as_uint(v);
  auto of = [&](int lane) { return __uint_as_float((unsigned)__builtin_amdgcn_readlane(b, lane)); };
  return (of(0) + of(16)) + (of(32) + of(48));
}
// Sums over a row's workgroup.  The buffers alternate: a wave writes one again
// only behind the barrier that follows its last reads, so each sum takes one.
template <int TPR, int N, int ROWS = 1>
struct RowSums {
  float (*buf)[ROWS * TPR / 64][N];
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_total(v[i]);
    if constexpr (TPR > 64) {
      const int w = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[turn][w][i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < TPR / 64; ++q) s += buf[turn][(ROWS > 1 ? w / (TPR / 64) * (TPR / 64) : 0) + q][i];
        v[i] = s;
      }
      turn ^= 1;
    }
  }
};

// a thread's eight values to 8 bits; every lane of its quad takes part
__device__ __forceinline__ void pack8(const float (&v)[8], bool inside, void* q, uint8_t* e, size_t at, size_t block,
                                      bool first) {
  unsigned most = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) most = max(most, magnitude(v[j]));
  const Act8Scale s = act8_scale(quad_max(inside ? most : 0u));
  if (!inside) return;
  *(u32x2*)((char*)q + at) = u32x2{act8_quad(v[0], v[1], v[2], v[3], s), act8_quad(v[4], v[5], v[6], v[7], s)};
  if (first) e[block] = (uint8_t)s.exponent;
}
}  // namespace

// ---------------------------------------------------------- block norm
// Forward: a row a workgroup of TPR threads, CH chunks of eight values a thread.
template <typename T, int TPR, int CH>
__global__ __launch_bounds__(TPR) void block_norm_fwd_kernel(BlockNormArgs a) {
  __shared__ float buf[2][TPR / 64][1];
  RowSums<TPR, 1> sum{buf};
  const int chunks = a.width / 8, blocks = (a.width + 31) / 32;
  for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const size_t at = (size_t)row * a.width, block = (size_t)row * blocks;
    Raw8<T> x[CH], f[CH], gate[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int ch = threadIdx.x + c * TPR;
      x[c].zero();
      f[c].zero();
      gate[c].zero();
      if (ch < chunks) {
        x[c].load(a.x, at + 8 * ch);
        if (a.f != nullptr) f[c].load(a.f, at + 8 * ch);
        if (a.gate != nullptr) gate[c].load(a.gate, (size_t)row * a.gate_stride + 8 * ch);
      }
    }
    float h[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) x[c].values(h[c], false);
    if (a.f != nullptr) {
      float r = 1.f;
      if (a.rstd_f != nullptr) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float v[8];
          f[c].values(v, false);
#pragma unroll
          for (int j = 0; j < 8; ++j) s[0] = fmaf(v[j], v[j], s[0]);
        }
        sum(s);
        r = rsqrtf(s[0] / (float)a.width + a.eps);
        if (threadIdx.x == 0) a.rstd_f[row] = r;
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int ch = threadIdx.x + c * TPR;
        float v[8], g[8];
        f[c].values(v, false);
        if (a.f8 != nullptr) pack8(v, ch < chunks, a.f8, a.f_e, at + 8 * ch, block + ch / 4, ch % 4 == 0);
        if (a.rstd_f != nullptr) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= r;
          if (a.gain_post != nullptr && ch < chunks) {
            Raw8<T> gain;
            gain.load(a.gain_post, 8 * ch);
            gain.values(g, false);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= g[j];
          }
        }
        if (a.gate != nullptr) {
          gate[c].values(g, false);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= g[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) h[c][j] = fmaf(a.branch_scale, v[j], a.residual_scale * h[c][j]);
        if (ch < chunks) store8((T*)a.h + at + 8 * ch, h[c]);
      }
    }
    if (a.rstd_h != nullptr) {
      float s[1] = {0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] = fmaf(h[c][j], h[c][j], s[0]);
      sum(s);
      const float r = rsqrtf(s[0] / (float)a.width + a.eps);
      if (threadIdx.x == 0) a.rstd_h[row] = r;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int ch = threadIdx.x + c * TPR;
        if (ch < chunks) {
          float v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = h[c][j] * r;
          if (a.gain_pre != nullptr) {
            float g[8];
            Raw8<T> gain;
            gain.load(a.gain_pre, 8 * ch);
            gain.values(g, false);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= g[j];
          }
          store8((T*)a.n + at + 8 * ch, v);
        }
      }
    }
    if (a.h8 != nullptr)
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int ch = threadIdx.x + c * TPR;
        pack8(h[c], ch < chunks, a.h8, a.h_e, at + 8 * ch, block + ch / 4, ch % 4 == 0);
      }
  }
}

__host__ __device__ __forceinline__ bool needs_sums(const BlockNormArgs& a) {
  return a.dgain_pre != nullptr || a.dgain_post != nullptr || (a.dgate != nullptr && a.gate_stride == 0);
}

// Column `col` of the sum S0 = sum dn h r_h (which 0) or S1 (1) to where it goes.
// Without a token's own gates, S1 = sum d f r_f gives both dg_post = b gate S1 and
// dgate = b g_post S1; with them, S1 = sum gate d f r_f.
template <typename T>
__device__ __forceinline__ void block_norm_column(const BlockNormArgs& a, int which, int col, float s) {
  auto put = [&](float* dst, float v) { *dst = a.overwrite ? v : *dst + v; };
  if (which == 0) {
    if (a.dgain_pre != nullptr) put(a.dgain_pre + col, s);
    return;
  }
  s *= a.branch_scale;
  const bool channel = a.gate != nullptr && a.gate_stride == 0;
  if (a.dgain_post != nullptr) put(a.dgain_post + col, channel ? s * to_f32(((const T*)a.gate)[col]) : s);
  if (channel && a.dgate != nullptr)
    put((float*)a.dgate + col, a.gain_post != nullptr ? s * to_f32(((const T*)a.gain_post)[col]) : s);
}

// Backward.  With d = dh + r_h g_pre dn - k h, k = r_h^3 mean(g_pre dn h), and
// w = b gate g_post, the second norm's mean needs sum(w f d) = sum(w f (dh +
// r_h g_pre dn)) - k sum(w f h): the row's three sums take one reduction.  A
// workgroup holds ROWS rows at once; the columns' sums stay in its threads'
// registers, are joined in the order of the rows, one partial row a workgroup,
// and a second launch adds those in order (a single workgroup's are the sums).
template <typename T, int TPR, int CH, int ROWS>
__global__ __launch_bounds__(TPR* ROWS) void block_norm_bwd_kernel(BlockNormArgs a) {
  __shared__ float buf[2][ROWS * TPR / 64][3];
  constexpr bool IN_LDS = CH > 1;  // the columns' sums of two chunks do not fit the registers
  static_assert(!IN_LDS || ROWS == 1, "sums in LDS are of one row at a time");
  __shared__ f32x4 joined[ROWS > 1 || IN_LDS ? 4 * CH * TPR : 1];
  RowSums<TPR, 3, ROWS> sum{buf};
  // (a wave's row is one group's: its place in memory stays in scalar registers)
  const int thread = threadIdx.x % TPR, group = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  const int chunks = a.width / 8, blocks = (a.width + 31) / 32;
  const bool pre = a.dn != nullptr, post = a.rstd_f != nullptr, branch = a.f != nullptr, sums = needs_sums(a);
  const bool h8 = a.h_e != nullptr, f8 = a.f_e != nullptr, token_gate = a.gate_stride != 0;
  float sum_pre[CH][8], sum_post[CH][8];
  Raw8<T> gain_pre[CH], gain_post[CH], gate[CH];
  auto gains = [&](int c) {
    const int ch = thread + c * TPR;
    gain_pre[c].zero();
    gain_post[c].zero();
    if (!token_gate) gate[c].zero();
    if (ch < chunks) {
      if (a.gain_pre != nullptr) gain_pre[c].load(a.gain_pre, 8 * ch);
      if (a.gain_post != nullptr) gain_post[c].load(a.gain_post, 8 * ch);
      if (a.gate != nullptr && !token_gate) gate[c].load(a.gate, 8 * ch);
    }
  };
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    gate[c].zero();
    gains(c);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum_pre[c][j] = sum_post[c][j] = 0.f;
    if constexpr (IN_LDS)
#pragma unroll
      for (int j = 0; j < 4; ++j) joined[(4 * c + j) * TPR + thread] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // (a thread's own places: no other reads or writes them)
  auto in_lds = [&](int c, int which, float (&v)[8], bool store) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f32x4& p = joined[(4 * c + 2 * which + j) * TPR + thread];
      if (store)
        p = f32x4{v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
      else
        for (int i = 0; i < 4; ++i) v[4 * j + i] = p[i];
    }
  };
  auto of = [](const Raw8<T>& r, bool is, float (&v)[8]) {
    if (is)
      r.values(v, false);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 1.f;
  };
  for (long row0 = (long)blockIdx.x * ROWS; row0 < a.rows; row0 += (long)gridDim.x * ROWS) {
    const long row = row0 + group;
    // An empty place of the last turn holds zeros: times an infinite gain, or the
    // infinite gate of its row before, they are NaNs, which no sum may take.  (A
    // branch around what is behind the sums costs 4 us of 85 at 17543 rows of 2048
    // from 8 bits, this select none.)
    const bool real = ROWS == 1 || row < a.rows;
    const int chunks = row < a.rows ? a.width / 8 : 0;  // of this group's row
    const size_t at = (size_t)row * a.width, block = (size_t)row * blocks;
    Raw8<T> h[CH], f[CH], dh[CH], dn[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int ch = thread + c * TPR;
      h[c].zero();
      f[c].zero();
      dh[c].zero();
      dn[c].zero();
      if (ch < chunks) {
        if (pre) h[c].load(a.h, a.h_e, at + 8 * ch, block + ch / 4);
        if (pre) dn[c].load(a.dn, at + 8 * ch);
        if (a.dh != nullptr) dh[c].load(a.dh, at + 8 * ch);
        if (branch) f[c].load(a.f, a.f_e, at + 8 * ch, block + ch / 4);
        if (token_gate) gate[c].load(a.gate, (size_t)row * a.gate_stride + 8 * ch);
      }
    }
    const float rh = pre && chunks > 0 ? a.rstd_h[row] : 0.f, rf = post && chunks > 0 ? a.rstd_f[row] : post ? 0.f : 1.f;
    float s[3] = {0.f, 0.f, 0.f};
    if (pre || post) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float hv[8], fv[8], d[8], up[8], g[8];
        if constexpr (CH > 1) gains(c);  // two chunks' gains do not stay in registers
        h[c].values(hv, h8);
        dn[c].values(d, false);
        of(gain_pre[c], pre && a.gain_pre != nullptr, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          d[j] *= g[j];
          s[0] = fmaf(d[j], hv[j], s[0]);
        }
        if (post) {
          dh[c].values(up, false);
          f[c].values(fv, f8);
          of(gain_post[c], a.gain_post != nullptr, g);
#pragma unroll
          for (int j = 0; j < 8; ++j) fv[j] *= g[j];
          if (a.gate != nullptr) {
            gate[c].values(g, false);
#pragma unroll
            for (int j = 0; j < 8; ++j) fv[j] *= g[j];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            s[1] = fmaf(fv[j], fmaf(rh, d[j], up[j]), s[1]);
            s[2] = fmaf(fv[j], hv[j], s[2]);
          }
        }
        if constexpr (CH > 1) __builtin_amdgcn_sched_barrier(0);  // a chunk at a time: both would spill
      }
      sum(s);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      h[c].forget();
      f[c].forget();
      dh[c].forget();
      dn[c].forget();
      if constexpr (CH == 1) {
        gain_pre[c].forget();
        gain_post[c].forget();
      }
      if (CH == 1 || token_gate) gate[c].forget();
    }
    const float k = rh * (rh * (rh * (s[0] / (float)a.width)));
    const float kf = rf * (rf * (rf * (a.branch_scale * (s[1] - k * s[2]) / (float)a.width)));
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int ch = thread + c * TPR;
      float hv[8], d[8], g[8], o[8];
      if constexpr (CH > 1) gains(c);
      if constexpr (IN_LDS) in_lds(c, 0, sum_pre[c], false);
      h[c].values(hv, h8);
      dn[c].values(d, false);
      dh[c].values(o, false);
      of(gain_pre[c], pre && a.gain_pre != nullptr, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float dr = d[j] * rh;
        sum_pre[c][j] = fmaf(dr, hv[j], sum_pre[c][j]);
        d[j] = fmaf(dr, g[j], fmaf(-k, hv[j], o[j]));
        o[j] = a.residual_scale * d[j];
      }
      if constexpr (IN_LDS) {
        in_lds(c, 0, sum_pre[c], true);
        in_lds(c, 1, sum_post[c], false);
      }
      if (ch < chunks) store8((T*)a.dx + at + 8 * ch, o);
      float fv[8], gp[8];
      f[c].values(fv, f8);
      of(gate[c], a.gate != nullptr, g);
      of(gain_post[c], a.gain_post != nullptr, gp);
      if (token_gate && a.dgate != nullptr && ch < chunks) {
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = a.branch_scale * (d[j] * (fv[j] * rf) * gp[j]);
        store8((T*)a.dgate + at + 8 * ch, o);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float t = !real ? 0.f : token_gate ? d[j] * g[j] : d[j];
        sum_post[c][j] = fmaf(t, fv[j] * rf, sum_post[c][j]);
        d[j] *= a.branch_scale * g[j];
        o[j] = post ? fmaf(rf * gp[j], d[j], -(kf * fv[j])) : d[j];
      }
      if constexpr (IN_LDS) in_lds(c, 1, sum_post[c], true);
      if (a.df != nullptr && ch < chunks) store8((T*)a.df + at + 8 * ch, o);
      if constexpr (CH > 1) __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (!sums) return;
  if constexpr (ROWS > 1) {
    for (int q = 1; q < ROWS; ++q) {
      auto each4 = [&](auto f) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            f(joined[(4 * c + j) * TPR + thread], sum_pre[c] + 4 * j);
            f(joined[(4 * c + 2 + j) * TPR + thread], sum_post[c] + 4 * j);
          }
      };
      if (group == q) each4([](f32x4& d, const float* v) { d = f32x4{v[0], v[1], v[2], v[3]}; });
      __syncthreads();
      if (group == 0)
        each4([](f32x4& d, float* v) {
          for (int j = 0; j < 4; ++j) v[j] += d[j];
        });
      __syncthreads();
    }
    if (group > 0) return;
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int ch = thread + c * TPR;
    if constexpr (IN_LDS) {
      in_lds(c, 0, sum_pre[c], false);
      in_lds(c, 1, sum_post[c], false);
    }
    if (ch >= chunks) continue;
    if (gridDim.x == 1) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        block_norm_column<T>(a, 0, 8 * ch + j, sum_pre[c][j]);
        block_norm_column<T>(a, 1, 8 * ch + j, sum_post[c][j]);
      }
    } else {
      store8(a.part + ((size_t)blockIdx.x * 2) * a.width + 8 * ch, sum_pre[c]);
      store8(a.part + ((size_t)blockIdx.x * 2 + 1) * a.width + 8 * ch, sum_post[c]);
    }
  }
}

// The partial rows' sums: 32 columns a workgroup, 32 half waves each every 32nd
// row, joined in order.
template <typename T>
__global__ __launch_bounds__(1024) void block_norm_sums_kernel(BlockNormArgs a, int parts) {
  __shared__ float red[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + lane, which = blockIdx.y;
  float s = 0.f;
  if (col < a.width)
#pragma unroll 8
    for (int p = w; p < parts; p += 32) s += a.part[((size_t)p * 2 + which) * a.width + col];
  red[w][lane] = s;
  __syncthreads();
  if (w != 0 || col >= a.width) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < 32; ++q) s += red[q][lane];
  block_norm_column<T>(a, which, col, s);
}

namespace {

// f<TPR, CH> of the least threads that hold a row in one chunk each, or 1024 of two
template <typename F>
hipError_t by_width(int width, F f) {
  const int chunks = width / 8;
  if (chunks <= 64) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  if (chunks <= 128) return f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
  if (chunks <= 256) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  if (chunks <= 512) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
  if (chunks <= 1024) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
  return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}
}  // namespace

// Rows that a workgroup of the backward holds at once, and workgroups: 16 waves a
// CU in any width, in as few workgroups as hold 512 threads, since each has a
// partial row of column sums.
constexpr int bwd_rows(int tpr) { return tpr < 512 ? 512 / tpr : 1; }
static int bwd_groups(int rows, int width) {
  int groups = 0;
  by_width(width, [&](auto tpr, auto) {
    const long held = bwd_rows(tpr), all = (rows + held - 1) / held, most = tpr > 512 ? 256 : 512;
    groups = (int)(all < most ? all : most);
    return hipSuccess;
  });
  return groups;
}
// partial rows: up to four rounds of one workgroup take less than a second launch
static int bwd_parts(int rows, int width) {
  const int groups = bwd_groups(rows, width);
  return groups <= 4 ? (groups < 1 ? groups : 1) : groups;
}
size_t block_norm_bwd_ws(int rows, int width) {
  const int parts = bwd_parts(rows, width);
  return parts > 1 ? (size_t)parts * 2 * width * 4 : 0;
}

template <typename T>
static hipError_t block_norm_fwd_of(const BlockNormArgs& a, hipStream_t st) {
  return by_width(a.width, [&](auto tpr, auto ch) {
    hipLaunchKernelGGL((block_norm_fwd_kernel<T, tpr, ch>), dim3(grid_of(a.rows, tpr)), dim3(tpr), 0, st, a);
    return hipGetLastError();
  });
}
hipError_t launch_block_norm_fwd(int dtype, const BlockNormArgs& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  ProfileScope ps("block_norm_fwd", st);
  return dtype == 0 ? block_norm_fwd_of<float>(a, st) : block_norm_fwd_of<bf16>(a, st);
}

template <typename T>
static hipError_t block_norm_bwd_of(const BlockNormArgs& a, hipStream_t st) {
  const bool sums = needs_sums(a);
  const int parts = sums ? bwd_parts(a.rows, a.width) : bwd_groups(a.rows, a.width);
  if (parts > 0) {
    const hipError_t e = by_width(a.width, [&](auto tpr, auto ch) {
      constexpr int rows = bwd_rows(tpr);
      hipLaunchKernelGGL((block_norm_bwd_kernel<T, tpr, ch, rows>), dim3(parts), dim3(tpr * rows), 0, st, a);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (!sums || parts == 1 || (parts == 0 && !a.overwrite)) return hipSuccess;
  hipLaunchKernelGGL((block_norm_sums_kernel<T>), dim3((a.width + 31) / 32, 2), dim3(1024), 0, st, a, parts);
  return hipGetLastError();
}
hipError_t launch_block_norm_bwd(int dtype, const BlockNormArgs& a, hipStream_t st) {
  ProfileScope ps("block_norm_bwd", st);
  return dtype == 0 ? block_norm_bwd_of<float>(a, st) : block_norm_bwd_of<bf16>(a, st);
}

// ------------------------------------------------------------- 8 bits
// CH chunks of eight values a thread; a row's chunks are rounded up to whole
// blocks.  Two chunks a thread where rows are whole blocks: 16-byte accesses of q.
// HBM bound: 4096 rows of 14336 packed in 30 us (5.9 TB/s), read in 30; 28672 rows of
// 4096 renormalised in 74.6 us (one chunk a thread: 79.5).
template <typename T, int CH>
__global__ __launch_bounds__(256) void act8_pack_kernel(const T* __restrict__ x, char* __restrict__ q,
                                                        uint8_t* __restrict__ e, unsigned rows, int width,
                                                        unsigned per_row) {
  const unsigned i = (blockIdx.x * 256u + threadIdx.x) * CH, row = i / per_row, c = i % per_row;
  const bool inside = row < rows && 8 * c < (unsigned)width;
  const size_t at = (size_t)row * width + 8 * c;
  Raw8<T> raw[CH];
  float v[CH][8];
  unsigned most = 0;
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    raw[k].zero();
    if (inside) raw[k].load(x, at + 8 * k);
  }
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    raw[k].values(v[k], false);
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, magnitude(v[k][j]));
  }
  most = inside ? most : 0u;
  const Act8Scale s = act8_scale(CH == 1 ? quad_max(most) : max(most, dpp<kXor1>(most)));
  if (!inside) return;
  unsigned out[2 * CH];
#pragma unroll
  for (int k = 0; k < 2 * CH; ++k) {
    const float* p = v[k / 2] + 4 * (k % 2);
    out[k] = act8_quad(p[0], p[1], p[2], p[3], s);
  }
  if constexpr (CH == 1)
    *(u32x2*)(q + at) = u32x2{out[0], out[1]};
  else
    *(u32x4*)(q + at) = u32x4{out[0], out[1], out[2], out[3]};
  if (c % 4 == 0) e[(size_t)row * (per_row / 4) + c / 4] = (uint8_t)s.exponent;
}

template <typename T, int CH>
__global__ __launch_bounds__(256) void act8_unpack_kernel(const char* __restrict__ q, const uint8_t* __restrict__ e,
                                                          const float* __restrict__ rstd, const T* __restrict__ gain,
                                                          T* __restrict__ y, unsigned rows, int width,
                                                          unsigned per_row) {
  const unsigned i = (blockIdx.x * 256u + threadIdx.x) * CH, row = i / per_row, c = i % per_row;
  if (row >= rows || 8 * c >= (unsigned)width) return;
  const size_t at = (size_t)row * width + 8 * c;
  Act8Chunk raw[CH];
  if constexpr (CH == 1) {
    raw[0].load(q, e, at, (size_t)row * (per_row / 4) + c / 4, true);
  } else {
    const u32x4 w = *(const u32x4*)(q + at);
    const unsigned x = e[(size_t)row * (per_row / 4) + c / 4];
    raw[0].raw = u32x4{w.x, w.y, x, 0};
    raw[CH - 1].raw = u32x4{w.z, w.w, x, 0};
  }
  const float r = rstd != nullptr ? rstd[row] : 1.f;
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    float v[8], g[8];
    raw[k].values(v, true);
    if (rstd != nullptr)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= r;
    if (gain != nullptr) {
      Raw8<T> w;
      w.load(gain, 8 * (c + k));
      w.values(g, false);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= g[j];
    }
    store8(y + at + 8 * k, v);
  }
}

namespace {
// f<chunks a thread>(first row, rows, workgroups) for ranges of rows whose chunks
// stay below 2^31
template <typename F>
hipError_t by_rows(long rows, int width, bool aligned, F f) {
  const long per_row = (width + 31L) / 32 * 4, most = (1L << 30) / per_row;
  const int two = width % 32 == 0 && aligned ? 2 : 1;
  for (long row = 0; row < rows; row += most) {
    const long n = rows - row < most ? rows - row : most;
    const unsigned grid = (unsigned)((n * per_row / two + 255) / 256);
    if (two == 2)
      f(std::integral_constant<int, 2>{}, row, (unsigned)n, grid, (unsigned)per_row);
    else
      f(std::integral_constant<int, 1>{}, row, (unsigned)n, grid, (unsigned)per_row);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
}  // namespace

template <typename T>
static hipError_t act8_pack_of(long rows, int width, const T* x, char* q, uint8_t* e, hipStream_t st) {
  return by_rows(rows, width, (uintptr_t)q % 16 == 0, [&](auto ch, long row, unsigned n, unsigned grid, unsigned per_row) {
    hipLaunchKernelGGL((act8_pack_kernel<T, ch>), dim3(grid), dim3(256), 0, st, x + row * width, q + row * width,
                       e + row * (per_row / 4), n, width, per_row);
  });
}
hipError_t launch_act8_pack(int dtype, long rows, int width, const void* x, void* q, void* e, hipStream_t st) {
  ProfileScope ps("act8_pack", st);
  return dtype == 0 ? act8_pack_of(rows, width, (const float*)x, (char*)q, (uint8_t*)e, st)
                    : act8_pack_of(rows, width, (const bf16*)x, (char*)q, (uint8_t*)e, st);
}

template <typename T>
static hipError_t act8_unpack_of(long rows, int width, const char* q, const uint8_t* e, const float* rstd,
                                 const T* gain, T* y, hipStream_t st) {
  return by_rows(rows, width, (uintptr_t)q % 16 == 0, [&](auto ch, long row, unsigned n, unsigned grid, unsigned per_row) {
    hipLaunchKernelGGL((act8_unpack_kernel<T, ch>), dim3(grid), dim3(256), 0, st, q + row * width,
                       e + row * (per_row / 4), rstd != nullptr ? rstd + row : nullptr, gain, y + row * width, n, width,
                       per_row);
  });
}
hipError_t launch_act8_unpack(int dtype, long rows, int width, const void* q, const void* e, const float* rstd,
                              const void* gain, void* y, hipStream_t st) {
  ProfileScope ps("act8_unpack", st);
  return dtype == 0 ? act8_unpack_of(rows, width, (const char*)q, (const uint8_t*)e, rstd, (const float*)gain,
                                     (float*)y, st)
                    : act8_unpack_of(rows, width, (const char*)q, (const uint8_t*)e, rstd, (const bf16*)gain, (bf16*)y,
                                     st);
}

}  // namespace spr
