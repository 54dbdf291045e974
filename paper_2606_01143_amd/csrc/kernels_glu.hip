// Gated feed-forward of a decoder block, dense or by expert: m = act(x Wg) * (x Wu)
// in one kernel, and backward through the down product and the activation in one:
//   dm = dy Wd^T,  dg = dm u act'(g),  du = dm act(g),  m = act(g) u.
// The tiles are experts.hpp's; this file holds the launches and their choice.
//
// Bound by the matrix cores where there are hundreds of rows, by the weights' bytes
// where there are few.  28672 rows of 4096 x 14336: m alone 5060 us (1331 TFLOP/s; the
// library's product of these sizes reaches 1302), m with g and u in 8 bits 5370 us,
// backward from 8 bits 3115 us (1081 TFLOP/s: 25 us of a tile's 130 read g and u and
// write dg, du and m).  Four rows of it forward 47 us (5.0 TB/s of weights).
// 128 experts of 2048 x 768, 8192 tokens of top-8: forward with bf16 g and u 460 us,
// backward 335 us (3.8 TB/s).
#include <algorithm>

#include "experts.hpp"

namespace spr {

namespace {

// Few tiles and a long contraction: a workgroup's W waves each take a W-th of the
// contraction of one tile of 32 rows and BN weight columns (glu: half of w_gate
// and half of w_up).  A wave loads and reads tiles of its own, so the loop has no
// barrier; the partial tiles are added in LDS, in the order of the waves.
template <int MODE, int BN, int STEP, int W, int RING>
__global__ __launch_bounds__(64 * W) void glu_split_kernel(ExpertArgs a) {
  constexpr int MI = 1, NI = BN / 32, BM = 32 * MI, A_ELEMS = BM * STEP, B_ELEMS = BN * STEP;
  constexpr bool DX = MODE == kGluBwd;
  constexpr int CN = DX ? BN : BN / 2;  // columns of the result
  typedef Natural<BM, STEP, 1> NatA;
  typedef Natural<BN, STEP, 1> NatB;
  typedef Transposed<BN, STEP, 1> TrB;
  constexpr int LOADS = NatA::I + (DX ? NatB::I : TrB::I);
  constexpr int PAD = BN + 4;  // of a row of partial sums
  constexpr int WAVE_ELEMS = RING * (A_ELEMS + B_ELEMS);
  static_assert(BM * PAD * 2 <= WAVE_ELEMS, "a partial tile fits its wave's ring");
  __shared__ __attribute__((aligned(1024))) bf16 smem[W * WAVE_ELEMS];
  const int lane = threadIdx.x & 63, w = wave_id(), r = lane & 31, h = lane >> 5;
  const int ncols = DX ? a.in_width : a.out_width, depth = DX ? a.out_width : a.in_width;
  const int tiles_n = (ncols + CN - 1) / CN;
  GroupTile g = find_tile<BM>(a, tiles_n, lane);
  if (!g.any) return;
  g.n0 *= CN;
  const int mrows = g.len - g.m0;
  const int steps = (depth + STEP - 1) / STEP, per = (steps + W - 1) / W;
  const int first = min(w * per, steps), last = min(first + per, steps);

  NatA an;
  NatB bn;
  TrB bt;
  an.init(0, lane, [&](int m) {
    const int row = g.lo + g.m0 + min(m, mrows - 1);
    long src = row;
    if (!DX && a.row_token != nullptr) src = clampi(a.row_token[row], 0, a.x_rows - 1);
    return (const bf16*)a.a + src * depth;
  });
  const size_t wsize = (size_t)a.in_width * a.out_width;
  if constexpr (DX) {
    bn.init(0, lane, [&](int n) {
      return (const bf16*)a.b + g.e * wsize + (size_t)min(g.n0 + n, ncols - 1) * a.out_width;
    });
  } else {
    const size_t at = (size_t)g.e * wsize + g.n0;
    bt.init_turns(0, lane, (const bf16*)a.b + at, (const bf16*)a.b2 + at, ncols - g.n0);
    bt.own_rows(2L * a.out_width);
  }
  const long b_step = DX ? 2L * STEP : 2L * STEP * a.out_width;
  auto advance = [&](long by) {
    an.advance(2L * STEP * by);
    if constexpr (DX)
      bn.advance(b_step * by);
    else
      bt.advance(b_step * by);
  };
  // points the loads at step s; behind the wave's last one they read zeros
  auto aim = [&](int s) {
    const int left = s < last ? depth - s * STEP : 0;
    if (left < STEP) {
      an.stop(left);
      if constexpr (DX)
        bn.stop(left);
      else
        bt.stop(left);
    }
  };
  bf16* ring = smem + w * WAVE_ELEMS;
  auto load = [&](auto buffer) {
    constexpr int b = decltype(buffer)::value;
    bf16 *ta = ring + b * A_ELEMS, *tb = ring + RING * A_ELEMS + b * B_ELEMS;
    each<NatA::I>([&](auto i) { an.template load<i>(ta); });
    if constexpr (DX)
      each<NatB::I>([&](auto i) { bn.template load<i>(tb); });
    else
      each<TrB::I>([&](auto i) { bt.template load<i>(tb); });
  };
  f32x16 acc[NI][MI];
#pragma unroll
  for (int n = 0; n < NI; ++n)
#pragma unroll
    for (int m = 0; m < MI; ++m) acc[n][m] = zero16();
  advance(first);
  aim(first);
  each<RING - 1>([&](auto b) {
    load(b);
    advance(1);
    aim(first + b + 1);
  });
  for (int s = first; s < last;) {
    each<RING>([&](auto buffer) {
      if (s >= last) return;
      constexpr int b = decltype(buffer)::value;
      // step s has landed, and the last step's reads are done: its buffer is free
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"((RING - 2) * LOADS) : "memory");
      load(std::integral_constant<int, (b + RING - 1) % RING>{});
      advance(1);
      aim(s + RING);
      const bf16 *ta = ring + b * A_ELEMS, *tb = ring + RING * A_ELEMS + b * B_ELEMS;
      each<STEP / 16>([&](auto v) {
        bf16x8 fa[MI], fb[NI];
        each<MI>([&](auto m) { fa[m] = *(const bf16x8*)(ta + NatA::frag(lane, v) + m * 32 * STEP); });
        each<NI>([&](auto n) {
          if constexpr (DX)
            fb[n] = *(const bf16x8*)(tb + NatB::frag(lane, v) + n * 32 * STEP);
          else
            fb[n] = tr_pair(tb + TrB::frag(lane, n, 0) + v * 16 * TrB::PW, tb + TrB::frag(lane, n, 1) + v * 16 * TrB::PW);
        });
        each<NI * MI>([&](auto q) { acc[q % NI][q / NI] = mfma32(fb[q % NI], fa[q / NI], acc[q % NI][q / NI]); });
      });
      ++s;
    });
  }
  // ---- the waves' partial tiles: row, then weight columns
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  float* part = (float*)(smem + w * WAVE_ELEMS);
  each<NI * MI * 4>([&](auto q) {
    constexpr int n = q / 4 % NI, m = q / 4 / NI, i = q % 4;
    *(f32x4*)(part + (32 * m + r) * PAD + 32 * n + 8 * i + 4 * h) =
        f32x4{acc[n][m][4 * i], acc[n][m][4 * i + 1], acc[n][m][4 * i + 2], acc[n][m][4 * i + 3]};
  });
  __syncthreads();
  auto sum4 = [&](int row, int col) {
    f32x4 s = *(const f32x4*)((const float*)smem + row * PAD + col);
#pragma unroll
    for (int q = 1; q < W; ++q) s += *(const f32x4*)((const float*)(smem + q * WAVE_ELEMS) + row * PAD + col);
    return s;
  };
  const int blocks = (ncols + 31) / 32;
  const bool small = a.ge != nullptr;
  if constexpr (DX) {
    for (int at = threadIdx.x; at < BM * BN / 8; at += 64 * W) {
      const int row = at / (BN / 8), c = 8 * (at % (BN / 8)), col = g.n0 + c;
      if (row >= mrows || col >= ncols) continue;
      const size_t out_row = (size_t)(g.lo + g.m0 + row), dst = out_row * ncols + col;
      Act8Chunk kg, ku;
      kg.load(a.g, a.ge, dst, out_row * blocks + col / 32, small);
      ku.load(a.u, a.ue, dst, out_row * blocks + col / 32, small);
      const f32x4 lo = sum4(row, c), hi = sum4(row, c + 4);
      float gv[8], uv[8], dg[8], du[8], mv[8];
      kg.values(gv, small);
      ku.values(uv, small);
      with_act(a.act, [&](auto f) {
#pragma unroll
        for (int j = 0; j < 8; ++j) glu_gradients(f, j < 4 ? lo[j] : hi[j - 4], gv[j], uv[j], dg[j], du[j], mv[j]);
      });
      store_bf16x8((bf16*)a.c + dst, dg);
      store_bf16x8((bf16*)a.c2 + dst, du);
      if (a.c3 != nullptr) store_bf16x8((bf16*)a.c3 + dst, mv);
    }
  } else {
    // eight lanes a row, whose 32 columns are one block of the 8-bit form
    for (int at = threadIdx.x; at < BM * CN / 4; at += 64 * W) {
      const int row = at / (CN / 4), c = 4 * (at % (CN / 4)), col = g.n0 + c, in = c / 32 * 64 + c % 32;
      const bool inside = row < mrows && col < ncols;
      const size_t out_row = (size_t)(g.lo + g.m0 + row), dst = out_row * ncols + col;
      const f32x4 gv = sum4(row, in), uv = sum4(row, in + 32);
      if (inside) {
        bf16x4 m;
        with_act(a.act, [&](auto f) {
#pragma unroll
          for (int j = 0; j < 4; ++j) m[j] = (bf16)(decltype(f)::of(gv[j]).value * uv[j]);
        });
        *(bf16x4*)((bf16*)a.c + dst) = m;
      }
      if (a.g == nullptr) continue;
      auto keep = [&](const f32x4& v, void* p, uint8_t* e) {
        if (!small) {
          if (inside) *(bf16x4*)((bf16*)p + dst) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
          return;
        }
        unsigned most = max(max(magnitude(v[0]), magnitude(v[1])), max(magnitude(v[2]), magnitude(v[3])));
        const Act8Scale s = act8_scale(eight_max(inside ? most : 0u));
        if (!inside) return;
        *(unsigned*)((char*)p + dst) = act8_quad(v[0], v[1], v[2], v[3], s);
        if (c % 32 == 0) e[out_row * blocks + col / 32] = (uint8_t)s.exponent;
      };
      keep(gv, a.g, a.ge);
      keep(uv, a.u, a.ue);
    }
  }
}

template <int MODE, int BN, int STEP, int W, int RING>
hipError_t launch_split(const ExpertArgs& a, hipStream_t st) {
  constexpr int CN = MODE == kGluBwd ? BN : BN / 2;
  const int ncols = MODE == kGluBwd ? a.in_width : a.out_width;
  const long some = a.E < a.rows ? a.E : a.rows;
  long grid = (long)((ncols + CN - 1) / CN) * ((a.rows + some * 31) / 32);
  grid = (grid + kXcds - 1) / kXcds * kXcds;
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL((glu_split_kernel<MODE, BN, STEP, W, RING>), dim3((unsigned)grid), dim3(64 * W), 0, st, a);
  return hipGetLastError();
}

// Which tiles: the least of an estimate of each form's time.  A launch is rounds of
// `slots` workgroups; a round takes its steps of 64 contraction indices and a
// tile's beginning and end, both longer where the CUs are full (they then share
// the memory and, two workgroups a CU, the matrix cores).  Groups' ragged ends
// count as half a tile of rows each, and one dense block's last round as a whole
// one.  Where the weights are all there is to read their bytes count: the split
// form of glu reads half a line of either weight at a time.
// The constants (us) were fitted to one half of 529 sizes drawn from 1 to 28672
// tokens, widths of 128 to 14336 and 1 to 128 experts, before the backward's stores
// went past the caches.  Timed again on these kernels, the form taken is on the other
// half 1.3% (glu) and 1.6% (glu_bwd) slower than the best of them on average.  The worst of
// all 529 are 41% (glu, 60 experts of 3888 x 352, 29 tokens) and 27% (glu_bwd, 128 rows of
// 4096 x 14336, as the table shows; 96 rows take 48 us where 64 x 128 takes 40).
// Measured at 4096 x 14336, us for 4, 64, 128, 256, 512, 1299, 28672 tokens, glu keeping
// neither g nor u, glu_bwd from 8 bits and with m, the form taken marked *:
//   glu      64 x 128 48* 52* 85 118 199 435 9170, 128 x 128 deep 51 53 58* 95 169 380
//            7670, 128 x 128 72 71 74 94 161 348 6410, 192 x 256 93 93 95 96 177 322 5730,
//            256 x 256 94 94 97 102* 109* 297* 5060*, split 71 104 165 274 515 1085 -
//   glu_bwd  64 x 128 35 40 42 65 113 234 4260, 128 x 128 deep 35 40 53* 55* 101 224 4220,
//            128 x 128 58 61 66 69 93* 215 3730, 192 x 256 74 77 85 91 106 203* 3150, 256 x
//            256 77 81 89 113 122 228 3115*, split 25* 36* 56 97 172 380 -, split narrow 27
//            50 80 151 293 611 -
// and the split forms against the best other: glu 4 tokens of 4624 x 128 10.5 / 22.0,
// 253 of 1560 x 336 10.8 / 13.9; glu_bwd 339 of 3784 x 336 narrow 13, wide 18, other 31.
// (A CU takes in about 43 KB a us, with 48 KB on their way as with 96: the split
// forms differ by the lines that they read whole and the CUs that they reach.)
enum GluForm { k64x128, k128x128Deep, k128x128, k192x256, k256x256, kSplit, kSplitNarrow };
struct GluCost {
  int rows, cols, slots, threads;           // of a tile (cols of the result), the card, a workgroup
  double step, step_full, tile, tile_full;  // us: alone, and more where all slots are taken
};
constexpr int kGluForms = 6, kGluBwdForms = 7;
constexpr GluCost kGluCost[kGluForms] = {
    {64, 64, 512, 256, 0.24, 0.57, 2.8, 0.1},   {128, 64, 256, 256, 0.33, 0.31, 2.7, 1.0},
    {128, 64, 512, 256, 0.54, 0.75, 2.6, 0.6},  {192, 128, 256, 512, 0.74, 0.72, 4.0, 0.},
    {256, 128, 256, 512, 0.75, 0.88, 5.0, 0.},  {32, 32, 512, 256, 0.16, 0.33, 2.4, 0.}};
constexpr GluCost kGluBwdCost[kGluBwdForms] = {
    {64, 128, 512, 256, 0.21, 0.62, 3.2, 2.2},   {128, 128, 256, 256, 0.24, 0.47, 4.4, 3.0},
    {128, 128, 512, 256, 0.38, 0.94, 4.0, 5.9},  {192, 256, 256, 512, 0.75, 0.92, 4.0, 11.0},
    {256, 256, 256, 512, 0.77, 1.21, 5.0, 14.9}, {32, 64, 512, 192, 0.07, 0.27, 3.8, 0.},
    {32, 32, 256, 256, 0.05, 0.07, 2.8, 0.}};

// Whether a launch, of at most 2^32 - 1 threads, holds a form's tiles: at most one
// of rows that is not whole for every expert with rows, as many workgroups on every
// XCD.  Where one form's do not fit, larger tiles' may.
inline bool launches(const GluCost& c, int experts, long rows, long cols) {
  const long some = std::min<long>(experts, rows);
  const long groups = (cols + c.cols - 1) / c.cols * ((rows + some * (c.rows - 1)) / c.rows);
  return (groups + 7) / 8 * 8 * c.threads <= (long)UINT32_MAX;
}
template <int FORMS>
bool glu_fits(const GluCost (&cost)[FORMS], int experts, long rows, long cols) {
  return std::any_of(cost, cost + FORMS, [&](const GluCost& c) { return launches(c, experts, rows, cols); });
}

template <int FORMS>
int glu_form(const GluCost (&cost)[FORMS], int experts, long rows, long cols, long depth, double weight_mb) {
  const double some = (double)std::min<long>(experts, rows);
  int best = 0;
  double least = -1.;
  for (int f = 0; f < FORMS; ++f) {
    const GluCost& c = cost[f];
    if (!launches(c, experts, rows, cols)) continue;
    const double high = experts == 1 ? (double)((rows + c.rows - 1) / c.rows)
                                     : std::max(some, (double)rows / c.rows + 0.5 * some);
    const double x = high * (double)((cols + c.cols - 1) / c.cols) / c.slots, fill = std::min(x, 1.);
    const double rounds = x <= 1. ? 1. : experts == 1 && x < 8. ? (double)(long)(x + 0.999999) : x + 0.5;
    const double steps = (double)((depth + 63) / 64);
    const double bytes = some * weight_mb / (FORMS == kGluForms && f == kSplit ? 3.3 : 4.9);  // at TB/s
    const double t = std::max(rounds * (steps * (c.step + c.step_full * fill) + c.tile + c.tile_full * fill), bytes);
    if (least < 0. || t < least) {
      best = f;
      least = t;
    }
  }
  return best;
}

template <int MODE>
hipError_t launch_glu(const ExpertArgs& a, int form, hipStream_t st) {
  static_assert(kXcds == 8, "launches() counts workgroups of eight XCDs");
  switch (form) {
    case k64x128: return launch_tiles<MODE, 64, 128, 2, 2, 64, 3>(a, st);
    case k128x128Deep: return launch_tiles<MODE, 128, 128, 2, 2, 64, 4>(a, st);
    case k128x128: return launch_tiles<MODE, 128, 128, 2, 2, 64, 2>(a, st);
    case k192x256: return launch_tiles<MODE, 192, 256, 2, 4, 64, 2>(a, st);
    case k256x256: return launch_tiles<MODE, 256, 256, 2, 4, 64, 2>(a, st);
  }
  if constexpr (MODE == kGlu) return launch_split<kGlu, 64, 32, 4, 3>(a, st);
  else return form == kSplit ? launch_split<kGluBwd, 64, 64, 3, 2>(a, st) : launch_split<kGluBwd, 32, 64, 4, 3>(a, st);
}

}  // namespace

bool glu_fwd_fits(int experts, int rows, int mid_width) { return glu_fits(kGluCost, experts, rows, mid_width); }
bool glu_bwd_fits(int experts, int rows, int mid_width) { return glu_fits(kGluBwdCost, experts, rows, mid_width); }

hipError_t launch_glu_fwd(const ExpertArgs& a, hipStream_t st) {
  ProfileScope ps("glu_fwd", st);
  const double mb = 4e-6 * a.in_width * a.out_width;
  return launch_glu<kGlu>(a, glu_form(kGluCost, a.E, a.rows, a.out_width, a.in_width, mb), st);
}

hipError_t launch_glu_bwd(const ExpertArgs& a, hipStream_t st) {
  ProfileScope ps("glu_bwd", st);
  const double mb = 2e-6 * a.in_width * a.out_width;
  return launch_glu<kGluBwd>(a, glu_form(kGluBwdCost, a.E, a.rows, a.in_width, a.out_width, mb), st);
}

}  // namespace spr
