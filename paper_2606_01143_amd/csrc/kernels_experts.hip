// Products grouped by expert with ragged sizes, on bf16 matrix instructions.
//
// The rows of expert e are offsets[e] .. offsets[e + 1] - 1.  One kernel, three
// products of a tile of C (BM rows by BN columns, fp32 in registers):
//   fwd    C = x rows (gathered) . w[e]          contraction over in_width
//   bwd_x  C = dy rows . w[e]^T (two pairs)      contraction over out_width
//   bwd_w  C = (x rows)^T . dy rows              contraction over e's rows
// An operand whose contraction index is contiguous in memory ("natural") is
// staged as [row][32] tiles and read 16 bytes a lane; one whose contraction
// index is the slow one is staged as [32][128] panels and read transposed
// (ds_read_b64_tr_b16).  Tiles arrive by direct-to-LDS loads two steps of 32
// ahead, in a ring of three buffers, one barrier a step.  The weights' side is
// the matrix instruction's first operand, so that a lane's four consecutive
// results are consecutive columns of C.
//
// Ragged ends: contraction indices past the end are read from a line of zeros
// (both operands: a zero times another row's infinity would be a NaN); C rows
// and columns past the end repeat a valid address and are not stored.  A wave
// whose rows are all past the end skips its products.
#include "launch.hpp"
#include "tile.hpp"

namespace spr {

namespace {

enum ExpertMode { kFwd = 0, kBwdX = 1, kBwdW = 2 };
constexpr int kStep = 32;   // contraction indices per step
constexpr int kRing = 3;    // tile buffers
constexpr int kXcds = 8;

__device__ const uint4 zero_line = {0, 0, 0, 0};

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// Natural operand: ROWS rows of 32 contiguous contraction indices, 64 bytes a
// row.  Chunk c (16 bytes) of row m lies at chunk c ^ ((m >> 2) & 3): the 16
// lanes of a read phase then cover 256 bytes once.
template <int ROWS, int WAVES>
struct Natural {
  static constexpr int N = ROWS / 16, I = (N + WAVES - 1) / WAVES;  // 1 KB loads: of the tile, of a wave
  const char* p[I];
  int col, w;
  template <typename RowPtr>
  __device__ __forceinline__ void init(int wave, int lane, RowPtr row_ptr) {
    w = wave;
    col = 8 * ((lane & 3) ^ ((lane >> 4) & 3));
#pragma unroll
    for (int i = 0; i < I; ++i) p[i] = (const char*)(row_ptr(16 * ((w + WAVES * i) % N) + (lane >> 2)) + col);
  }
  // indices k0 .. k0 + 31 of [.., end), `off` bytes from each row's pointer
  __device__ __forceinline__ void load(bf16* tile, long off, int k0, int end) const {
    const bool cut = k0 + kStep > end;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const char* q = p[i] + off;
      if (cut) q = k0 + col < end ? q : (const char*)&zero_line;
      dma_lds16(q, lds_addr(tile + 512 * ((w + WAVES * i) % N)));
    }
  }
  static __device__ __forceinline__ int frag(int lane, int v) {
    const int r = lane & 31, h = lane >> 5;
    return r * kStep + 8 * ((2 * v + h) ^ ((r >> 2) & 3));
  }
};

// Transposed operand: 32 contraction rows of COLS columns, in panels of 128.
template <int COLS, int WAVES>
struct Transposed {
  static constexpr int N = COLS / 16, I = (N + WAVES - 1) / WAVES;
  int row[I], col[I], w;
  __device__ __forceinline__ void init(int wave, int lane, int ncols) {
    w = wave;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int q = (w + WAVES * i) % N;  // panel q / 8, rows 4 (q % 8) ..
      row[i] = 4 * (q & 7) + (lane >> 4);
      const int c = 128 * (q >> 3) + 8 * ((lane & 15) ^ swz<128>(row[i]));
      col[i] = c < ncols ? c : 0;
    }
  }
  // row_ptr(k): contraction row k's first column of this tile
  template <typename RowPtr>
  __device__ __forceinline__ void load(bf16* tile, int k0, int end, RowPtr row_ptr) const {
    const bool cut = k0 + kStep > end;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const bf16* q;
      if (cut)
        q = k0 + row[i] < end ? row_ptr(k0 + row[i]) + col[i] : (const bf16*)&zero_line;
      else
        q = row_ptr(k0 + row[i]) + col[i];
      dma_lds16(q, lds_addr(tile + 512 * ((w + WAVES * i) % N)));
    }
  }
  // element offset of 32-column block b's operand, contraction rows 8 h + 4 hi ..
  static __device__ __forceinline__ int frag(int lane, int b, int hi) {
    const int h = lane >> 5, i16 = lane & 15;
    return (b >> 2) * kStep * 128 +
           toff<128>(8 * h + 4 * hi + (i16 >> 2), 32 * (b & 3) + (lane & 16) + 4 * (i16 & 3));
  }
};

__device__ __forceinline__ bf16x8 tr_pair(const bf16* lo, const bf16* hi) {
  const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)lo);
  const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)hi);
  return bf16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

template <int N>
__device__ __forceinline__ void wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(N) : "memory");
}

// A workgroup's tile: expert, its rows, first row and column of C.
struct GroupTile {
  int e, lo, len, m0, n0, part;
  bool any;
};

// Tile t of the launch: experts in order, each expert's tiles column by
// column (`cols` columns of tiles), ceil(len / BM) rows of tiles.  A wave adds
// up the experts' tile rows 64 ranges at a time and finds the one that holds t.
// The workgroups of one XCD (blockIdx modulo 8) take consecutive tiles, which
// share an expert's weights and rows in its L2.
template <int BM>
__device__ __forceinline__ GroupTile find_tile(const ExpertArgs& a, int cols, int lane) {
  const int per = (a.E + 63) / 64;
  auto rows_of = [&](int e, int& lo) {
    lo = clampi(a.offsets[e], 0, a.rows);
    return clampi(a.offsets[e + 1], lo, a.rows) - lo;
  };
  int mine = 0, lo;
  for (int q = 0; q < per; ++q) {
    const int e = lane * per + q;
    if (e < a.E) mine += (rows_of(e, lo) + BM - 1) / BM;
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  const long total = (long)__builtin_amdgcn_readlane(upto, 63) * cols;
  const long chunk = (total + kXcds - 1) / kXcds;
  const long at = blockIdx.x / kXcds, t = (blockIdx.x % kXcds) * chunk + at;
  GroupTile g;
  g.any = at < chunk && t < total;
  if (!g.any) return g;
  // offsets that overlap can add up to more tiles than the launch has, or wrap
  // the sum: then no expert may hold t, and the search ends at the last one
  const unsigned long long past = __ballot((long)upto * cols > t);
  const int owner = past != 0 ? __builtin_ctzll(past) : 63;
  long left = t - (long)__builtin_amdgcn_readlane(upto - mine, owner) * cols;
  for (g.e = owner * per; g.e < a.E; ++g.e) {
    g.len = rows_of(g.e, g.lo);
    const int mt = (g.len + BM - 1) / BM;
    if (left >= 0 && left < (long)mt * cols) {
      g.m0 = (int)(left % mt) * BM;
      g.n0 = (int)(left / mt);  // column of tiles; the caller turns it into columns
      return g;
    }
    left -= (long)mt * cols;
  }
  g.any = false;
  return g;
}

template <int MODE, int BM, int BN, int MW, int NW>
__global__ __launch_bounds__(64 * MW * NW, 2) void experts_kernel(ExpertArgs a) {
  constexpr int WAVES = MW * NW, MI = BM / 32 / MW, NI = BN / 32 / NW;
  constexpr bool A_TR = MODE == kBwdW, B_TR = MODE != kBwdX;
  constexpr int A_ELEMS = BM * kStep, B_ELEMS = BN * kStep;
  constexpr int LOADS = (BM / 16 + WAVES - 1) / WAVES + (BN / 16 + WAVES - 1) / WAVES;
  constexpr int OUT_STRIDE = NI * 32 + 8;  // staged output rows, 16 bytes apart in banks
  constexpr int SMEM = kRing * (A_ELEMS + B_ELEMS);
  static_assert(WAVES * 32 * OUT_STRIDE <= SMEM, "the output staging fits the ring");
  __shared__ __attribute__((aligned(1024))) bf16 smem[SMEM];
  const int lane = threadIdx.x & 63, w = wave_id(), wm = w / NW, wn = w % NW;
  const int r = lane & 31, h = lane >> 5;
  // columns of C, and of tiles: C is [rows, out_width], [rows, in_width] or [in_width, out_width]
  const int ncols = MODE == kBwdX ? a.in_width : a.out_width;
  const int tiles_n = (ncols + BN - 1) / BN, parts = a.b2 != nullptr ? 2 : 1;

  GroupTile g;
  if constexpr (MODE == kBwdW) {
    const int tiles_m = (a.in_width + BM - 1) / BM;
    const long total = (long)a.E * parts * tiles_n * tiles_m, chunk = (total + kXcds - 1) / kXcds;
    const long at = blockIdx.x / kXcds, t = (blockIdx.x % kXcds) * chunk + at;
    if (at >= chunk || t >= total) return;
    g.m0 = (int)(t % tiles_m) * BM;
    g.n0 = (int)(t / tiles_m % tiles_n) * BN;
    g.part = (int)(t / tiles_m / tiles_n % parts);
    g.e = (int)(t / tiles_m / tiles_n / parts);
    g.lo = clampi(a.offsets[g.e], 0, a.rows);
    g.len = clampi(a.offsets[g.e + 1], g.lo, a.rows) - g.lo;
    if (g.len == 0 && !a.overwrite) return;
  } else {
    const int cols = MODE == kFwd ? tiles_n * parts : tiles_n;
    g = find_tile<BM>(a, cols, lane);
    if (!g.any) return;
    g.part = g.n0 / tiles_n;
    g.n0 = g.n0 % tiles_n * BN;
  }
  const int mrows = MODE == kBwdW ? a.in_width - g.m0 : g.len - g.m0;  // rows of C left
  // this wave's 32-row blocks are wm, wm + MW, ..; act of them have rows
  const int act = clampi((mrows - 32 * wm + 32 * MW - 1) / (32 * MW), 0, MI);
  const int depth = MODE == kFwd ? a.in_width : MODE == kBwdX ? a.out_width : g.len;
  const int steps1 = (depth + kStep - 1) / kStep;
  const int steps = MODE == kBwdX ? steps1 * parts : steps1;
  const size_t wsize = (size_t)a.in_width * a.out_width;

  // ---- operands
  const bf16* bsrc = g.part != 0 && MODE != kBwdX ? (const bf16*)a.b2 : (const bf16*)a.b;
  Natural<BM, WAVES> an;
  Transposed<BM, WAVES> at;
  Natural<BN, WAVES> bn;
  Transposed<BN, WAVES> bt;
  long a_part = 0, b_part = 0;  // bytes from a pair's first operands to its second's
  if constexpr (!A_TR) {
    an.init(w, lane, [&](int m) {
      const int row = g.lo + g.m0 + min(m, mrows - 1);
      long src = row;
      if (MODE == kFwd && a.row_token != nullptr) src = clampi(a.row_token[row], 0, a.x_rows - 1);
      return (const bf16*)a.a + src * depth;
    });
    if (MODE == kBwdX && parts == 2) a_part = (const char*)a.a2 - (const char*)a.a;
  } else {
    at.init(w, lane, mrows);
  }
  if constexpr (!B_TR) {
    bn.init(w, lane, [&](int n) {
      return bsrc + g.e * wsize + (size_t)min(g.n0 + n, ncols - 1) * a.out_width;
    });
    if (parts == 2) b_part = (const char*)a.b2 - (const char*)a.b;
  } else {
    bt.init(w, lane, ncols - g.n0);
  }
  auto issue = [&](int s) {
    bf16* ta = smem + (s % kRing) * (A_ELEMS + B_ELEMS);
    bf16* tb = ta + A_ELEMS;
    const bool second = MODE == kBwdX && s >= steps1;
    const int k0 = (second ? s - steps1 : s) * kStep;
    if constexpr (!A_TR)
      an.load(ta, 2L * k0 + (second ? a_part : 0), k0, depth);
    else
      at.load(ta, k0, depth, [&](int k) {
        long src = g.lo + k;
        if (a.row_token != nullptr) src = clampi(a.row_token[src], 0, a.x_rows - 1);
        return (const bf16*)a.a + src * a.in_width + g.m0;
      });
    if constexpr (!B_TR)
      bn.load(tb, 2L * k0 + (second ? b_part : 0), k0, depth);
    else if constexpr (MODE == kFwd)
      bt.load(tb, k0, depth, [&](int k) { return bsrc + g.e * wsize + (size_t)k * a.out_width + g.n0; });
    else
      bt.load(tb, k0, depth, [&](int k) { return bsrc + (size_t)(g.lo + k) * a.out_width + g.n0; });
  };

  // ---- offsets of the operand reads
  int aoff[2][A_TR ? MI : 1], boff[2][B_TR ? NI : 1];
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    if constexpr (A_TR) {
#pragma unroll
      for (int i = 0; i < MI; ++i) aoff[v][i] = Transposed<BM, WAVES>::frag(lane, i * MW + wm, v);
    } else {
      aoff[v][0] = Natural<BM, WAVES>::frag(lane, v) + wm * 32 * kStep;
    }
    if constexpr (B_TR) {
#pragma unroll
      for (int i = 0; i < NI; ++i) boff[v][i] = Transposed<BN, WAVES>::frag(lane, wn * NI + i, v);
    } else {
      boff[v][0] = Natural<BN, WAVES>::frag(lane, v) + wn * NI * 32 * kStep;
    }
  }

  f32x16 acc[NI][MI];
#pragma unroll
  for (int n = 0; n < NI; ++n)
#pragma unroll
    for (int m = 0; m < MI; ++m) acc[n][m] = zero16();

  for (int s = 0; s < min(kRing - 1, steps); ++s) issue(s);
  for (int s = 0; s < steps; ++s) {
    if (s + 1 < steps)
      wait_barrier<LOADS>();
    else
      wait_barrier<0>();
    if (s + kRing - 1 < steps) issue(s + kRing - 1);
    const bf16* ta = smem + (s % kRing) * (A_ELEMS + B_ELEMS);
    const bf16* tb = ta + A_ELEMS;
    if (act == 0) continue;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      bf16x8 fb[NI], fa[MI];
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        if constexpr (B_TR)
          fb[n] = tr_pair(tb + boff[0][n] + v * 16 * 128, tb + boff[1][n] + v * 16 * 128);
        else
          fb[n] = *(const bf16x8*)(tb + boff[v][0] + n * 32 * kStep);
      }
#pragma unroll
      for (int m = 0; m < MI; ++m) {
        if constexpr (A_TR)
          fa[m] = tr_pair(ta + aoff[0][m] + v * 16 * 128, ta + aoff[1][m] + v * 16 * 128);
        else
          fa[m] = *(const bf16x8*)(ta + aoff[v][0] + m * MW * 32 * kStep);
      }
#pragma unroll
      for (int n = 0; n < NI; ++n)
#pragma unroll
        for (int m = 0; m < MI; ++m) acc[n][m] = mfma32(fb[n], fa[m], acc[n][m]);
    }
  }

  // ---- C: lane (r, h) holds row r of a 32-row block, columns 8 i + 4 h .. + 3
  if constexpr (MODE == kBwdW) {
    float* c = (float*)(g.part ? a.c2 : a.c) + g.e * wsize;
#pragma unroll
    for (int m = 0; m < MI; ++m) {
      const int row = g.m0 + 32 * (m * MW + wm) + r;
      if (row >= a.in_width) continue;
#pragma unroll
      for (int n = 0; n < NI; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int col = g.n0 + 32 * (wn * NI + n) + 8 * i + 4 * h;
          if (col >= ncols) continue;
          f32x4* dst = (f32x4*)(c + (size_t)row * a.out_width + col);
          f32x4 v = {acc[n][m][4 * i], acc[n][m][4 * i + 1], acc[n][m][4 * i + 2], acc[n][m][4 * i + 3]};
          if (!a.overwrite) v += *dst;
          *dst = v;
        }
    }
  } else {
    // through LDS, so that a row's 64 columns leave as one line
    wait_barrier<0>();
    bf16* out = smem + w * 32 * OUT_STRIDE;
    bf16* c = (bf16*)(g.part ? a.c2 : a.c);
    constexpr int CH = NI * 4;  // 16-byte chunks of a row
#pragma unroll
    for (int m = 0; m < MI; ++m) {
      const int row0 = 32 * (m * MW + wm);
      if (row0 >= mrows) break;
#pragma unroll
      for (int n = 0; n < NI; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(bf16x4*)(out + r * OUT_STRIDE + 32 * n + 8 * i + 4 * h) =
              bf16x4{(bf16)acc[n][m][4 * i], (bf16)acc[n][m][4 * i + 1], (bf16)acc[n][m][4 * i + 2],
                     (bf16)acc[n][m][4 * i + 3]};
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int q = lane; q < 32 * CH; q += 64) {
        const int row = q / CH, col = g.n0 + 32 * wn * NI + 8 * (q % CH);
        const bf16x8 v = *(const bf16x8*)(out + row * OUT_STRIDE + 8 * (q % CH));
        if (row0 + row < mrows && col < ncols)
          *(bf16x8*)(c + (size_t)(g.lo + g.m0 + row0 + row) * ncols + col) = v;
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

template <int MODE, int BM, int BN, int MW, int NW>
hipError_t launch_tiles(const ExpertArgs& a, hipStream_t st) {
  const int ncols = MODE == kBwdX ? a.in_width : a.out_width, parts = a.b2 != nullptr ? 2 : 1;
  const long tiles_n = (ncols + BN - 1) / BN;
  long grid;
  if (MODE == kBwdW) {
    grid = (long)a.E * parts * tiles_n * ((a.in_width + BM - 1) / BM);
  } else {
    // at most a partial tile of rows for every expert that has any
    const long some = a.E < a.rows ? a.E : a.rows;
    grid = (MODE == kFwd ? parts : 1) * tiles_n * ((a.rows + some * (BM - 1)) / BM);
  }
  grid = (grid + kXcds - 1) / kXcds * kXcds;
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL((experts_kernel<MODE, BM, BN, MW, NW>), dim3((unsigned)grid), dim3(64 * MW * NW), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_experts_fwd(const ExpertArgs& a, hipStream_t st) {
  ProfileScope ps("experts_fwd", st);
  return launch_tiles<kFwd, 128, 128, 2, 2>(a, st);
}
hipError_t launch_experts_bwd_x(const ExpertArgs& a, hipStream_t st) {
  ProfileScope ps("experts_bwd_x", st);
  return launch_tiles<kBwdX, 128, 128, 2, 2>(a, st);
}
hipError_t launch_experts_bwd_w(const ExpertArgs& a, hipStream_t st) {
  ProfileScope ps("experts_bwd_w", st);
  return launch_tiles<kBwdW, 128, 128, 2, 2>(a, st);
}

}  // namespace spr
