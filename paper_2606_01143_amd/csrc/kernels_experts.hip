// Products grouped by expert with ragged sizes, on bf16 matrix instructions.
//
// The rows of expert e are offsets[e] .. offsets[e + 1] - 1.  One kernel, three
// products of a tile of C (BM rows by BN columns, fp32 in registers):
//   fwd    C = x rows (gathered) . w[e]          contraction over in_width
//   bwd_x  C = dy rows . w[e]^T (two pairs)      contraction over out_width
//   bwd_w  C = (x rows)^T . dy rows              contraction over e's rows
// An operand whose contraction index is contiguous in memory ("natural") is
// staged as [row][STEP] tiles and read 16 bytes a lane; one whose contraction
// index is the slow one is staged as [STEP][128] panels and read transposed
// (ds_read_b64_tr_b16).  Tiles arrive by direct-to-LDS loads RING - 1 steps
// ahead, one barrier a step; the weights' side is the matrix instruction's first
// operand, so that a lane's four consecutive results are consecutive columns of
// C.  A step's code is one block: each product is followed by an operand read of
// the next slice, and in two of the slices by a load of a later step, so that the
// matrix cores are not left waiting for either.
//
// Bound by the matrix cores where experts have hundreds of rows, by the weights'
// bytes where they have few.  In 256 x 256 tiles of eight waves (128 x 64 a wave,
// one workgroup a CU; 256 x 128 tiles of four waves, two a CU, read a half more
// bytes into LDS and took 582 us where these took 430) 128 experts of 2048 x 768,
// 8192 tokens of top-8: gate and up 456 us (904 TFLOP/s, on some cards 425; a plain
// matrix product of the same operations reaches 1182 in the library), row gradients
// of both 474 us (870), weight gradients of both 681 us (605 TFLOP/s, 2.4 TB/s of
// fp32 gradients written).  Eight experts of 4096 x 1536: 1138, 1090 and 1205 TFLOP/s.
//
// Ragged ends: contraction indices past the end are read from a line of zeros
// (both operands: a zero times another row's infinity would be a NaN); C rows
// and columns past the end repeat a valid address and are not stored.  A wave
// skips the products of its 32-row blocks that are past the end.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "launch.hpp"
#include "tile.hpp"

namespace spr {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

enum ExpertMode { kFwd = 0, kBwdX = 1, kBwdW = 2 };
constexpr int kXcds = 8;
constexpr int kBand = 4;    // tile rows of a band

__device__ const uint4 zero_line = {0, 0, 0, 0};

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// Natural operand: ROWS rows of STEP (32 or 64) contiguous contraction indices.
// Chunk c (16 bytes) of row m lies at chunk c ^ place(m), so that the 16 lanes
// of a read phase (16 rows, one chunk) cover 256 bytes once.
template <int ROWS, int STEP, int WAVES>
struct Natural {
  static constexpr int CH = STEP / 8, RPL = 64 / CH;  // chunks of a row, rows of a 1 KB load
  static constexpr int N = ROWS / RPL, I = (N + WAVES - 1) / WAVES;  // loads: of the tile, of a wave
  const char* p[I];
  int col, w;
  static __device__ __forceinline__ int place(int m) { return STEP == 64 ? swz<64>(m) : (m >> 2) & 3; }
  template <typename RowPtr>
  __device__ __forceinline__ void init(int wave, int lane, RowPtr row_ptr) {
    w = wave;
    // place() repeats every 16 rows; with 8 rows a load it depends on the load's parity
    static_assert(STEP == 32 || (WAVES % 2 == 0 && N % 2 == 0), "a wave's loads are all odd or all even");
    col = 8 * (lane % CH ^ place(RPL * w + lane / CH));
#pragma unroll
    for (int i = 0; i < I; ++i) p[i] = (const char*)(row_ptr(RPL * ((w + WAVES * i) % N) + lane / CH) + col);
  }
  __device__ __forceinline__ void advance(long bytes) {
#pragma unroll
    for (int i = 0; i < I; ++i) p[i] += bytes;
  }
  // chunks of a step with `left` indices that are past the end
  __device__ __forceinline__ void stop(int left) {
#pragma unroll
    for (int i = 0; i < I; ++i) p[i] = col < left ? p[i] : (const char*)&zero_line;
  }
  // load i of the step the pointers stand at
  template <int i>
  __device__ __forceinline__ void load(bf16* tile) const {
    dma_lds16(p[i], lds_addr(tile + 512 * ((w + WAVES * i) % N)));
  }
  static __device__ __forceinline__ int frag(int lane, int v) {
    const int r = lane & 31, h = lane >> 5;
    return r * STEP + 8 * ((2 * v + h) ^ place(r));
  }
};

// Transposed operand: STEP contraction rows of COLS columns, in panels of 128
// (or one of 64).
template <int COLS, int STEP, int WAVES>
struct Transposed {
  static constexpr int PW = COLS < 128 ? COLS : 128, CH = PW / 8, RPL = 64 / CH;  // chunks of a row, rows of a load
  static constexpr int PER = STEP / RPL;  // loads of a panel
  static constexpr int N = COLS / PW * PER, I = (N + WAVES - 1) / WAVES;
  const char* p[I];  // column of load i in row 0 of `base`
  int row[I], w;
  __device__ __forceinline__ void init(int wave, int lane, const bf16* base, int ncols) {
    w = wave;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int q = (w + WAVES * i) % N;  // panel q / PER, rows RPL (q % PER) ..
      row[i] = RPL * (q % PER) + lane / CH;
      const int c = PW * (q / PER) + 8 * (lane % CH ^ swz<PW>(row[i]));
      p[i] = (const char*)(base + (c < ncols ? c : 0));
    }
  }
  // rows `ld` bytes apart: the pointers move to their load's own row
  __device__ __forceinline__ void own_rows(long ld) {
#pragma unroll
    for (int i = 0; i < I; ++i) p[i] += row[i] * ld;
  }
  __device__ __forceinline__ void advance(long bytes) {
#pragma unroll
    for (int i = 0; i < I; ++i) p[i] += bytes;
  }
  __device__ __forceinline__ void stop(int left) {
#pragma unroll
    for (int i = 0; i < I; ++i) p[i] = row[i] < left ? p[i] : (const char*)&zero_line;
  }
  template <int i>
  __device__ __forceinline__ void load(bf16* tile, unsigned long extra = 0) const {
    dma_lds16(p[i] + extra, lds_addr(tile + 512 * ((w + WAVES * i) % N)));
  }
  // element offset of 32-column block b's operand, contraction rows 8 h + 4 hi ..
  static __device__ __forceinline__ int frag(int lane, int b, int hi) {
    const int h = lane >> 5, i16 = lane & 15;
    return 32 * b / PW * STEP * PW +
           toff<PW>(8 * h + 4 * hi + (i16 >> 2), 32 * b % PW + (lane & 16) + 4 * (i16 & 3));
  }
};

__device__ __forceinline__ bf16x8 tr_pair(const bf16* lo, const bf16* hi) {
  const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)lo);
  const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t*)hi);
  return bf16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// The tokens of the contraction rows that one wave loads in a step: rows 4 w ..
// and, where a panel has more loads than there are waves, 4 (WAVES + w) .. (rows
// past the end: token 0, which adds nothing to the address of the line of
// zeros).  Scalar loads one step ahead of their use: a vector load's wait would
// also wait for the tiles in flight.
template <int WAVES, int STEP>
struct StepTokens {
  static constexpr bool TWO = STEP / 4 == 2 * WAVES;
  static_assert(TWO || STEP / 4 == WAVES, "a wave's loads cover one or two groups of four rows");
  i32x4 lo4, hi4;  // vectors, not arrays: those would be moved to LDS
  __device__ __forceinline__ void fetch(const int32_t* row_token, int lo, int k0, int len, int w) {
    typedef const __attribute__((address_space(4))) int32_t scalar_int;
    typedef int32_t quad __attribute__((ext_vector_type(4), aligned(4)));
    typedef const __attribute__((address_space(4))) quad scalar_quad;
    const uintptr_t src = (uintptr_t)(row_token + lo);
    const int k = k0 + 4 * w, last = len - 1;
    if (k0 + STEP <= len) {
      lo4 = *(scalar_quad*)(src + 4L * k);
      if constexpr (TWO) hi4 = *(scalar_quad*)(src + 4L * (k + 4 * WAVES));
    } else {
      auto at = [&](int q) {
        const int t = ((scalar_int*)src)[min(k + q, last)];
        return k + q < len ? t : 0;
      };
      lo4 = i32x4{at(0), at(1), at(2), at(3)};
      if constexpr (TWO) hi4 = i32x4{at(4 * WAVES), at(4 * WAVES + 1), at(4 * WAVES + 2), at(4 * WAVES + 3)};
    }
  }
  // of load i, this lane's row
  __device__ __forceinline__ int of(int i, int lane) const {
    const i32x4 v = TWO && (i & 1) ? hi4 : lo4;
    const int a = lane & 16 ? v[1] : v[0], b = lane & 16 ? v[3] : v[2];
    return lane & 32 ? b : a;
  }
};

// f(0), f(1), .. f(N - 1) with each index a compile-time constant: register
// arrays are then never indexed by a variable
template <typename F, int... J>
__device__ __forceinline__ void each_of(std::integer_sequence<int, J...>, F f) {
  (f(std::integral_constant<int, J>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  each_of(std::make_integer_sequence<int, N>{}, f);
}

template <int N>
__device__ __forceinline__ void wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(N) : "memory");
}

// Pairs of operands: with a second result, or in bwd_x a second product to add.
// (Without rows bwd_w's dy2 may be NULL where there is a dw2 to clear.)
template <int MODE>
__host__ __device__ __forceinline__ int pairs(const ExpertArgs& a) {
  return (MODE == kBwdX ? a.b2 : a.c2) != nullptr ? 2 : 1;
}

// A workgroup's tile: expert, its rows, first row and column of C.
struct GroupTile {
  int e, lo, len, m0, n0, part;
  bool any;
};

// Tile t of the launch: experts in order, each expert's ceil(len / BM) rows of
// tiles in bands of kBand rows, a band column by column (`cols` columns).  The
// 32 large tiles that an XCD runs at once then share kBand tiles of rows and
// eight columns of the weights.  A wave adds up the experts' tile rows, a range
// of experts a lane, and finds the range that holds t.
// The workgroups of one XCD (blockIdx modulo 8) take consecutive tiles, which
// share an expert's weights and rows in its L2.
//
// Group e is [M(e), M(e + 1)) with M the running maximum of the offsets, clamped
// into [0, rows]: groups of any offsets at all are apart, and their tiles no more
// than the launch has.  Offsets in order, as one ballot tells, are their own M.
template <int BM>
__device__ __forceinline__ GroupTile find_tile(const ExpertArgs& a, int cols, int lane) {
  const int per = (a.E + 63) / 64;
  auto offset = [&](int e) { return clampi(a.offsets[e], 0, a.rows); };
  // tile rows of this lane's experts, and their last M; `lo`: M of the expert before
  // them, or less where that is no larger than their first offset
  auto count = [&](int lo, int& top, bool& sorted) {
    const int e0 = lane * per;
    int tiles = 0, first = offset(min(e0, a.E));
    lo = max(lo, first);
#pragma unroll 4
    for (int q = 1; q <= per; ++q) {
      const int next = offset(min(e0 + q, a.E)), hi = max(lo, next);
      sorted &= next >= first;
      tiles += (hi - lo + BM - 1) / BM;
      lo = hi;
      first = next;
    }
    top = lo;
    return tiles;
  };
  int before = 0, top;
  bool sorted = true;
  int mine = count(0, top, sorted);
  if (__ballot(!sorted) != 0) {
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(top, o);
      if (lane >= o) top = max(top, v);
    }
    before = __shfl_up(top, 1);
    if (lane == 0) before = 0;
    mine = count(before, top, sorted);
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
  const int owner = __builtin_ctzll(__ballot((long)upto * cols > t));
  long left = t - (long)__builtin_amdgcn_readlane(upto - mine, owner) * cols;
  int next = max(__builtin_amdgcn_readlane(before, owner), offset(owner * per));
  for (g.e = owner * per; g.e < a.E; ++g.e) {
    g.lo = next;
    next = max(g.lo, offset(g.e + 1));
    g.len = next - g.lo;
    const int mt = (g.len + BM - 1) / BM;
    if (left < (long)mt * cols) {
      const int band = (int)(left / (kBand * cols)), in = (int)(left % (kBand * cols));
      const int high = min(kBand, mt - band * kBand);
      g.m0 = (band * kBand + in % high) * BM;
      g.n0 = in / high;  // column of tiles; the caller turns it into columns
      return g;
    }
    left -= (long)mt * cols;
  }
  g.any = false;
  return g;
}

// first row of group e, M(e) as above
__device__ __forceinline__ int group_start(const ExpertArgs& a, int e, int lane) {
  const int own = clampi(a.offsets[e], 0, a.rows);
  int most = own;
#pragma unroll 4
  for (int q = 0; q < e; q += 64) most = max(most, clampi(a.offsets[min(q + lane, e)], 0, a.rows));
  if (__ballot(most > own) == 0) return own;
  for (int o = 32; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o));
  return __builtin_amdgcn_readfirstlane(most);
}

// an XCD's tiles of an expert in bwd_w
__host__ __device__ __forceinline__ int bwd_w_share(int tiles) { return (tiles + kXcds - 1) / kXcds; }

// TOKENS: the contraction rows of bwd_w are gathered
template <int MODE, int BM, int BN, int MW, int NW, int STEP, int RING, bool TOKENS>
__global__ __launch_bounds__(64 * MW * NW, 2) void experts_kernel(ExpertArgs a) {
  constexpr int WAVES = MW * NW, MI = BM / 32 / MW, NI = BN / 32 / NW;
  constexpr bool A_TR = MODE == kBwdW, B_TR = MODE != kBwdX;
  constexpr int A_ELEMS = BM * STEP, B_ELEMS = BN * STEP, SLICES = STEP / 16;
  constexpr int IA = (BM * STEP / 512 + WAVES - 1) / WAVES, IB = (BN * STEP / 512 + WAVES - 1) / WAVES;
  constexpr int LOADS = IA + IB;  // a wave's loads of a step
  // of which so many are issued in the last slice, the others in the next step's first
  constexpr int EARLY = STEP == 64 ? LOADS / 2 : LOADS;
  constexpr int OUT_STRIDE = NI * 32 + 8;  // staged output rows, 16 bytes apart in banks
  constexpr int SMEM = RING * (A_ELEMS + B_ELEMS);  // elements: the A tiles, then the B tiles
  static_assert(WAVES * 32 * OUT_STRIDE <= SMEM, "the output staging fits the ring");
  __shared__ __attribute__((aligned(1024))) bf16 smem[SMEM];
  const int lane = threadIdx.x & 63, w = wave_id(), wm = w / NW, wn = w % NW;
  const int r = lane & 31, h = lane >> 5;
  // columns of C, and of tiles: C is [rows, out_width], [rows, in_width] or [in_width, out_width]
  const int ncols = MODE == kBwdX ? a.in_width : a.out_width;
  const int tiles_n = (ncols + BN - 1) / BN, parts = pairs<MODE>(a);

  GroupTile g;
  if constexpr (MODE == kBwdW) {
    // Every XCD takes an eighth of every expert's tiles, because an expert's
    // tiles take as long as it has rows; the eighths turn with the expert, so
    // that short last ones meet every XCD.  (Whole experts per XCD: 18% of the
    // time idle at 128 experts of unequal sizes, 49% at eight.)
    const int tiles_m = (a.in_width + BM - 1) / BM, cols = tiles_n * parts, per = bwd_w_share(tiles_m * cols);
    const int xcd = blockIdx.x % kXcds, at = blockIdx.x / kXcds;
    g.e = at / per;
    const int left = (xcd + g.e) % kXcds * per + at % per;
    if (left >= tiles_m * cols) return;
    const int band = left / (kBand * cols), in = left % (kBand * cols), high = min(kBand, tiles_m - band * kBand);
    g.m0 = (band * kBand + in % high) * BM;
    g.n0 = in / high % tiles_n * BN;
    g.part = in / high / tiles_n;
    if (!a.overwrite && a.offsets[g.e + 1] <= a.offsets[g.e]) return;  // M(e) is no smaller
    g.lo = group_start(a, g.e, lane);
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
  const int steps1 = (depth + STEP - 1) / STEP;
  const int steps = MODE == kBwdX ? steps1 * parts : steps1;
  const size_t wsize = (size_t)a.in_width * a.out_width;

  const bool gathers = MODE == kBwdW ? TOKENS : MODE == kFwd && a.row_token != nullptr;

  // ---- operands
  typedef Natural<BM, STEP, WAVES> NatA;
  typedef Natural<BN, STEP, WAVES> NatB;
  typedef Transposed<BM, STEP, WAVES> TrA;
  typedef Transposed<BN, STEP, WAVES> TrB;
  NatA an;
  TrA at;
  NatB bn;
  TrB bt;
  // pointers at the first step of a part
  auto start = [&](int part) {
    if constexpr (!A_TR) {
      an.init(w, lane, [&](int m) {
        const int row = g.lo + g.m0 + min(m, mrows - 1);
        long src = row;
        if (gathers) src = clampi(a.row_token[row], 0, a.x_rows - 1);
        return (const bf16*)(part ? a.a2 : a.a) + src * depth;
      });
    } else {
      at.init(w, lane, (const bf16*)a.a + g.m0 + (gathers ? 0 : (size_t)g.lo * a.in_width), mrows);
      if (!gathers) at.own_rows(2L * a.in_width);
    }
    if constexpr (!B_TR) {
      bn.init(w, lane, [&](int n) {
        return (const bf16*)(part ? a.b2 : a.b) + g.e * wsize + (size_t)min(g.n0 + n, ncols - 1) * a.out_width;
      });
    } else {
      const size_t row0 = MODE == kFwd ? (size_t)g.e * a.in_width : (size_t)g.lo;
      bt.init(w, lane, (const bf16*)(g.part ? a.b2 : a.b) + row0 * a.out_width + g.n0, ncols - g.n0);
      bt.own_rows(2L * a.out_width);
    }
  };
  start(0);
  StepTokens<TOKENS ? WAVES : 8, TOKENS ? STEP : 32> tok;
  if constexpr (TOKENS)
    if (steps > 0) tok.fetch(a.row_token, g.lo, 0, g.len, w);
  // The pointers stand at the next step to issue; tok holds its tokens.
  const long a_step = A_TR ? 2L * STEP * a.in_width : 2L * STEP;
  const long b_step = B_TR ? 2L * STEP * a.out_width : 2L * STEP;
  auto gathered = [&](int i) -> unsigned long {  // bytes to the row of load i's token
    if constexpr (!TOKENS) return 0;
    return (unsigned long)(unsigned)clampi(tok.of(i, lane), 0, a.x_rows - 1) * (2u * a.in_width);
  };
  // load j of the LOADS of a step into buffer b of the ring
  auto load = [&](auto index, auto buffer) {
    constexpr int j = decltype(index)::value, b = decltype(buffer)::value;
    bf16* ta = smem + b * A_ELEMS;
    bf16* tb = smem + RING * A_ELEMS + b * B_ELEMS;
    if constexpr (j < IA) {
      if constexpr (A_TR)
        at.template load<j>(ta, gathered(j));
      else
        an.template load<j>(ta);
    } else {
      if constexpr (B_TR)
        bt.template load<j - IA>(tb);
      else
        bn.template load<j - IA>(tb);
    }
  };
  // Points the loads at step s, whose predecessor they stood at.  Past the last
  // index they read zeros: the last step of a part that is not whole, and the
  // steps behind the last one, which the loop issues like all others.
  auto aim = [&](int s) {
    const bool second = MODE == kBwdX && s >= steps1;
    const int left = s < steps ? depth - (second ? s - steps1 : s) * STEP : 0;
    if (MODE == kBwdX && s == steps1 && s < steps) start(1);
    if (left < STEP) {
      asm volatile("");  // stays a branch: as selects it would run every step
      if constexpr (A_TR)
        at.stop(left);
      else
        an.stop(left);
      if constexpr (B_TR)
        bt.stop(left);
      else
        bn.stop(left);
    }
  };
  auto advance = [&](int s) {
    if constexpr (!A_TR)
      an.advance(a_step);
    else if constexpr (!TOKENS)
      at.advance(a_step);
    else
      tok.fetch(a.row_token, g.lo, s * STEP, g.len, w);
    if constexpr (!B_TR)
      bn.advance(b_step);
    else
      bt.advance(b_step);
    aim(s);
  };

  // ---- addresses of the operand reads in the first buffer: a natural one's per
  // slice, a transposed one's per 32-column block and row quad.  The buffer, the
  // slice's rows and the block add a constant.
  const char *aptr[A_TR ? 2 : SLICES][A_TR ? MI : 1], *bptr[B_TR ? 2 : SLICES][B_TR ? NI : 1];
  const bf16* tb0 = smem + RING * A_ELEMS;
  if constexpr (A_TR)
    each<2 * MI>([&](auto q) { aptr[q / MI][q % MI] = (const char*)(smem + TrA::frag(lane, q % MI * MW + wm, q / MI)); });
  else
    each<SLICES>([&](auto v) { aptr[v][0] = (const char*)(smem + NatA::frag(lane, v) + wm * 32 * STEP); });
  if constexpr (B_TR)
    each<2 * NI>([&](auto q) { bptr[q / NI][q % NI] = (const char*)(tb0 + TrB::frag(lane, wn * NI + q % NI, q / NI)); });
  else
    each<SLICES>([&](auto v) { bptr[v][0] = (const char*)(tb0 + NatB::frag(lane, v) + wn * NI * 32 * STEP); });

  f32x16 acc[NI][MI];
#pragma unroll
  for (int n = 0; n < NI; ++n)
#pragma unroll
    for (int m = 0; m < MI; ++m) acc[n][m] = zero16();

  // Operands are read one slice (16 contraction indices) ahead of the products.
  // The barrier stands before a step's last slice: by then every wave has read
  // the whole step, so its buffer takes step s + RING at once, and the next
  // step, whose loads are waited for there, is read while the last slice's
  // products run.
  if (steps > 0) {
    aim(0);
    each<RING>([&](auto s) {
      each<LOADS>([&](auto j) {
        if constexpr (s < RING - 1 || j < EARLY) load(j, s);
      });
      if constexpr (s < RING - 1) advance(s + 1);
    });
  }
  auto sweep = [&](auto active) {
    constexpr int ACT = decltype(active)::value;
    bf16x8 fb[2][NI], fa[2][ACT > 0 ? ACT : 1];
    constexpr int FRAGS = ACT > 0 ? ACT + NI : 0, PRODUCTS = ACT * NI;
    constexpr int MOST = PRODUCTS > FRAGS ? PRODUCTS : FRAGS, MOST2 = MOST > LOADS ? MOST : LOADS;
    // fragment j of slice v, in the order of use: b0 a0 b1 .. then the other a
    auto read = [&](auto buffer, auto slice, auto index) {
      constexpr int v = decltype(slice)::value, j = decltype(index)::value;
      constexpr int ta = 2 * A_ELEMS * decltype(buffer)::value, tb = 2 * B_ELEMS * decltype(buffer)::value;
      if constexpr (j != 1 && j <= NI) {
        constexpr int n = j == 0 ? 0 : j - 1;
        if constexpr (B_TR)
          fb[v & 1][n] = tr_pair((const bf16*)(bptr[0][n] + tb + v * 32 * TrB::PW), (const bf16*)(bptr[1][n] + tb + v * 32 * TrB::PW));
        else
          fb[v & 1][n] = *(const bf16x8*)(bptr[v][0] + tb + n * 64 * STEP);
      } else {
        constexpr int m = j == 1 ? 0 : j - NI;
        if constexpr (A_TR)
          fa[v & 1][m] = tr_pair((const bf16*)(aptr[0][m] + ta + v * 32 * TrA::PW), (const bf16*)(aptr[1][m] + ta + v * 32 * TrA::PW));
        else
          fa[v & 1][m] = *(const bf16x8*)(aptr[v][0] + ta + m * MW * 64 * STEP);
      }
    };
    auto multiply = [&](auto slice, auto index) {
      constexpr int v = decltype(slice)::value, m = decltype(index)::value / NI, n = decltype(index)::value % NI;
      acc[n][m] = mfma32(fb[v & 1][n], fa[v & 1][m], acc[n][m]);
    };
    const std::integral_constant<int, 0> first{};
    const std::integral_constant<int, SLICES - 1> last{};
    if (steps == 0) return;
    wait_barrier<(RING - 2) * LOADS + EARLY>();
    each<FRAGS>([&](auto j) { read(first, first, j); });
    // one round of the ring: a buffer's offset is part of each read instruction
    for (int s = 0; s < steps;) {
      each<RING>([&](auto buffer) {
        if (s >= steps) return;
        constexpr int b = decltype(buffer)::value;
        const std::integral_constant<int, b + 1 < RING ? b + 1 : 0> next{};
        const std::integral_constant<int, (b + RING - 1) % RING> previous{};
        // each product is followed by a read of the next slice, and in the first
        // one by a load of the second half of step s + RING - 1
        each<SLICES - 1>([&](auto v) {
          each<MOST2>([&](auto j) {
            if constexpr (j < PRODUCTS) multiply(v, j);
            if constexpr (j < FRAGS) read(buffer, std::integral_constant<int, v + 1>{}, j);
            if constexpr (v == 0 && EARLY + j < LOADS) load(std::integral_constant<int, EARLY + j>{}, previous);
            __builtin_amdgcn_sched_barrier(0);
          });
          if constexpr (v == 0) advance(s + RING);
        });
        wait_barrier<(RING - 2) * LOADS>();
        // in the last one by a load of the first half of step s + RING
        each<MOST2>([&](auto j) {
          if constexpr (j < PRODUCTS) multiply(last, j);
          if constexpr (j < FRAGS) read(next, first, j);
          if constexpr (j < EARLY) load(j, buffer);
          __builtin_amdgcn_sched_barrier(0);
        });
        ++s;
      });
    }
  };
  switch (act) {
    case 0: sweep(std::integral_constant<int, 0>{}); break;
    case 1: sweep(std::integral_constant<int, 1>{}); break;
    case 2: sweep(std::integral_constant<int, MI < 2 ? MI : 2>{}); break;
    case 3: sweep(std::integral_constant<int, MI < 3 ? MI : 3>{}); break;
    default: sweep(std::integral_constant<int, MI>{}); break;
  }

  // ---- C: lane (r, h) holds row r of a 32-row block, columns 8 i + 4 h .. + 3
  if constexpr (MODE == kBwdW) {
    // through LDS, so that a row's 64 columns leave as two whole lines
    wait_barrier<0>();
    constexpr int PAD = NI * 32 + 4;
    static_assert(WAVES * 32 * PAD * 2 <= SMEM, "the output staging fits the ring");
    float* out = (float*)smem + w * 32 * PAD;
    float* c = (float*)(g.part ? a.c2 : a.c) + g.e * wsize;
    constexpr int CH = NI * 8;  // 16-byte chunks of a row
    constexpr int PER = 32 * CH / 64;  // chunks of a lane in a block of 32 rows
    f32x4 old[2][PER];  // what the sums are added to, read a block ahead
    auto place = [&](int m, int q, bool& inside) {
      const int at = lane + 64 * q, row = g.m0 + 32 * (m * MW + wm) + at / CH, col = g.n0 + 32 * wn * NI + 4 * (at % CH);
      inside = row < a.in_width && col < ncols;
      return (f32x4*)(c + (size_t)row * a.out_width + col);
    };
    auto fetch = [&](auto block) {
      each<PER>([&](auto q) {
        bool inside;
        const f32x4* src = place(block, q, inside);
        if (inside) old[block & 1][q] = *src;
      });
    };
    if (!a.overwrite) fetch(std::integral_constant<int, 0>{});
    each<MI>([&](auto block) {
      constexpr int m = decltype(block)::value;
      if (m >= act) return;
      if constexpr (m + 1 < MI)
        if (!a.overwrite) fetch(std::integral_constant<int, m + 1>{});
      each<NI * 4>([&](auto q) {
        constexpr int n = q / 4, i = q % 4;
        *(f32x4*)(out + r * PAD + 32 * n + 8 * i + 4 * h) =
            f32x4{acc[n][m][4 * i], acc[n][m][4 * i + 1], acc[n][m][4 * i + 2], acc[n][m][4 * i + 3]};
      });
      __builtin_amdgcn_wave_barrier();
      each<PER>([&](auto q) {
        const int at = lane + 64 * q;
        const f32x4 v = *(const f32x4*)(out + at / CH * PAD + 4 * (at % CH));
        bool inside;
        f32x4* dst = place(m, q, inside);
        // written once and not read again here: past the caches, which keeps the
        // operands in them (128 experts of 2048 x 768: 735 -> 600 us)
        if (inside) __builtin_nontemporal_store(a.overwrite ? v : v + old[m & 1][q], dst);
      });
      __builtin_amdgcn_wave_barrier();
    });
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

template <int MODE, int BM, int BN, int MW, int NW, int STEP, int RING, bool TOKENS = false>
hipError_t launch_tiles(const ExpertArgs& a, hipStream_t st) {
  const int ncols = MODE == kBwdX ? a.in_width : a.out_width, parts = pairs<MODE>(a);
  const long tiles_n = (ncols + BN - 1) / BN;
  long grid;
  if (MODE == kBwdW) {
    grid = (long)kXcds * a.E * bwd_w_share((int)(parts * tiles_n * ((a.in_width + BM - 1) / BM)));
  } else {
    // at most a partial tile of rows for every expert that has any
    const long some = a.E < a.rows ? a.E : a.rows;
    grid = (MODE == kFwd ? parts : 1) * tiles_n * ((a.rows + some * (BM - 1)) / BM);
  }
  grid = (grid + kXcds - 1) / kXcds * kXcds;
  if (grid * (64L * MW * NW) > (long)UINT32_MAX) return hipErrorInvalidConfiguration;  // threads of a launch
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL((experts_kernel<MODE, BM, BN, MW, NW, STEP, RING, TOKENS>), dim3((unsigned)grid), dim3(64 * MW * NW),
                     0, st, a);
  return hipGetLastError();
}

// Which tiles.  A launch of 256 x 256 tiles runs one workgroup a CU, one of 128 x
// 128 tiles two; the latter's CU does 0.68 of the work in a tile's time (dense
// 1010 against 1205 TFLOP/s, and more rows and weights read).  Rounds are
// counted from the rows' average, a good half tile of padding per expert that has
// rows; half a round is added for the last one where there are several.
// Measured 256 / 128, us: 128 experts of 2048 x 768 top-8, forward, tokens 1024
// 195 / 171, 2045 207 / 213 (128 is taken), 4096 269 / 306, 8192 432 / 530; eight of 4096 x
// 1536 top-2, 300 tokens, forward 91 / 62, row gradients 74 / 60; 1000 tokens 97
// / 85 and 86 / 118.
bool small_tiles(const ExpertArgs& a, int cols_of_c, int parts) {
  const long some = std::min(a.E, a.rows);
  auto cost = [&](long tile, long slots) {
    const long high = std::max(some, a.rows / tile + some * 11 / 20);
    const double rounds = (double)(high * ((cols_of_c + tile - 1) / tile) * parts) / (double)slots;
    return rounds <= 1. ? 1. : rounds + 0.5;
  };
  return 0.68 * cost(128, 512) < cost(256, 256);
}
// Few rows an expert: the weights are all there is to read, and tiles of 32 rows
// and 64 columns, three workgroups of two waves a CU, put more of their loads in
// flight.  Up to four rows on average, or up to 16 where 128 x 128 tiles leave
// CUs idle.  Measured 128 x 128 / 32 x 64, us: 128 experts of 2048 x 768 top-8,
// forward, tokens 1 22 / 11.5, 4 38 / 36, 64 125 / 118, 256 140 / 151; eight of
// 4096 x 1536 top-2, 1 token 38 / 16, 32 tokens 60 / 50; 60 of 1024 x 512 top-4,
// 100 tokens 23.0 / 24.8.
bool few_rows(const ExpertArgs& a, int cols_of_c, int parts) {
  if ((long)a.rows <= 4L * a.E) return true;
  return (long)a.rows <= 16L * a.E && (long)std::min(a.E, a.rows) * ((cols_of_c + 127) / 128) * parts <= 256;
}

template <int MODE>
hipError_t launch_rows_of(const ExpertArgs& a, int cols_of_c, int parts, hipStream_t st) {
  if (few_rows(a, cols_of_c, parts)) return launch_tiles<MODE, 32, 64, 1, 2, 64, 4>(a, st);
  if (small_tiles(a, cols_of_c, parts)) return launch_tiles<MODE, 128, 128, 2, 2, 64, 2>(a, st);
  return launch_tiles<MODE, 256, 256, 2, 4, 64, 2>(a, st);
}

template <bool TOKENS>
hipError_t launch_bwd_w(const ExpertArgs& a, hipStream_t st) {
  // An expert's tiles of C do not depend on its rows.  Half the chip or less in
  // 256 x 256 tiles, or little more than the writes to do: 128 x 128 ones.
  // Measured 256 / 128, us: four experts of 1024 x 1024, 8192 rows each 242 / 203;
  // 60 of 1024 x 512, 67 rows each 58 / 50, 533 rows each 116 / 115; 64 of 2560 x
  // 1280, 384 rows each 582 / 643.
  const long tiles = (long)a.E * pairs<kBwdW>(a) * ((a.in_width + 255) / 256) * ((a.out_width + 255) / 256);
  if (tiles <= 128 || a.rows / a.E < 100) return launch_tiles<kBwdW, 128, 128, 2, 2, 32, 3, TOKENS>(a, st);
  // gathered rows: longer steps, which fetch their tokens half as often
  if constexpr (TOKENS)
    return launch_tiles<kBwdW, 256, 256, 2, 4, 64, 2, true>(a, st);
  else
    return launch_tiles<kBwdW, 256, 256, 2, 4, 32, 3, false>(a, st);
}

}  // namespace

hipError_t launch_experts_fwd(const ExpertArgs& a, hipStream_t st) {
  ProfileScope ps("experts_fwd", st);
  return launch_rows_of<kFwd>(a, a.out_width, pairs<kFwd>(a), st);
}
hipError_t launch_experts_bwd_x(const ExpertArgs& a, hipStream_t st) {
  ProfileScope ps("experts_bwd_x", st);
  return launch_rows_of<kBwdX>(a, a.in_width, 1, st);
}
hipError_t launch_experts_bwd_w(const ExpertArgs& a, hipStream_t st) {
  ProfileScope ps("experts_bwd_w", st);
  return a.row_token != nullptr ? launch_bwd_w<true>(a, st) : launch_bwd_w<false>(a, st);
}

}  // namespace spr
