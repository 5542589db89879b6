// Kernels of the experts' products for one type of element, included by one source a type.
//
// Every product is C[m, n] = sum_k A(m, k) B(n, k) on the matrix cores, in tiles of BM x BN with
// the operands staged through LDS 128 bytes of k at a time.  An operand lies in memory either
// with k contiguous (its rows are m or n) or with m or n contiguous (its rows are k); the second
// is transposed while it is read from LDS.
//   h  = x w1^T      rows: an expert's pairs, x gathered      -> act = silu(gate) up, (pre)
//   y  = act w2^T                                             -> y, then joined by token
//   da = dout w2     dout gathered; pre                       -> dpre, wact, parts of dweights
//   dx = dpre w1                                              -> dxr, then joined by token
//   dw1 = dpre^T x,  dw2 = dout^T wact       k: an expert's pairs
// act, dpre and wact are rounded to the type of the elements, as the matrix cores take operands of
// one type and binary32 ones at an eighth of the rate (0.153 to 1.28 PFLOP/s in large products): a
// result has the error of one more rounding, and in f16 the range of that type.  Sums, the first
// product's results for the backward pass, and the rows that are joined by token are binary32.
#pragma once

#include "experts.h"

#include <type_traits>

#pragma clang fp contract(fast)

namespace gsn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int64_t kFewTokens = 2;    // for which one launch makes the second product and the sum
// pairs up to which weights go straight into fragments; a workgroup lists that many at most
template <typename T>
constexpr int64_t kFewPairs = sizeof(T) == 4 ? 768 : 256;
constexpr int kRowBytes = 128;  // bytes of k (contiguous operands) in a stage

// 16 bytes of an operand in a lane: 8 or 4 values of k of row (lane & 15)
union Frag {
  u32x4 u;
  bf16x8 b;
  f16x8 h;
  f32x4 f;
  s16x4 s[2];
};

// acc[i] += sum over the fragment's k of n-row (lane >> 4) * 4 + i and m-row lane & 15; of a 4-byte
// type part q of four, so that products of one sum do not wait for each other.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 4 : 1;
template <typename T>
__device__ __forceinline__ f32x4 multiply(const Frag& n, const Frag& m, f32x4 acc, int q) {
  if constexpr (sizeof(T) == 4)
    return __builtin_amdgcn_mfma_f32_16x16x4f32(n.f[q], m.f[q], acc, 0, 0, 0);
  else if constexpr (__is_same(T, bf16_t))
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(n.b, m.b, acc, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(n.h, m.h, acc, 0, 0, 0);
}

// Place of 16-byte chunk c in row r of a staged operand with k contiguous (8 chunks a row): the
// 16 rows that a quarter wave reads at one k fall on different banks.
__device__ __forceinline__ int chunk_k(int r, int c) { return c ^ ((r >> 1) & 7); }
// The same with k as the row: the 4 (2-byte types) or 1 rows that 16 lanes read 32 or 64 bytes
// of, and those of the wave's other quarters, fall on different banks.
template <typename T, int CHUNKS = 16>  // CHUNKS of a row, at least
__device__ __forceinline__ int chunk_n(int k, int c) {
  if constexpr (sizeof(T) == 2 && CHUNKS < 16) return c ^ ((k & 3) << 1);
  else if constexpr (sizeof(T) == 2) return c ^ (((k & 3) | ((k >> 1) & 4)) << 1);
  else return c ^ (((k >> 2) & 3) << 2);
}

// Fragment of 16 rows at `r0` and the s-th half of a stage's k; R rows (k contiguous) or columns
// (k as the row) in all.
template <typename T, bool TR, int R>
__device__ __forceinline__ Frag fragment(const char* tile, int r0, int s, int lane) {
  const int g = lane >> 4, i = lane & 15;
  Frag f;
  if constexpr (!TR) {
    const int r = r0 + i;
    f.u = *reinterpret_cast<const u32x4*>(tile + r * kRowBytes + chunk_k(r, 4 * s + g) * 16);
  } else if constexpr (sizeof(T) == 2) {
    // Each 16 lanes read 4 rows of k, 16 columns wide, and get them column by column.
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int k = 32 * s + 8 * g + 4 * j + (i >> 2);
      const int col = r0 + (i & 3) * 4;
      const char* p = tile + (k * R + (chunk_n<T, R / 8>(k, col >> 3) << 3) + (col & 7)) * 2;
      f.s[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)(p));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = 16 * s + 4 * g + j;
      const int col = r0 + i;
      f.f[j] = *reinterpret_cast<const float*>(
          tile + (k * R + (chunk_n<T>(k, col >> 2) << 2) + (col & 3)) * 4);
    }
  }
  return f;
}

// Four results of a row at column n, N columns in all.  Rows start at any element.
template <typename T>
struct LooseOf {
  typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};
template <typename T>
__device__ __forceinline__ void store4(T* row, int32_t n, int32_t N, const float* v) {
  if (n + 4 <= N) {
    typename LooseOf<T>::type o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = from_float<T>(v[i]);
    *reinterpret_cast<typename LooseOf<T>::type*>(row + n) = o;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < N) row[n + i] = from_float<T>(v[i]);
}
template <typename T>
__device__ __forceinline__ void load4(const T* row, int32_t n, int32_t N, float* v) {
  if (n + 4 <= N) {
    const auto o = *reinterpret_cast<const typename LooseOf<T>::type*>(row + n);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_float(o[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = n + i < N ? to_float(row[n + i]) : 0.0f;
}

// What the backward pass makes of d = dout . w2 at a pair's gate and up: the gradients of both,
// the activation times the pair's weight, and the term of the weight's gradient.
struct Gated {
  float dg, du, wa, dot;
};
__device__ __forceinline__ Gated gated(float d, float g, float u, float w) {
  const float s = sigmoid(g), sg = g * s, act = sg * u;
  // silu' = s (1 + g (1 - s)), 1 - s without the cancellation
  return Gated{w * d * u * (s + sg * sigmoid(-g)), w * d * sg, w * act, d * act};
}

// Results of a tile: rows m0 + 0 .. mrows - 1 of the weights' products, or rows row0 + 0 .. of
// the others; columns from n0.  Uses WN * BM floats of LDS.
template <typename T, Kind KIND, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void finish(const Experts& x, f32x4 (&acc)[BM / WM / 16][BN / WN / 16],
                                       float* dot, int32_t e, int32_t m0, int32_t mrows,
                                       int32_t n0, int64_t row0) {
  constexpr int kThr = WM * WN * kWave, MT = BM / WM / 16, NT = BN / WN / 16;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int wm = wave / WN, wn = wave % WN;
  const int32_t D = x.dim, F = x.hidden;
  const int32_t N = KIND == kForwardGate || KIND == kBackwardGate || KIND == kWeightsOut ? F : D;
  // a lane's results: row m = lane & 15 of each 16, columns n = (lane >> 4) * 4 + 0..3
  const int li = lane & 15, lg = (lane >> 4) * 4;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int32_t m = wm * (BM / WM) + i * 16 + li;
    const bool live = m < mrows;
    float part = 0.0f;
    if (live) {
      if constexpr (KIND == kForwardGate) {
#pragma unroll
        for (int j = 0; j < NT / 2; ++j) {
          const int32_t f = n0 + wn * (BN / WN / 2) + j * 16 + lg;
          float g[4], u[4], v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            g[q] = acc[i][j][q];
            u[q] = acc[i][j + NT / 2][q];
            v[q] = g[q] * sigmoid(g[q]) * u[q];
          }
          store4(static_cast<T*>(x.act) + (row0 + m) * F, f, F, v);
          if (x.pre) {
            store4(x.pre + (row0 + m) * 2 * F, f, F, g);
            store4(x.pre + (row0 + m) * 2 * F + F, f, F, u);
          }
        }
      } else if constexpr (KIND == kBackwardGate) {
        const float w = x.weights[x.plan.rows[row0 + m]];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int32_t f = n0 + wn * (BN / WN) + j * 16 + lg;
          float g[4], u[4], dg[4], du[4], wa[4];
          load4(x.pre + (row0 + m) * 2 * F, f, F, g);
          load4(x.pre + (row0 + m) * 2 * F + F, f, F, u);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const Gated r = gated(acc[i][j][q], g[q], u[q], w);
            part += f + q < F ? r.dot : 0.0f;
            wa[q] = r.wa;
            du[q] = r.du;
            dg[q] = r.dg;
          }
          store4(static_cast<T*>(x.wact) + (row0 + m) * F, f, F, wa);
          store4(static_cast<T*>(x.dpre) + (row0 + m) * 2 * F, f, F, dg);
          store4(static_cast<T*>(x.dpre) + (row0 + m) * 2 * F + F, f, F, du);
        }
      } else {
        constexpr bool kF32 = KIND == kForwardOut || KIND == kBackwardIn;
        float* const c32 = KIND == kForwardOut ? x.y : x.dxr;
        T* const ct = static_cast<T*>(KIND == kWeightsIn ? x.dw1 : x.dw2);
        const int64_t M = KIND == kWeightsIn ? 2 * F : D;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int32_t n = n0 + wn * (BN / WN) + j * 16 + lg;
          float v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = acc[i][j][q];
          if constexpr (kF32) store4(c32 + (row0 + m) * N, n, N, v);
          else store4(ct + (e * M + m0 + m) * N, n, N, v);
        }
      }
    }
    if constexpr (KIND == kBackwardGate) {
      part += __shfl_xor(part, 16);
      part += __shfl_xor(part, 32);
      if (lane < 16) dot[wn * BM + m] = part;
    }
  }
  if constexpr (KIND == kBackwardGate) {
    __syncthreads();
    for (int32_t m = tid; m < BM && m < mrows; m += kThr) {
      float s = 0.0f;
#pragma unroll
      for (int q = 0; q < WN; ++q) s += dot[q * BM + m];
      x.dots[(row0 + m) * x.dot_tiles + n0 / BN] = s;
    }
  }
}

// 16 zero bytes that lanes load where an operand has no more k
__device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};

// A lane's 16 bytes of a row of K elements at k, zeros past its end (INSIDE: there is none in
// them).  Rows start at any element.
template <bool INSIDE, typename T>
__device__ __forceinline__ Frag row_chunk(const T* row, int32_t k, int32_t K) {
  constexpr int kE = 16 / sizeof(T);
  typedef T Loose __attribute__((ext_vector_type(kE), aligned(sizeof(T))));
  Frag f;
  if (INSIDE || k + kE <= K) {
    // (said to be global: a pointer chosen between two is taken for any, whose loads LDS reads wait
    // for)
    f.u = __builtin_bit_cast(u32x4, *(const __attribute__((address_space(1))) Loose*)(row + k));
  } else {
    Vec<T, kE> v;
#pragma unroll
    for (int j = 0; j < kE; ++j) v.v[j] = k + j < K ? row[k + j] : from_float<T>(0.0f);
    f.u = __builtin_bit_cast(u32x4, v);
  }
  return f;
}

// Workgroups go round the 8 XCDs.  Runs of `run` tiles go to one XCD, where the tiles that its CUs
// work on at a time share operands through its L2; the next run goes to the next XCD.
// Fewer tiles than 8 runs are dealt out evenly.  -1: no tile for this workgroup (for any of them,
// where no pair has an expert and there are no tiles).
__device__ __forceinline__ int32_t spread(int32_t block, int32_t total, int32_t run) {
  if (total <= 0) return -1;
  if (total < 8 * run) run = (total + 7) / 8;
  const int32_t in = block >> 3;
  const int32_t id = (in / run * 8 + (block & 7)) * run + in % run;
  return id < total ? id : -1;
}
// Place of a tile in a block of tiles_m x tiles_n, taken TALL tiles of m by all of n at a time, m
// first: 32 tiles in a row, 4 x 8, have 4 + 8 tiles of operands.
template <int32_t TALL>
__device__ __forceinline__ int2 tile_place(int32_t id, int32_t tiles_m, int32_t tiles_n) {
  const int32_t g = id / (TALL * tiles_n), in = id - g * TALL * tiles_n;
  const int32_t left = tiles_m - g * TALL, tall = left < TALL ? left : TALL;
  return int2{g * TALL + in % tall, in / tall};
}
// Runs of the large tiles, one a CU, and of the middle ones, two a CU; small ones go round in order
// (runs of 128 in blocks of 8 x 16 gained 2% on 32,768 pairs and lost up to 50% on small products).
// Middle tiles in order, in runs of 16 and of 64, us: 16,384 tokens, 2 of 32 experts, 2,047 x
// 2,047: 5,353, 5,252, 5,318; forward of 8,192, 4 of 32, 777 x 1,501: 609, 556, 550; 4,096, 2 of
// 16, 1,023 x 1,023: 535, 533, 594.
template <int SIDE>
constexpr int32_t kTall = SIDE == kSmallRows ? 1 : 4;
template <int SIDE>
constexpr int32_t kRun = tile_run(SIDE);

// Gradients of the weights of the pairs from j on, one a thread: the sums of their parts.
__device__ __forceinline__ void sum_dots(const Experts& x, int64_t j) {
  j += threadIdx.x;
  if (j >= x.pairs) return;
  const int32_t r = x.plan.pos[j];
  float s = 0.0f;
  if (r >= 0)
    for (int i = 0; i < x.dot_tiles; ++i) s += x.dots[static_cast<int64_t>(r) * x.dot_tiles + i];
  x.dweights[j] = s;
}

// Workgroups of the backward pass's second launch: for dxr, dw1, dw2 and dweights.  The launch
// begins with those from `begin` on and ends with those before.
struct Shares {
  int32_t in_x, in_w1, in_w2, begin;
  __device__ __forceinline__ int32_t mine() const {
    const int32_t all = gridDim.x, id = blockIdx.x + begin;
    return id < all ? id : id - all;
  }
};

// One tile of SIDE x SIDE by four waves, or GROUPS times four that share k, for any sizes and
// alignment: a stage's 16-byte chunks are loaded into registers two stages ahead, and from there to
// one of two places in LDS.  A chunk that a row's end cuts is loaded as the row's last 16 bytes and
// shifted on its way to LDS, so that every load is one instruction without a branch (one with a
// branch has to be awaited at once); TINY: rows may be shorter than that, and are loaded element by
// element.
// Several workgroups share a CU, so that one's loads, barriers and results hide behind another's
// products.  In binary32 bound by the matrix cores (0.153 PFLOP/s in a large library product):
// 4,096 tokens, 2 of 16 experts, 1,024 x 1,024, forward and backward 1.55 ms, 0.10 PFLOP/s with
// the rows that fill up tiles left out.  2-byte elements, tiles of 128: bound by what moves the
// operands through registers and LDS, 16,384, 2 of 32, 2,047 x 2,047: 5.3 ms, 0.47 PFLOP/s.  Small
// calls are bound by the latency of a tile (the list, the tokens, the rows: three loads that wait
// for each other) and of a launch: 777, 3 of 7, 501 x 333, binary32 150 us in 8 launches.
template <int SIDE>
constexpr int kLooseLds = 2 * 2 * SIDE * kRowBytes;
template <typename T, Kind KIND, int SIDE, bool TINY, int GROUPS = 1>
__device__ __forceinline__ void loose_tile(const Experts& x, int32_t id, char* smem) {
  constexpr int BM = SIDE, BN = SIDE, WM = 2, WN = 2;
  constexpr int kThr = WM * WN * kWave;
  constexpr int kE = 16 / sizeof(T);         // elements of a chunk
  constexpr int kBK = kRowBytes / sizeof(T);  // k staged at a time
  constexpr bool kWeightsKind = KIND == kWeightsIn || KIND == kWeightsOut;
  constexpr bool kTrA = kWeightsKind;
  constexpr bool kTrB = kWeightsKind || KIND == kBackwardGate || KIND == kBackwardIn;
  constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
  constexpr int LA = BM * 8 / kThr, LB = BN * 8 / kThr;
  constexpr int kStage = kLooseLds<SIDE> / 2;

  const int group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThr);
  const int tid = threadIdx.x - group * kThr, lane = tid % kWave, wave = tid / kWave;
  smem += group * kLooseLds<SIDE>;
  const int wm = wave / WN, wn = wave % WN;
  const int32_t D = x.dim, F = x.hidden;
  const int32_t N = KIND == kForwardGate || KIND == kBackwardGate || KIND == kWeightsOut ? F : D;
  constexpr int kCols = KIND == kForwardGate ? BN / 2 : BN;  // columns of N in a tile
  const int32_t tiles_n = (N + kCols - 1) / kCols;

  int32_t e, m0, mrows, K;
  int32_t n0;
  int64_t row0;  // first of the expert's rows in this tile (or of its k)
  if constexpr (kWeightsKind) {
    const int32_t M = KIND == kWeightsIn ? 2 * F : D;
    const int32_t tiles_m = (M + BM - 1) / BM;
    if constexpr (kRun<SIDE> > 1) {
      id = spread(id, x.experts * tiles_m * tiles_n, kRun<SIDE>);
      if (id < 0) return;
    }
    e = id / (tiles_m * tiles_n);
    const int2 at = tile_place<kTall<SIDE>>(id - e * tiles_m * tiles_n, tiles_m, tiles_n);
    m0 = at.x * BM;
    n0 = at.y * BN;
    mrows = M - m0;
    row0 = x.plan.offsets[e];
    K = x.plan.offsets[e + 1] - static_cast<int32_t>(row0);
  } else {
    m0 = 0;
    if constexpr (SIDE == kSmallRows) {
      const int32_t i = id / tiles_n;
      const int4 t = x.plan.small[i];  // (past the listed ones it is not used)
      if (i >= x.plan.tile_count[1]) return;
      e = t.x;
      row0 = t.y;
      n0 = id % tiles_n * kCols;
      mrows = t.z;
    } else {
      constexpr int kSub = kPlanRows / SIDE;
      id = spread(id, x.plan.tile_count[0] * kSub * tiles_n, kRun<SIDE>);
      if (id < 0) return;
      const int4 t = x.plan.tiles[id / (kSub * tiles_n)];
      const int2 at = tile_place<kTall<SIDE>>(id - t.z * kSub * tiles_n, t.w * kSub, tiles_n);
      e = t.x;
      row0 = t.y + at.x * SIDE;
      n0 = at.y * kCols;
      mrows = x.plan.offsets[e + 1] - static_cast<int32_t>(row0);
      if (mrows <= 0) return;
    }
    K = KIND == kForwardGate || KIND == kBackwardGate ? D : KIND == kForwardOut ? F : 2 * F;
  }

  // this group's part of k (what of it is past the end loads zeros)
  const int32_t part = GROUPS == 1 ? K : (K + GROUPS * kBK - 1) / (GROUPS * kBK) * kBK;
  const int32_t k_begin = group * part, k_end = k_begin + part;
  // With k contiguous: this lane's LA (LB) rows, null outside.
  const auto token = [&](int64_t r) { return static_cast<int64_t>(x.plan.token[r]); };
  const T* rows_a[LA];
  const T* rows_b[LB];
  if constexpr (!kTrA) {
#pragma unroll
    for (int j = 0; j < LA; ++j) {
      const int32_t m = (j * kThr + tid) >> 3;
      rows_a[j] = nullptr;
      if (m >= mrows) continue;
      if constexpr (KIND == kForwardGate)
        rows_a[j] = static_cast<const T*>(x.x) + token(row0 + m) * x.x_stride;
      else if constexpr (KIND == kForwardOut)
        rows_a[j] = static_cast<const T*>(x.act) + (row0 + m) * F;
      else if constexpr (KIND == kBackwardGate)
        rows_a[j] = static_cast<const T*>(x.dout) + token(row0 + m) * D;
      else
        rows_a[j] = static_cast<const T*>(x.dpre) + (row0 + m) * 2 * F;
    }
  }
  if constexpr (!kTrB) {
#pragma unroll
    for (int j = 0; j < LB; ++j) {
      const int32_t c = (j * kThr + tid) >> 3;
      rows_b[j] = nullptr;
      if constexpr (KIND == kForwardGate) {
        // a wave's columns: half of them gates, half the same columns' ups
        constexpr int kW = BN / WN, kHalf = kW / 2;
        const int32_t f = n0 + c / kW * kHalf + c % kHalf;
        const int q = c % kW / kHalf;
        if (f < F)
          rows_b[j] = static_cast<const T*>(x.w1) +
                      (static_cast<int64_t>(e) * 2 * F + q * F + f) * D;
      } else if (n0 + c < D) {
        rows_b[j] = static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + n0 + c) * F;
      }
    }
  }
  // With k as the row: rows of A and B (from their first column in the tile) that are not gathered,
  // and the steps from row to row.
  constexpr bool kGatherA = KIND == kWeightsOut, kGatherB = KIND == kWeightsIn;
  const T *base_a = nullptr, *base_b = nullptr;
  int64_t step_a = 0, step_b = 0;
  if constexpr (KIND == kWeightsIn) {
    base_a = static_cast<const T*>(x.dpre) + row0 * 2 * F + m0;
    step_a = 2 * static_cast<int64_t>(F);
    base_b = static_cast<const T*>(x.x) + n0;
    step_b = x.x_stride;
  } else if constexpr (KIND == kWeightsOut) {
    base_a = static_cast<const T*>(x.dout) + m0;
    step_a = D;
    base_b = static_cast<const T*>(x.wact) + row0 * F + n0;
    step_b = F;
  } else if constexpr (KIND == kBackwardGate) {
    base_b = static_cast<const T*>(x.w2) + static_cast<int64_t>(e) * D * F + n0;
    step_b = F;
  } else if constexpr (KIND == kBackwardIn) {
    base_b = static_cast<const T*>(x.w1) + static_cast<int64_t>(e) * 2 * F * D + n0;
    step_b = D;
  }
  // chunk j's place in a stage, k0 the stage's first k: k (or the column) where it begins, and the
  // length of its row from there (0 or less: nothing of it is inside)
  const T* const zeros = reinterpret_cast<const T*>(kZeros);
  const auto begin = [&](bool is_a, int j, int32_t k0) {
    const int i = j * kThr + tid;
    if (is_a ? !kTrA : !kTrB) return k0 + chunk_k(i >> 3, i & 7) * kE;
    constexpr int kCA = BM / kE, kCB = BN / kE;
    return (is_a ? chunk_n<T, kCA>(i / kCA, i % kCA) : chunk_n<T, kCB>(i / kCB, i % kCB)) * kE;
  };
  const auto length = [&](bool is_a) { return (is_a ? !kTrA : !kTrB) ? K : is_a ? mrows : N - n0; };
  // Chunks with k as the row: their first k in the stage, where k ends for them (0 for columns
  // outside), and their address, which moves on from stage to stage; gathered rows have their
  // token's, loaded a stage before it is used and ahead of that stage's chunks, as a wait for a
  // load is one for all before it.
  int32_t first[LA + LB], end[LA + LB], tokens[LA + LB];
  const T* walk[LA + LB];
  const auto load_tokens = [&](int32_t k0) {
#pragma unroll
    for (int j = 0; j < LA + LB; ++j) {
      if (!(j < LA ? kGatherA : kGatherB)) continue;
      const int32_t k = k0 + first[j];
      tokens[j] = x.plan.token[row0 + (k < K ? k : K - 1)];
    }
  };
#pragma unroll
  for (int j = 0; j < LA + LB; ++j) {
    const bool is_a = j < LA;
    if (is_a ? !kTrA : !kTrB) continue;
    const int q = is_a ? j : j - LA, i = q * kThr + tid;
    const int32_t at = begin(is_a, q, 0), len = length(is_a);
    first[j] = i / ((is_a ? BM : BN) / kE);
    end[j] = at < len ? K : 0;
    walk[j] = (is_a ? base_a : base_b) + (TINY || at + kE <= len ? at : len - kE);
    if (!(is_a ? kGatherA : kGatherB))
      walk[j] += (k_begin + first[j]) * (is_a ? step_a : step_b);
  }
  if (K > 0) load_tokens(k_begin);
  Frag ahead[2][LA + LB];
  const auto load = [&](int32_t k0, Frag (&to)[LA + LB]) {
    const T* from[LA + LB];
#pragma unroll
    for (int j = 0; j < LA + LB; ++j) {
      const bool is_a = j < LA;
      if (is_a ? kGatherA : kGatherB)
        from[j] = walk[j] + tokens[j] * (is_a ? step_a : step_b);
    }
    if constexpr (kGatherA || kGatherB) load_tokens(k0 + kBK);
#pragma unroll
    for (int j = 0; j < LA + LB; ++j) {
      const bool is_a = j < LA;
      const int q = is_a ? j : j - LA;
      const int32_t at = begin(is_a, q, k0), len = length(is_a);
      bool in;
      if (is_a ? kTrA : kTrB) {
        in = k0 + first[j] < end[j];
        if (!(is_a ? kGatherA : kGatherB)) {
          from[j] = walk[j];
          walk[j] += kBK * (is_a ? step_a : step_b);
        }
      } else {
        const T* row = nullptr;
        if constexpr (!kTrA) row = is_a ? rows_a[is_a ? q : 0] : row;
        if constexpr (!kTrB) row = is_a ? row : rows_b[is_a ? 0 : q];
        in = row && at < len;
        from[j] = row + (TINY || at + kE <= len ? at : len - kE);
      }
      if constexpr (TINY) {
        to[j].u = u32x4{0, 0, 0, 0};
        if (in) to[j] = row_chunk<false>(from[j] - at, at, len);
      } else {
        to[j] = row_chunk<true>(in ? from[j] : zeros, 0, kE);
      }
    }
  };
  // the elements from the cut on come first, zeros after them
  const auto shifted = [&](Frag f, bool is_a, int q, int32_t k0) {
    if constexpr (!TINY) {
      const int32_t over = begin(is_a, q, k0) + kE - length(is_a);
      if (over > 0) {  // (a chunk wholly outside is zeros already)
        unsigned __int128 v = __builtin_bit_cast(unsigned __int128, f.u);
        v = over < kE ? v >> (over * 8 * static_cast<int>(sizeof(T))) : 0;
        f.u = __builtin_bit_cast(u32x4, v);
      }
    }
    return f;
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const auto stage = [&](int32_t k0, Frag (&chunks)[LA + LB], char* sa) {
    char* const sb = sa + BM * kRowBytes;
#pragma unroll
    for (int j = 0; j < LA; ++j)
      *reinterpret_cast<u32x4*>(sa + (j * kThr + tid) * 16) = shifted(chunks[j], true, j, k0).u;
#pragma unroll
    for (int j = 0; j < LB; ++j)
      *reinterpret_cast<u32x4*>(sb + (j * kThr + tid) * 16) =
          shifted(chunks[LA + j], false, j, k0).u;
    __syncthreads();
    if (k0 + 2 * kBK < k_end) load(k0 + 2 * kBK, chunks);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Frag fa[MT], fb[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i)
        fa[i] = fragment<T, kTrA, BM>(sa, wm * (BM / WM) + i * 16, s, lane);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        fb[j] = fragment<T, kTrB, BN>(sb, wn * (BN / WN) + j * 16, s, lane);
#pragma unroll
      for (int q = 0; q < kParts<T>; ++q)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j], q);
    }
  };
  if (part > 0) load(k_begin, ahead[0]);
  if (part > kBK) load(k_begin + kBK, ahead[1]);
  for (int32_t k0 = k_begin; k0 < k_end; k0 += 2 * kBK) {
    stage(k0, ahead[0], smem);
    if (k0 + kBK < k_end) stage(k0 + kBK, ahead[1], smem + kStage);
  }
  __syncthreads();
  if constexpr (GROUPS > 1) {
    static_assert(kThr * MT * NT * 16 <= kLooseLds<SIDE>);
    f32x4* const sums = reinterpret_cast<f32x4*>(smem);
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < MT * NT; ++i) sums[i * kThr + tid] = acc[i / NT][i % NT];
    }
    __syncthreads();
    if (group > 0) {
      if constexpr (KIND == kBackwardGate) __syncthreads();  // (the one in finish)
      return;
    }
#pragma unroll
    for (int g = 1; g < GROUPS; ++g)
#pragma unroll
      for (int i = 0; i < MT * NT; ++i)
        acc[i / NT][i % NT] +=
            *reinterpret_cast<const f32x4*>(smem + g * kLooseLds<SIDE> + (i * kThr + tid) * 16);
  }

  finish<T, KIND, BM, BN, WM, WN>(x, acc, reinterpret_cast<float*>(smem), e, m0, mrows, n0, row0);
}

constexpr int kLooseThreads = 256;
// Waves of a SIMD that registers have to last for.  Five in place of four, steps in us: binary32,
// 4,096 tokens, 2 of 16 experts, 1,024 x 1,024: 1,556 and 1,625; bfloat16, 465, 3 of 32, 343 x
// 1,343: 195 and 179.  Middle tiles, two in place of one: 16,384, 2 of 32, 2,047 x 2,047: 5,350 and
// 8,216.
template <typename T, int SIDE>
constexpr int kLooseWaves = SIDE == kMiddleRows ? 2 : sizeof(T) == 4 ? 5 : 4;
template <typename T, Kind KIND, int SIDE, bool TINY>
__global__ __launch_bounds__(kLooseThreads, (kLooseWaves<T, SIDE>)) void ex_loose(Experts x) {
  __shared__ __attribute__((aligned(16))) char smem[kLooseLds<SIDE>];
  loose_tile<T, KIND, SIDE, TINY>(x, blockIdx.x, smem);
}
// The groups of four waves each take a part of k, and add their sums up in the groups' order.
template <typename T, Kind KIND, int GROUPS>
__global__ __launch_bounds__(GROUPS* kLooseThreads) void ex_split(Experts x) {
  __shared__ __attribute__((aligned(16))) char smem[GROUPS * kLooseLds<kSmallRows>];
  loose_tile<T, KIND, kSmallRows, false, GROUPS>(x, blockIdx.x, smem);
}
template <typename T, int SIDE, bool TINY>
__global__ __launch_bounds__(kLooseThreads, (kLooseWaves<T, SIDE>)) void ex_loose_gradients(
    Experts x, Shares n) {
  __shared__ __attribute__((aligned(16))) char smem[kLooseLds<SIDE>];
  int32_t id = n.mine();
  if (id < n.in_x) return loose_tile<T, kBackwardIn, SIDE, TINY>(x, id, smem);
  id -= n.in_x;
  if (id < n.in_w1) return loose_tile<T, kWeightsIn, SIDE, TINY>(x, id, smem);
  id -= n.in_w1;
  if (id < n.in_w2) return loose_tile<T, kWeightsOut, SIDE, TINY>(x, id, smem);
  sum_dots(x, static_cast<int64_t>(id - n.in_w2) * kLooseThreads);
}

// ------------------------------------------------------------------ aligned operands ----

// 16 bytes a lane from its address to LDS offset `at` + 16 lane, without a register between.
// The compiler does not count these loads: meet() does (with the builtin of this load the
// compiler waits for all of them before every read of LDS, as it cannot tell the buffers apart).
// m0 is a reserved register, which asm cannot declare as written; no other instruction of these
// kernels reads it (tests/test_experts_assembly.py; putting its old value back after every load
// took up to 3% of a training step's time).
__device__ __forceinline__ void load_to_lds(const void* p, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(at), "v"(p)
               : "memory");
}
__device__ __forceinline__ void load_word_to_lds(const void* p, uint32_t at) {  // 4 bytes a lane
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(at), "v"(p)
               : "memory");
}
// Waits for the workgroup's other waves; before that until this wave's reads of LDS are done, or
// its loads too.  One block of asm each, so that no access of LDS comes between.
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }
__device__ __forceinline__ void meet_read() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
template <int LEFT>  // but for so many of the last loads
__device__ __forceinline__ void meet_loaded() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// Waits until at most LEFT of this wave's loads and stores are under way; until its reads of LDS
// are done.
template <int LEFT>
__device__ __forceinline__ void await_own() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void await_reads() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// What a wave's lanes wrote to LDS before it, they may read from each other after it.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// 16 rows of COLS results of a wave, turned round in its own LDS: a lane has four columns of one
// row, and 4 lanes of 64 share it, so stores from the lanes would go out in pieces of 32 or 64
// bytes; from here they go out in whole rows of 64 to 256 bytes.
template <typename U, int COLS>
struct Turn {
  static constexpr int kRow = COLS * static_cast<int>(sizeof(U)) + 16;  // (spreads the banks)
  static constexpr int kBytes = 16 * kRow;
  static constexpr int kW = 16 / static_cast<int>(sizeof(U));
  static constexpr int kLanes = COLS / kW;  // of a row
  static constexpr int kStores = 16 * kLanes / kWave;
  char* at;
  __device__ __forceinline__ void put(int row, int col, const float* v) const {
    Vec<U, 4> o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = from_float<U>(v[i]);
    *reinterpret_cast<Vec<U, 4>*>(at + row * kRow + col * static_cast<int>(sizeof(U))) = o;
  }
  // rows `rows` of the 16, columns `cols` of a matrix with rows of ld elements
  __device__ __forceinline__ void out(U* to, int64_t ld, int32_t rows, int32_t cols,
                                      int lane) const {
#pragma unroll
    for (int i = 0; i < kStores; ++i) {
      const int row = i * (kWave / kLanes) + lane / kLanes, col = lane % kLanes * kW;
      const u32x4 v = *reinterpret_cast<const u32x4*>(at + row * kRow +
                                                      col * static_cast<int>(sizeof(U)));
      if (row < rows && col < cols) *reinterpret_cast<u32x4*>(to + row * ld + col) = v;
    }
  }
};

// Results of a tile, as finish() makes them, by way of the stages' LDS, an equal part a wave.
template <typename T, Kind KIND, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void finish_rows(const Experts& x,
                                            f32x4 (&acc)[BM / WM / 16][BN / WN / 16], char* smem,
                                            uint32_t lds, int32_t e, int32_t m0, int32_t mrows,
                                            int32_t n0, int64_t row0) {
  constexpr int kThr = WM * WN * kWave, MT = BM / WM / 16, NT = BN / WN / 16, kW = BN / WN;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wm = wave / WN, wn = wave % WN;
  const int32_t D = x.dim, F = x.hidden;
  const int32_t N = KIND == kForwardGate || KIND == kBackwardGate || KIND == kWeightsOut ? F : D;
  const int li = lane & 15, lg = (lane >> 4) * 4;
  constexpr int kRoom = 2 * (BM + BN) * kRowBytes / (WM * WN);  // of a wave
  char* const room = smem + wave * kRoom;
  const int32_t n = n0 + wn * (KIND == kForwardGate ? kW / 2 : kW);  // the wave's first column
  const int32_t cols = N - n;

  if constexpr (KIND == kForwardGate) {
    constexpr int kC = kW / 2;
    using Wide = Turn<float, kC>;
    using Narrow = Turn<T, kC>;
    static_assert(2 * Wide::kBytes + Narrow::kBytes <= kRoom);
    const Narrow act{room};
    const Wide gate{room + Narrow::kBytes}, up{room + Narrow::kBytes + Wide::kBytes};
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int32_t m = wm * (BM / WM) + i * 16;
      if (m >= mrows) break;
#pragma unroll
      for (int j = 0; j < NT / 2; ++j) {
        float g[4], u[4], v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          g[q] = acc[i][j][q];
          u[q] = acc[i][j + NT / 2][q];
          v[q] = g[q] * sigmoid(g[q]) * u[q];
        }
        act.put(li, j * 16 + lg, v);
        if (x.pre) {
          gate.put(li, j * 16 + lg, g);
          up.put(li, j * 16 + lg, u);
        }
      }
      wave_fence();
      const int64_t row = row0 + m;
      act.out(static_cast<T*>(x.act) + row * F + n, F, mrows - m, cols, lane);
      if (x.pre) {
        gate.out(x.pre + row * 2 * F + n, 2 * F, mrows - m, cols, lane);
        up.out(x.pre + row * 2 * F + F + n, 2 * F, mrows - m, cols, lane);
      }
      wave_fence();
    }
  } else if constexpr (KIND == kBackwardGate) {
    // The gates and ups of 16 rows come to LDS while the rows before are worked on.
    using Narrow = Turn<T, kW>;
    constexpr int kPre = 16 * kW * 4;  // bytes of 16 rows of gates, or of ups
    static_assert(2 * kPre + 3 * Narrow::kBytes <= kRoom && kPre % 1024 == 0);
    const char* const pre = room;
    char* const turns = room + 2 * kPre;
    const Narrow dgate{turns}, dup{turns + Narrow::kBytes}, wact{turns + 2 * Narrow::kBytes};
    const uint32_t pre_at = lds + wave * kRoom;
    constexpr int kLanes = kW / 4;  // of a row of 4-byte elements
    const auto fetch = [&](int i) {
      // (rows and columns past the ends load the last ones)
      const int32_t m = wm * (BM / WM) + i * 16;
      const int col = lane % kLanes * 4;
      const int32_t f = col < cols ? n + col : F - 4;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int v = 0; v < kPre / 1024; ++v) {
          int32_t r = m + v * (kWave / kLanes) + lane / kLanes;
          if (r >= mrows) r = mrows - 1;
          load_to_lds(x.pre + (row0 + r) * 2 * F + h * F + f, pre_at + h * kPre + v * 1024);
        }
    };
    fetch(0);
    float parts[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int32_t m = wm * (BM / WM) + i * 16;
      const float w = m + li < mrows ? x.weights[x.plan.rows[row0 + m + li]] : 0.0f;
      // (The stores since then count too.  A wave whose rows or columns have ended sends none and
      // may read what is not there yet, of which it uses nothing; but its loads may not outlast the
      // loop, after which others write the dots to their place.)
      if (i == 0 || i + 1 == MT) await_own<0>();
      else await_own<3 * Narrow::kStores>();
      const int64_t row = row0 + m;
      float part = 0.0f;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int at = (li * kW + j * 16 + lg) * 4;
        const f32x4 g = *reinterpret_cast<const f32x4*>(pre + at);
        const f32x4 u = *reinterpret_cast<const f32x4*>(pre + kPre + at);
        float dg[4], du[4], wa[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const Gated r = gated(acc[i][j][q], g[q], u[q], w);
          part += j * 16 + lg < cols ? r.dot : 0.0f;
          dg[q] = r.dg;
          du[q] = r.du;
          wa[q] = r.wa;
        }
        dgate.put(li, j * 16 + lg, dg);
        dup.put(li, j * 16 + lg, du);
        wact.put(li, j * 16 + lg, wa);
      }
      // (summed here: left to the compiler, the terms of all rows wait in memory for the end)
      asm volatile("" : "+v"(part));
      wave_fence();
      parts[i] = part;
      if (i + 1 < MT) {
        await_reads();
        fetch(i + 1);
      }
      T* const to = static_cast<T*>(x.dpre) + row * 2 * F + n;
      dgate.out(to, 2 * F, mrows - m, cols, lane);
      dup.out(to + F, 2 * F, mrows - m, cols, lane);
      wact.out(static_cast<T*>(x.wact) + row * F + n, F, mrows - m, cols, lane);
      wave_fence();
    }
    __syncthreads();
    float* const dot = reinterpret_cast<float*>(smem);  // [WN][BM]
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float part = parts[i];
      part += __shfl_xor(part, 16);
      part += __shfl_xor(part, 32);
      if (lane < 16) dot[wn * BM + wm * (BM / WM) + i * 16 + li] = part;
    }
    __syncthreads();
    for (int32_t m = tid; m < BM && m < mrows; m += kThr) {
      float s = 0.0f;
#pragma unroll
      for (int q = 0; q < WN; ++q) s += dot[q * BM + m];
      x.dots[(row0 + m) * x.dot_tiles + n0 / BN] = s;
    }
  } else {
    constexpr bool kF32 = KIND == kForwardOut || KIND == kBackwardIn;
    using U = std::conditional_t<kF32, float, T>;
    const Turn<U, kW> turn{room};
    static_assert(Turn<U, kW>::kBytes <= kRoom);
    U* const to = static_cast<U*>(KIND == kForwardOut    ? static_cast<void*>(x.y)
                                  : KIND == kBackwardIn  ? static_cast<void*>(x.dxr)
                                  : KIND == kWeightsIn   ? x.dw1
                                                         : x.dw2);
    const int64_t M = KIND == kWeightsIn ? 2 * F : D;
    const int64_t first = kF32 ? row0 : e * M + m0;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int32_t m = wm * (BM / WM) + i * 16;
      if (m >= mrows) break;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        turn.put(li, j * 16 + lg, v);
      }
      wave_fence();
      turn.out(to + (first + m) * N + n, N, mrows - m, cols, lane);
      wave_fence();
    }
  }
}

// One tile of 256 x 256 of 2-byte elements by eight waves.  Rows of every operand start at a
// multiple of 16 bytes and hold a multiple of 16 bytes.
// So large a tile moves the fewest bytes per product into LDS: 64 KB a stage of 64 k, which the
// card's L2 caches bring in 1.19 us when all CUs load (14 TB/s), while the products alone take 1.0
// us at the clock that they leave; together 1.2 to 1.3.  Besides its stages a tile takes 7 us to
// start (list, tokens, first stages) and 12 for its results, which nothing hides, as LDS holds one
// workgroup a CU; the gates' gradients, with 0.9 MB a tile to read and write, some 40.
// 16,384 tokens, 2 of 32 experts, 2,048 x 2,048, bfloat16 (a large library product reaches 1.28
// PFLOP/s): first product 564 us (0.97 PFLOP/s), second 282 (0.97), gates' gradients
// 424 (0.65), the other three together 1,500 (0.92); the matrix cores are busy 47, 46, 29 and 42%
// of the cycles.
constexpr int kLargeThreads = 512;
constexpr int kLargeLds = 5 * kTileRows * kRowBytes;
template <typename T, Kind KIND>
__device__ __forceinline__ void large_tile(const Experts& x, int32_t block, char* smem) {
  constexpr int BM = kTileRows, BN = kTileRows, WM = 2, WN = 4;
  constexpr int kThr = WM * WN * kWave, kWaves = WM * WN;
  constexpr int kE = 16 / sizeof(T);          // elements of a chunk
  constexpr int kBK = kRowBytes / sizeof(T);  // k staged at a time
  constexpr bool kWeightsKind = KIND == kWeightsIn || KIND == kWeightsOut;
  constexpr bool kTrA = kWeightsKind;
  constexpr bool kTrB = kWeightsKind || KIND == kBackwardGate || KIND == kBackwardIn;
  constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
  constexpr int LA = BM * 8 / kThr, LB = BN * 8 / kThr;  // chunks a lane loads of each operand
  // SA and SB places for a stage of A and of B; of gathered k, the tokens of four stages
  constexpr int SA = kWeightsKind ? 2 : 3, SB = 2;
  constexpr int kSlotA = BM * kRowBytes, kSlotB = BN * kRowBytes;
  static_assert(kThr == kLargeThreads &&
                SA * kSlotA + SB * kSlotB + (kWeightsKind ? 4 * kWave * 4 : 0) <= kLargeLds);

  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wm = wave / WN, wn = wave % WN;
  const int32_t D = x.dim, F = x.hidden;
  const int32_t N = KIND == kForwardGate || KIND == kBackwardGate || KIND == kWeightsOut ? F : D;
  constexpr int kCols = KIND == kForwardGate ? BN / 2 : BN;  // columns of N in a tile
  const int32_t tiles_n = (N + kCols - 1) / kCols;

  int32_t e, m0, mrows, K, n0;
  int64_t row0;  // first of the expert's rows in this tile (or of its k)
  if constexpr (kWeightsKind) {
    const int32_t M = KIND == kWeightsIn ? 2 * F : D;
    const int32_t tiles_m = (M + BM - 1) / BM;
    const int32_t id = spread(block, x.experts * tiles_m * tiles_n, kRun<kTileRows>);
    if (id < 0) return;
    e = id / (tiles_m * tiles_n);
    const int2 at = tile_place<kTall<kTileRows>>(id - e * tiles_m * tiles_n, tiles_m, tiles_n);
    m0 = at.x * BM;
    n0 = at.y * BN;
    mrows = M - m0;
    row0 = x.plan.offsets[e];
    K = x.plan.offsets[e + 1] - static_cast<int32_t>(row0);
  } else {
    const int32_t id = spread(block, x.plan.tile_count[0] * tiles_n, kRun<kTileRows>);
    if (id < 0) return;
    const int4 t = x.plan.tiles[id / tiles_n];
    const int2 at = tile_place<kTall<kTileRows>>(id - t.z * tiles_n, t.w, tiles_n);
    e = t.x;
    m0 = 0;
    row0 = t.y + at.x * BM;
    n0 = at.y * kCols;
    mrows = x.plan.offsets[e + 1] - static_cast<int32_t>(row0);
    K = KIND == kForwardGate || KIND == kBackwardGate ? D : KIND == kForwardOut ? F : 2 * F;
  }

  // What this lane loads of an operand: chunk i = j kThr + tid of a stage for j = 0, 1, ..  With k
  // contiguous that is chunk c of row r + j kStepK, c the same for all j; with k as the row, chunk
  // c of row r + j kStep of the stage.  An address is the lane's own, which moves on from stage to
  // stage, and the same step for all lanes from one j to the next; gathered rows have their
  // token's row instead.  What lies outside loads zeros, all of them from one place, so that blocks
  // that an expert's rows do not fill ask less of the L2 (with the idle half below: first product
  // of 8,191 tokens, 4 of 64 experts, 2,048 x 1,024 355 -> 337 us).
  const char* const zeros = reinterpret_cast<const char*>(kZeros);
  constexpr int kStepK = kThr / 8, kCA = BM / kE, kCB = BN / kE;
  constexpr int kStepA = kTrA ? kThr / kCA : kStepK, kStepB = kTrB ? kThr / kCB : kStepK;
  constexpr int kSize = static_cast<int>(sizeof(T));
  constexpr bool kGatherA = KIND == kForwardGate || KIND == kBackwardGate || KIND == kWeightsOut;
  constexpr bool kGatherB = KIND == kWeightsIn;
  const int ra = kTrA ? tid / kCA : tid >> 3, rb = kTrB ? tid / kCB : tid >> 3;
  // (kStep is a multiple of 16, which leaves the chunk's place alone)
  static_assert(sizeof(T) == 2 && kStepA % 16 == 0 && kStepB % 16 == 0);
  const int ca = kTrA ? chunk_n<T>(ra, tid % kCA) : chunk_k(ra, tid & 7);
  const int cb = kTrB ? chunk_n<T>(rb, tid % kCB) : chunk_k(rb, tid & 7);
  const int32_t ka = kTrA ? ra : ca * kE, kb = kTrB ? rb : cb * kE;  // k of j = 0 in stage 0
  int64_t lda, ldb;  // bytes from row to row
  const T *a0, *b0;
  if constexpr (KIND == kForwardGate) {
    a0 = static_cast<const T*>(x.x);
    lda = x.x_stride * kSize;
    // a wave's columns: half of them gates, half the same columns' ups
    constexpr int kW = BN / WN, kHalf = kW / 2;
    static_assert(kW == kStepK);
    b0 = static_cast<const T*>(x.w1) +
         (static_cast<int64_t>(e) * 2 * F + rb / kHalf * F + n0 + rb % kHalf) * D;
    ldb = int64_t{kSize} * D;
  } else if constexpr (KIND == kForwardOut) {
    a0 = static_cast<const T*>(x.act) + (row0 + ra) * F;
    lda = int64_t{kSize} * F;
    b0 = static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + n0 + rb) * F;
    ldb = lda;
  } else if constexpr (KIND == kBackwardGate) {
    a0 = static_cast<const T*>(x.dout);
    lda = int64_t{kSize} * D;
    b0 = static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + rb) * F + n0;
    ldb = int64_t{kSize} * F;
  } else if constexpr (KIND == kBackwardIn) {
    a0 = static_cast<const T*>(x.dpre) + (row0 + ra) * 2 * F;
    lda = int64_t{kSize} * 2 * F;
    b0 = static_cast<const T*>(x.w1) + (static_cast<int64_t>(e) * 2 * F + rb) * D + n0;
    ldb = int64_t{kSize} * D;
  } else if constexpr (KIND == kWeightsIn) {
    a0 = static_cast<const T*>(x.dpre) + (row0 + ra) * 2 * F + m0;
    lda = int64_t{kSize} * 2 * F;
    b0 = static_cast<const T*>(x.x) + n0;
    ldb = x.x_stride * kSize;
  } else {
    a0 = static_cast<const T*>(x.dout) + m0;
    lda = int64_t{kSize} * D;
    b0 = static_cast<const T*>(x.wact) + (row0 + rb) * F + n0;
    ldb = int64_t{kSize} * F;
  }
  const char* pa = reinterpret_cast<const char*>(a0 + ca * kE);
  const char* pb = reinterpret_cast<const char*>(b0 + cb * kE);
  const int64_t step_a = !kTrA ? kRowBytes : kGatherA ? 0 : kBK * lda;
  const int64_t step_b = !kTrB ? kRowBytes : kGatherB ? 0 : kBK * ldb;
  // rows of B with k contiguous: of w1 the next kHalf gates and ups, of w2 the next kStepK columns
  constexpr int kNextB = KIND == kForwardGate ? kStepK / 2 : kStepB;
  const int32_t nb = n0 + (KIND == kForwardGate ? rb % kNextB : rb);
  const uint32_t lds = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem));
  const uint32_t at_a = lds + wave * (kWave * 16), at_b = at_a + SA * kSlotA;

  // Rows gathered as k: their tokens come to LDS too, a stage before the loads that need them, by
  // every wave alike (the same values to the same place; of 64 a stage uses the first kBK).
  const int32_t* const tokens = reinterpret_cast<const int32_t*>(smem + SA * kSlotA + SB * kSlotB);
  const auto load_tokens = [&](int32_t h) {
    const int32_t k = h * kBK + lane;
    load_word_to_lds(x.plan.token + row0 + (k < K ? k : K - 1),
                     lds + SA * kSlotA + SB * kSlotB + (h & 3) * (kWave * 4));
  };
  int32_t token[kGatherB ? LB : LA];  // of the gathered operand
  const auto read_tokens = [&](int32_t h) {
#pragma unroll
    for (int j = 0; j < (kGatherB ? LB : LA); ++j)
      token[j] = tokens[(h & 3) * kWave + (kGatherB ? rb + j * kStepB : ra + j * kStepA)];
  };
  if constexpr (kGatherA && !kTrA) {
#pragma unroll
    for (int j = 0; j < LA; ++j) {
      const int32_t r = ra + j * kStepA;
      token[j] = x.plan.token[row0 + (r < mrows ? r : mrows - 1)];
    }
  }
  // Loads of stage h to their slots; then the addresses are those of the next stage.
  const auto load_a = [&](int32_t h, int slot) {
#pragma unroll
    for (int j = 0; j < LA; ++j) {
      const char* p = pa;
      if constexpr (kGatherA) p += token[j] * lda;
      else p += j * (kStepA * lda);
      bool in = h * kBK + ka + (kTrA ? j * kStepA : 0) < K;
      in = in && (kTrA ? ca * kE : ra + j * kStepA) < mrows;
      load_to_lds(in ? p : zeros, at_a + slot * kSlotA + j * (kThr * 16));
    }
    pa += step_a;
  };
  const auto load_b = [&](int32_t h, int slot) {
#pragma unroll
    for (int j = 0; j < LB; ++j) {
      const char* p = pb;
      if constexpr (kGatherB) p += token[j] * ldb;
      else p += j * (kNextB * ldb);
      bool in = h * kBK + kb + (kTrB ? j * kStepB : 0) < K;
      in = in && (kTrB ? n0 + cb * kE : nb + j * kNextB) < N;
      load_to_lds(in ? p : zeros, at_b + slot * kSlotB + j * (kThr * 16));
    }
    pb += step_b;
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // Each SIMD has a wave of the workgroup's first half and one of its second.  The halves work in
  // opposite phases, with a barrier at the end of each: while one multiplies, the other reads the
  // fragments of its next products from LDS and sends loads out, so neither waits in the other's
  // way.  A stage is four phases of a wave: read half of k, multiply, read the other half,
  // multiply.  With three places for A its loads go out in the third phase, two stages ahead, and
  // those of B in the first, one ahead; with two, all in the first.  They are awaited at the end
  // of the third phase, which is before either half reads what they bring; a place is loaded again
  // when the later half has read its last fragment of it, a phase before.  The scheduling barriers
  // hold the compiler to the phases.
  const bool late = wave >= kWaves / 2;
  // a half without any of the expert's rows only loads and waits with the other
  const bool idle = !kWeightsKind && wm * (BM / WM) >= mrows;
  Frag fa[MT], fb[NT];
  const auto read = [&](int s, int slot_a, int slot_b) {
    if (idle) return;
    const char* const sa = smem + slot_a * kSlotA;
    const char* const sb = smem + SA * kSlotA + slot_b * kSlotB;
#pragma unroll
    for (int j = 0; j < NT; ++j)
      fb[j] = fragment<T, kTrB, BN>(sb, wn * (BN / WN) + j * 16, s, lane);
#pragma unroll
    for (int i = 0; i < MT; ++i)
      fa[i] = fragment<T, kTrA, BM>(sa, wm * (BM / WM) + i * 16, s, lane);
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto multiply_all = [&] {
    if (idle) return;
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j], 0);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  };
  int sa = 0, sb = 0;  // this stage's places
  const auto after_a = [&](int n) { return sa + n >= SA ? sa + n - SA : sa + n; };
  // next_a: A of stage h + SA - 1 is loaded; next_b: B of stage h + 1
  const auto stage = [&](auto next_a, auto next_b, int32_t h) {
    constexpr bool kNextA = decltype(next_a)::value, kMore = decltype(next_b)::value;
    read(0, sa, sb);
    if constexpr (kMore) {
      if constexpr (SA == 2) load_a(h + 1, sa ^ 1);
      load_b(h + 1, sb ^ 1);
      if constexpr (kWeightsKind) load_tokens(h + 3);
    }
    meet_read();
    multiply_all();
    meet();
    read(1, sa, sb);
    if constexpr (SA == 3 && kNextA) load_a(h + 2, after_a(2));
    if constexpr (kMore && kWeightsKind) read_tokens(h + 2);
    if constexpr (SA == 3 && kNextA) meet_loaded<LA>();
    else if constexpr (kMore) meet_loaded<0>();
    else meet_read();
    multiply_all();
    meet();
    sa = after_a(1);
    sb ^= 1;
  };

  if (K > 0) {
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    const int32_t stages = (K + kBK - 1) / kBK;
    if constexpr (kWeightsKind) {
      load_tokens(0);
      load_tokens(1);
      load_tokens(2);
      meet_loaded<0>();
      read_tokens(0);
    }
    load_a(0, 0);
    load_b(0, 0);
    if constexpr (kWeightsKind) read_tokens(1);
    if (SA == 3 && stages > 1) {
      load_a(1, 1);
      meet_loaded<LA>();
    } else {  // (of one stage no later meet waits for loads, and the results take their places)
      meet_loaded<0>();
    }
    if (late) meet();
    int32_t h = 0;
    for (; h + SA - 1 < stages; ++h) stage(yes, yes, h);
    if (SA == 3 && h + 1 < stages) {
      stage(no, yes, h);
      ++h;
    }
    stage(no, no, h);
    if (!late) meet();
  }
  __syncthreads();
  finish_rows<T, KIND, BM, BN, WM, WN>(x, acc, smem, lds, e, m0, mrows, n0, row0);
}

template <typename T, Kind KIND>
__global__ __launch_bounds__(kLargeThreads) void ex_large(Experts x) {
  __shared__ __attribute__((aligned(1024))) char smem[kLargeLds];
  large_tile<T, KIND>(x, blockIdx.x, smem);
}
template <typename T>
__global__ __launch_bounds__(kLargeThreads) void ex_large_gradients(Experts x, Shares n) {
  __shared__ __attribute__((aligned(1024))) char smem[kLargeLds];
  int32_t block = n.mine();
  if (block < n.in_x) return large_tile<T, kBackwardIn>(x, block, smem);
  block -= n.in_x;
  if (block < n.in_w1) return large_tile<T, kWeightsIn>(x, block, smem);
  block -= n.in_w1;
  if (block < n.in_w2) return large_tile<T, kWeightsOut>(x, block, smem);
  sum_dots(x, static_cast<int64_t>(block - n.in_w2) * kLargeThreads);
}

// ------------------------------------------------------------------------- few pairs ----

// With a few pairs an expert the products read every weight once and are bound by that: no
// staging, a wave loads 16 rows of weights straight into fragments and multiplies them with 16
// rows of tokens.  A workgroup takes one expert and 16 GT columns; its four waves each take a
// quarter of k, joined through LDS.  An expert's pairs are listed from all ids by every workgroup
// (rows of act and y are the pairs' numbers: no plan), 16 at a time.  32 tokens, 8 of 64 experts,
// 2,048 x 1,024, bfloat16: 0.6 GB in 158 us (3.9 TB/s; a large copy 4.75).
template <typename T, bool GATE, int GT>
__global__ __launch_bounds__(256) void ex_few(Experts x) {
  constexpr int kE = 16 / sizeof(T), kStep = 8 * kE;  // 128 bytes of k a step
  constexpr int NT = GATE ? 2 * GT : GT;
  constexpr int kCols = 16 * GT, kRows = 16;
  __shared__ int32_t list[kFewPairs<T>];
  __shared__ int32_t found[5];
  __shared__ float part[4][NT][64][4];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = lane >> 4, i = lane & 15;
  const int32_t D = x.dim, F = x.hidden, pairs = static_cast<int32_t>(x.pairs);
  const int32_t N = GATE ? F : D, K = GATE ? D : F;
  const int32_t n0 = blockIdx.x * kCols;

  // the expert: of a pair (unless an earlier one has it), where there are fewer pairs than experts
  int32_t e = blockIdx.y;
  const bool by_pair = pairs <= x.experts;
  if (by_pair) {
    e = x.ids[blockIdx.y];
    if (e < 0 || e >= x.experts) return;
  }
  int32_t count = 0;
  bool again = false;
  for (int32_t j0 = 0; j0 < pairs; j0 += 256) {
    const int32_t j = j0 + tid;
    const bool hit = j < pairs && x.ids[j] == e;
    again |= by_pair && hit && j < static_cast<int32_t>(blockIdx.y);
    const uint64_t m = __ballot(hit);
    if (lane == 0) found[wave] = __popcll(m);
    __syncthreads();
    int32_t at = count;
    for (int w = 0; w < wave; ++w) at += found[w];
    if (hit) list[at + __popcll(m & ((uint64_t{1} << lane) - 1))] = j;
    count += found[0] + found[1] + found[2] + found[3];
    __syncthreads();
  }
  if (__syncthreads_or(again) || count == 0) return;

  const T* w[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    int32_t n = n0 + t % GT * 16 + i;
    if (n >= N) n = N - 1;
    w[t] = GATE ? static_cast<const T*>(x.w1) +
                      (static_cast<int64_t>(e) * 2 * F + (t >= GT ? F : 0) + n) * D
                : static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + n) * F;
  }
  const int32_t steps = (K + kStep - 1) / kStep, per = (steps + 3) / 4;
  const int32_t k_begin = wave * per * kStep;
  const int32_t k_end = (wave + 1) * per * kStep < K ? (wave + 1) * per * kStep : K;

  for (int32_t r0 = 0; r0 < count; r0 += kRows) {
    const bool live = r0 + i < count;
    const int32_t mine = list[live ? r0 + i : 0];
    const T* const a = GATE ? static_cast<const T*>(x.x) +
                                  static_cast<int64_t>(mine / x.top) * x.x_stride
                            : static_cast<const T*>(x.act) + static_cast<int64_t>(mine) * F;
    f32x4 acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const auto step = [&](auto inside, int32_t k0) {
      constexpr bool kIn = decltype(inside)::value;
      Frag fw[2][NT], fa[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int32_t k = k0 + (4 * h + g) * kE;
#pragma unroll
        for (int n = 0; n < NT; ++n) fw[h][n] = row_chunk<kIn>(w[n], k, K);
        fa[h].u = u32x4{0, 0, 0, 0};
        if (live) fa[h] = row_chunk<kIn>(a, k, K);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int q = 0; q < kParts<T>; ++q) acc[n] = multiply<T>(fw[h][n], fa[h], acc[n], q);
    };
    int32_t k0 = k_begin;
    for (; k0 + kStep <= k_end; k0 += kStep) step(std::true_type(), k0);
    if (k0 < k_end) step(std::false_type(), k0);
#pragma unroll
    for (int n = 0; n < NT; ++n) *reinterpret_cast<f32x4*>(part[wave][n][lane]) = acc[n];
    __syncthreads();
    const int32_t rows = count - r0 < kRows ? count - r0 : kRows;
    for (int o = tid; o < rows * kCols; o += 256) {
      const int m = o / kCols, c = o % kCols, n = n0 + c;
      if (n >= N) continue;
      const int32_t j = list[r0 + m];
      const int at = ((c & 15) >> 2) * 16 + m;
      const auto sum = [&](int t) {
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v) s += part[v][t][at][c & 3];
        return s;
      };
      if constexpr (GATE) {
        const float gate = sum(c >> 4), up = sum(GT + (c >> 4));
        static_cast<T*>(x.act)[static_cast<int64_t>(j) * F + n] =
            from_float<T>(gate * sigmoid(gate) * up);
      } else {
        x.y[static_cast<int64_t>(j) * D + n] = sum(c >> 4);
      }
    }
    __syncthreads();
  }
}

// The second product and the sum over a token's experts in one launch, for one or two tokens (with
// 2 tokens 41 us a call, 47 us as two launches; with 4 as long, with 16 164 us and 135 us): a
// workgroup takes 16 columns of one token, two waves an expert (half of k each).
template <typename T>
__global__ __launch_bounds__(1024) void ex_few_join(Experts x) {
  constexpr int kE = 16 / sizeof(T), kStep = 8 * kE;
  __shared__ float part[2][64][16];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int waves = blockDim.x / kWave;
  const int g = lane >> 4, i = lane & 15;
  const int32_t D = x.dim, F = x.hidden;
  const int32_t n0 = blockIdx.x * 16, half = wave & 1;
  const int64_t t = blockIdx.y;
  const int32_t n = n0 + i < D ? n0 + i : D - 1;
  const int32_t steps = (F + kStep - 1) / kStep, per = (steps + 1) / 2;
  const int32_t k_begin = half * per * kStep;
  const int32_t k_end = (half + 1) * per * kStep < F ? (half + 1) * per * kStep : F;
  for (int q = wave >> 1; q < x.top; q += waves >> 1) {
    const int64_t j = t * x.top + q;
    const int32_t e = x.ids[j];
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (e >= 0 && e < x.experts) {
      const T* w = static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + n) * F;
      const T* a = static_cast<const T*>(x.act) + j * F;
      const auto step = [&](auto inside, int32_t k0) {
        constexpr bool kIn = decltype(inside)::value;
        Frag fw[2], fa[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int32_t k = k0 + (4 * h + g) * kE;
          fw[h] = row_chunk<kIn>(w, k, F);
          fa[h].u = u32x4{0, 0, 0, 0};
          if (i == 0) fa[h] = row_chunk<kIn>(a, k, F);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int p = 0; p < kParts<T>; ++p) acc = multiply<T>(fw[h], fa[h], acc, p);
      };
      int32_t k0 = k_begin;
      for (; k0 + kStep <= k_end; k0 += kStep) step(std::true_type(), k0);
      if (k0 < k_end) step(std::false_type(), k0);
    }
    if (i == 0) *reinterpret_cast<f32x4*>(&part[half][q][g * 4]) = acc;
  }
  __syncthreads();
  if (threadIdx.x < 16 && n0 + static_cast<int>(threadIdx.x) < D) {
    float s = 0.0f;
    for (int q = 0; q < x.top; ++q) {
      const int64_t j = t * x.top + q;
      const int32_t e = x.ids[j];
      if (e >= 0 && e < x.experts)
        s += x.weights[j] * (part[0][q][threadIdx.x] + part[1][q][threadIdx.x]);
    }
    static_cast<T*>(x.out)[t * D + n0 + threadIdx.x] = from_float<T>(s);
  }
}

// The sum over a token's pairs where rows of y are the pairs' numbers.
template <typename T>
__global__ __launch_bounds__(256) void ex_pairs_join(Experts x) {
  const int64_t t = blockIdx.y;
  const int32_t d = blockIdx.x * 256 + threadIdx.x;
  if (d >= x.dim) return;
  float s = 0.0f;
  for (int k = 0; k < x.top; ++k) {
    const int64_t j = t * x.top + k;
    const int32_t e = x.ids[j];
    if (e >= 0 && e < x.experts) s += x.weights[j] * x.y[j * x.dim + d];
  }
  static_cast<T*>(x.out)[t * x.dim + d] = from_float<T>(s);
}

// out[t] = sum_k weight[t, k] y[row of (t, k)], k ascending, in binary32, rounded once.  Bound by
// memory: 32,768 rows of 2,048, 0.34 GB, 71 us (4.7 TB/s).  (Rows of y in 16 bits would be half of
// that, and a second rounding of every result.)
template <typename T, bool WEIGHTED>
__global__ __launch_bounds__(256) void ex_join(Experts x, const float* __restrict__ y,
                                               T* __restrict__ out) {
  constexpr int kW = 4;
  typedef T Some __attribute__((ext_vector_type(kW), aligned(sizeof(T))));
  typedef float Four __attribute__((ext_vector_type(kW), aligned(4)));
  const int32_t each = (x.dim + kW - 1) / kW;  // lanes of a token
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < x.tokens * each;
       at += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t t = at / each;
    const int32_t d = static_cast<int32_t>(at - t * each) * kW;
    const bool whole = d + kW <= x.dim;
    float s[kW] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int k = 0; k < x.top; ++k) {
      const int64_t j = t * x.top + k;
      const int32_t r = x.plan.pos[j];
      const float w = r < 0 ? 0.0f : WEIGHTED ? x.weights[j] : 1.0f;
      const float* row = y + static_cast<int64_t>(r < 0 ? 0 : r) * x.dim + d;
      if (whole) {
        const Four v = *reinterpret_cast<const Four*>(row);
#pragma unroll
        for (int i = 0; i < kW; ++i) s[i] += r < 0 ? 0.0f : w * v[i];
      } else {
        for (int i = 0; i < kW; ++i) s[i] += r < 0 || d + i >= x.dim ? 0.0f : w * row[i];
      }
    }
    T* to = out + t * x.dim + d;
    if (whole) {
      Some v;
#pragma unroll
      for (int i = 0; i < kW; ++i) v[i] = from_float<T>(s[i]);
      *reinterpret_cast<Some*>(to) = v;
    } else {
      for (int i = 0; i < kW; ++i)
        if (d + i < x.dim) to[i] = from_float<T>(s[i]);
    }
  }
}

inline uint32_t blocks_of(int64_t n, int64_t per) {
  return static_cast<uint32_t>((n + per - 1) / per);
}

inline uint32_t join_blocks(const Experts& x) {
  const int64_t n = (x.tokens * ((x.dim + 3) / 4) + 255) / 256;
  return static_cast<uint32_t>(n < (1 << 20) ? n : 1 << 20);
}

template <typename T>
bool tiny(const Experts& x) {
  constexpr int kE = 16 / sizeof(T);
  return x.dim < kE || x.hidden < kE;
}

template <typename T, Kind KIND>
void product(Experts x, hipStream_t st) {
  x.dot_tiles = static_cast<int32_t>(blocks_of(x.hidden, x.side));
  const uint32_t grid = static_cast<uint32_t>(product_blocks(KIND, x));
  if (grid == 0) return;
  if constexpr (sizeof(T) == 2) {
    if (x.side == kTileRows) {
      ex_large<T, KIND><<<grid, kLargeThreads, 0, st>>>(x);
      return;
    }
    if (x.side == kMiddleRows) {
      ex_loose<T, KIND, kMiddleRows, false><<<grid, kLooseThreads, 0, st>>>(x);
      return;
    }
  }
  if (tiny<T>(x)) {
    ex_loose<T, KIND, kSmallRows, true><<<grid, kLooseThreads, 0, st>>>(x);
    return;
  }
  // Few tiles of many stages leave a CU's SIMDs one wave each, which waits for its own loads: as
  // many groups as fill the CU take parts of k.  Forward and backward pass with one, two and four
  // groups, us: 78 tokens, 1 of 16 experts, 3,636 x 320, bfloat16: 160, 146, 135; 64, 2 of 8, 2,048
  // x 512: 91, 79, 73; forward of 100, 4 of 8, 2,048 x 1,024 (some 320 tiles): 44, 41, 48.
  const int64_t depth = KIND == kForwardOut ? x.hidden : x.dim;
  const int64_t blocks = x.pairs / kSmallRows + (x.pairs < x.experts ? x.pairs : x.experts) / 2;
  const int64_t tiles = blocks * (grid / static_cast<uint32_t>(x.plan.most_small));
  const bool deep = depth * static_cast<int64_t>(sizeof(T)) >= 16 * kRowBytes;
  if (deep && tiles <= 192)
    ex_split<T, KIND, 4><<<grid, 4 * kLooseThreads, 0, st>>>(x);
  else if (deep && tiles <= 448)
    ex_split<T, KIND, 2><<<grid, 2 * kLooseThreads, 0, st>>>(x);
  else
    ex_loose<T, KIND, kSmallRows, false><<<grid, kLooseThreads, 0, st>>>(x);
}

// What the backward pass makes of dpre, wact and the dots, in one launch, so that one product's
// last tiles do not leave the chip idle.  All of the backward and forward pass, with a launch for
// each of the four and with one, us: 2,000 tokens, 2 of 8 experts, 1,024 x 1,024, bfloat16: 245 and
// 209; 465, 3 of 32, 343 x 1,343: 232 and 196; 16,384, 2 of 32, 2,048 x 2,048: 3,026 and 2,994.
template <typename T>
void gradients(Experts x, hipStream_t st) {
  x.dot_tiles = static_cast<int32_t>(blocks_of(x.hidden, x.side));
  const auto in = [&](const void* wanted, Kind kind) {
    return static_cast<int32_t>(wanted ? product_blocks(kind, x) : 0);
  };
  Shares n{in(x.dx, kBackwardIn), in(x.dw1, kWeightsIn), in(x.dw2, kWeightsOut), 0};
  if (x.pairs > int64_t{2} * x.hidden * x.experts) n.begin = n.in_x;
  const uint32_t threads = x.side == kTileRows ? kLargeThreads : kLooseThreads;
  const uint32_t grid = n.in_x + n.in_w1 + n.in_w2 + (x.dweights ? blocks_of(x.pairs, threads) : 0);
  if (grid == 0) return;
  if (n.begin == static_cast<int32_t>(grid)) n.begin = 0;
  if constexpr (sizeof(T) == 2) {
    if (x.side == kTileRows) {
      ex_large_gradients<T><<<grid, threads, 0, st>>>(x, n);
      return;
    }
    if (x.side == kMiddleRows) {
      ex_loose_gradients<T, kMiddleRows, false><<<grid, threads, 0, st>>>(x, n);
      return;
    }
  }
  if (tiny<T>(x))
    ex_loose_gradients<T, kSmallRows, true><<<grid, threads, 0, st>>>(x, n);
  else
    ex_loose_gradients<T, kSmallRows, false><<<grid, threads, 0, st>>>(x, n);
}

}  // namespace

template <typename T, int GT>
void few(const Experts& x, hipStream_t st) {
  const uint32_t y = static_cast<uint32_t>(x.pairs < x.experts ? x.pairs : x.experts);
  ex_few<T, true, GT><<<dim3(blocks_of(x.hidden, 16 * GT), y), 256, 0, st>>>(x);
  if (x.tokens <= kFewTokens) {
    const uint32_t waves = 2 * static_cast<uint32_t>(x.top < 8 ? x.top : 8);
    ex_few_join<T><<<dim3(blocks_of(x.dim, 16), static_cast<uint32_t>(x.tokens)),
                     waves * kWave, 0, st>>>(x);
    return;
  }
  ex_few<T, false, GT><<<dim3(blocks_of(x.dim, 16 * GT), y), 256, 0, st>>>(x);
  ex_pairs_join<T><<<dim3(blocks_of(x.dim, 256), static_cast<uint32_t>(x.tokens)), 256, 0, st>>>(
      x);
}

template <typename T>
hipError_t launch_experts(const Experts& x, hipStream_t st) {
  // Few pairs, in all and an expert, and no backward pass that needs the rows in the experts'
  // order.  This and the tiles below, us, experts of 2,048 x 1,024, bfloat16: 8 of 64, 1 token 26
  // and 43, 8 tokens 100 and 123, 32 tokens 158 and 168, 64 tokens 196 and 178; 2 of 16, 32 tokens
  // 47 and 46, 64 tokens 60 and 50.  1,024 x 1,024, binary32: 4 of 128, 128 tokens 290 and 392, 192
  // tokens 347 and 425, 384 tokens 470 and 466; 2 of 16, 64 tokens 65 and 81, 128 tokens 86 and 83.
  constexpr int64_t kEach = sizeof(T) == 4 ? 16 : 4;
  if (!x.pre && x.pairs <= kFewPairs<T> && x.pairs <= kEach * x.experts) {
    if (x.pairs <= x.experts) few<T, 1>(x, st);
    else few<T, 2>(x, st);
    return hipGetLastError();
  }
  const hipError_t e = launch_plan(x, st);
  if (e != hipSuccess) return e;
  product<T, kForwardGate>(x, st);
  product<T, kForwardOut>(x, st);
  ex_join<T, true><<<join_blocks(x), 256, 0, st>>>(x, x.y, static_cast<T*>(x.out));
  return hipGetLastError();
}

template <typename T>
hipError_t launch_experts_backward(const Experts& x, hipStream_t st) {
  product<T, kBackwardGate>(x, st);  // (none without pairs)
  gradients<T>(x, st);
  if (x.dx && x.tokens > 0)
    ex_join<T, false><<<join_blocks(x), 256, 0, st>>>(x, x.dxr, static_cast<T*>(x.dx));
  return hipGetLastError();
}

}  // namespace gsn
