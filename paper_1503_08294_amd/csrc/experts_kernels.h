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
#pragma once

#include "experts.h"

#pragma clang fp contract(fast)

namespace gsn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#ifndef EX_BM
#define EX_BM 256
#define EX_BN 256
#define EX_WM 2
#define EX_WN 4
#endif
constexpr int kRowBytes = 128;  // bytes of k (contiguous operands) staged at a time

// 16 bytes of an operand in a lane: 8 or 4 values of k of row (lane & 15)
union Frag {
  u32x4 u;
  bf16x8 b;
  f16x8 h;
  f32x4 f;
  s16x4 s[2];
};

// acc[i] += sum over the fragment's k of n-row (lane >> 4) * 4 + i and m-row lane & 15
template <typename T>
__device__ __forceinline__ f32x4 multiply(const Frag& n, const Frag& m, f32x4 acc) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(n.f[i], m.f[i], acc, 0, 0, 0);
    return acc;
  } else if constexpr (__is_same(T, bf16_t)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(n.b, m.b, acc, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(n.h, m.h, acc, 0, 0, 0);
  }
}

// Place of 16-byte chunk c in row r of a staged operand with k contiguous (8 chunks a row): the
// 16 rows that a quarter wave reads at one k fall on different banks.
__device__ __forceinline__ int chunk_k(int r, int c) { return c ^ ((r >> 1) & 7); }
// The same with k as the row, `chunks` a row: the 4 (2-byte types) or 1 rows that 16 lanes read
// 32 or 64 bytes of, and those of the wave's other quarters, fall on different banks.
template <typename T>
__device__ __forceinline__ int chunk_n(int k, int c) {
  if constexpr (sizeof(T) == 2) return c ^ (((k & 3) | ((k >> 1) & 4)) << 1);
  else return c ^ (((k >> 2) & 3) << 2);
}

// Fragment of 16 rows at `r0` and the s-th half of the staged k
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
      const char* p = tile + (k * R + (chunk_n<T>(k, col >> 3) << 3) + (col & 7)) * 2;
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

enum Kind {
  kForwardGate,   // act (and pre) from x, w1
  kForwardOut,    // y from act, w2
  kBackwardGate,  // dpre, wact, dots from dout, w2
  kBackwardIn,    // dxr from dpre, w1
  kWeightsIn,     // dw1 from dpre, x
  kWeightsOut     // dw2 from dout, wact
};

// Four results of a row at column n, N columns in all
template <bool VEC, typename T>
__device__ __forceinline__ void store4(T* row, int32_t n, int32_t N, const float* v) {
  if constexpr (VEC) {
    Vec<T, 4> o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = from_float<T>(v[i]);
    if (n < N) *reinterpret_cast<Vec<T, 4>*>(row + n) = o;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < N) row[n + i] = from_float<T>(v[i]);
}
template <bool VEC, typename T>
__device__ __forceinline__ void load4(const T* row, int32_t n, int32_t N, float* v) {
  if constexpr (VEC) {
    Vec<T, 4> o{};
    if (n < N) o = *reinterpret_cast<const Vec<T, 4>*>(row + n);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_float(o.v[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = n + i < N ? to_float(row[n + i]) : 0.0f;
}

// Results of a tile: rows m0 + 0 .. mrows - 1 of the weights' products, or rows row0 + 0 .. of
// the others; columns from n0.  VEC: four results are one access.  Uses WN * BM floats of LDS.
template <typename T, Kind KIND, int BM, int BN, int WM, int WN, bool VEC>
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
          store4<VEC>(static_cast<T*>(x.act) + (row0 + m) * F, f, F, v);
          if (x.pre) {
            store4<VEC>(x.pre + (row0 + m) * 2 * F, f, F, g);
            store4<VEC>(x.pre + (row0 + m) * 2 * F + F, f, F, u);
          }
        }
      } else if constexpr (KIND == kBackwardGate) {
        const float w = x.weights[x.plan.rows[row0 + m]];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int32_t f = n0 + wn * (BN / WN) + j * 16 + lg;
          float g[4], u[4], dg[4], du[4], wa[4];
          load4<VEC>(x.pre + (row0 + m) * 2 * F, f, F, g);
          load4<VEC>(x.pre + (row0 + m) * 2 * F + F, f, F, u);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float s = sigmoid(g[q]), d = acc[i][j][q], sg = g[q] * s;
            part += f + q < F ? d * (sg * u[q]) : 0.0f;
            wa[q] = w * (sg * u[q]);
            du[q] = w * d * sg;
            // s (1 + g (1 - s)), 1 - s without the cancellation
            dg[q] = w * d * u[q] * (s + sg * sigmoid(-g[q]));
          }
          store4<VEC>(static_cast<T*>(x.wact) + (row0 + m) * F, f, F, wa);
          store4<VEC>(static_cast<T*>(x.dpre) + (row0 + m) * 2 * F, f, F, dg);
          store4<VEC>(static_cast<T*>(x.dpre) + (row0 + m) * 2 * F + F, f, F, du);
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
          if constexpr (kF32) store4<VEC>(c32 + (row0 + m) * N, n, N, v);
          else store4<VEC>(ct + (e * M + m0 + m) * N, n, N, v);
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

// One tile of BM x BN by WM x WN waves, for any sizes and alignment: elements are loaded one by
// one.
template <typename T, Kind KIND, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN* kWave) void ex_product(Experts x) {
  constexpr int kThr = WM * WN * kWave;
  constexpr int kE = 16 / sizeof(T);         // elements of a chunk
  constexpr int kBK = kRowBytes / sizeof(T);  // k staged at a time
  constexpr bool kWeightsKind = KIND == kWeightsIn || KIND == kWeightsOut;
  constexpr bool kTrA = kWeightsKind;
  constexpr bool kTrB = kWeightsKind || KIND == kBackwardGate || KIND == kBackwardIn;
  constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
  static_assert(BN >= kDotColumns || KIND != kBackwardGate);
  __shared__ __attribute__((aligned(16))) char smem[(BM + BN) * kRowBytes];
  char* const sa = smem;
  char* const sb = smem + BM * kRowBytes;

  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
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
    int32_t id = blockIdx.x;
    n0 = id % tiles_n * BN;
    id /= tiles_n;
    m0 = id % tiles_m * BM;
    e = id / tiles_m;
    mrows = M - m0;
    row0 = x.plan.offsets[e];
    K = x.plan.offsets[e + 1] - static_cast<int32_t>(row0);
  } else {
    const int32_t id = blockIdx.x / tiles_n;
    if (id >= *x.plan.tile_count * (kPlanRows / BM)) return;
    n0 = blockIdx.x % tiles_n * kCols;
    const int2 t = x.plan.tiles[id / (kPlanRows / BM)];
    e = t.x;
    m0 = 0;
    row0 = t.y + id % (kPlanRows / BM) * BM;
    mrows = x.plan.offsets[e + 1] - static_cast<int32_t>(row0);
    if (mrows <= 0) return;
    K = KIND == kForwardGate || KIND == kBackwardGate ? D : KIND == kForwardOut ? F : 2 * F;
  }

  // element (row, k) of the operands, 0 outside
  const auto token = [&](int64_t r) { return x.plan.token[r]; };
  const auto row_a = [&](int32_t m) -> const T* {  // k contiguous
    if (m >= mrows) return nullptr;
    if constexpr (KIND == kForwardGate)
      return static_cast<const T*>(x.x) + token(row0 + m) * x.x_stride;
    else if constexpr (KIND == kForwardOut)
      return static_cast<const T*>(x.act) + (row0 + m) * F;
    else if constexpr (KIND == kBackwardGate)
      return static_cast<const T*>(x.dout) + static_cast<int64_t>(token(row0 + m)) * D;
    else
      return static_cast<const T*>(x.dpre) + (row0 + m) * 2 * F;
  };
  const auto row_b = [&](int32_t c) -> const T* {  // k contiguous
    if constexpr (KIND == kForwardGate) {
      // a wave's columns: half of them gates, half the same columns' ups
      constexpr int kW = BN / WN, kHalf = kW / 2;
      const int32_t f = n0 + c / kW * kHalf + c % kHalf;
      const int q = c % kW / kHalf;
      if (f >= F) return nullptr;
      return static_cast<const T*>(x.w1) + (static_cast<int64_t>(e) * 2 * F + q * F + f) * D;
    } else {
      if (n0 + c >= D) return nullptr;
      return static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + n0 + c) * F;
    }
  };
  const auto krow_a = [&](int32_t k) -> const T* {  // m contiguous
    if constexpr (KIND == kWeightsIn)
      return static_cast<const T*>(x.dpre) + (row0 + k) * 2 * F + m0;
    else
      return static_cast<const T*>(x.dout) + static_cast<int64_t>(token(row0 + k)) * D + m0;
  };
  const auto krow_b = [&](int32_t k) -> const T* {  // n contiguous
    if constexpr (KIND == kWeightsIn)
      return static_cast<const T*>(x.x) + token(row0 + k) * x.x_stride + n0;
    else if constexpr (KIND == kWeightsOut)
      return static_cast<const T*>(x.wact) + (row0 + k) * F + n0;
    else if constexpr (KIND == kBackwardGate)
      return static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + k) * F + n0;
    else
      return static_cast<const T*>(x.w1) + (static_cast<int64_t>(e) * 2 * F + k) * D + n0;
  };
  const auto stage_k = [&](char* tile, int rows, int32_t k0, const auto& row) {
    for (int i = tid; i < rows * 8; i += kThr) {
      const int r = i >> 3, c = chunk_k(r, i & 7);
      const T* p = row(r);
      Vec<T, kE> v;
#pragma unroll
      for (int j = 0; j < kE; ++j) {
        const int32_t k = k0 + c * kE + j;
        v.v[j] = p && k < K ? p[k] : from_float<T>(0.0f);
      }
      *reinterpret_cast<Vec<T, kE>*>(tile + i * 16) = v;
    }
  };
  const auto stage_n = [&](char* tile, auto width, int32_t k0, int32_t cols, const auto& row) {
    constexpr int kC = decltype(width)::value / kE;  // chunks of a row
    for (int i = tid; i < kBK * kC; i += kThr) {
      const int r = i / kC, c = chunk_n<T>(r, i % kC);
      const int32_t k = k0 + r;
      const T* p = k < K ? row(k) : nullptr;
      Vec<T, kE> v;
#pragma unroll
      for (int j = 0; j < kE; ++j)
        v.v[j] = p && c * kE + j < cols ? p[c * kE + j] : from_float<T>(0.0f);
      *reinterpret_cast<Vec<T, kE>*>(tile + i * 16) = v;
    }
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  for (int32_t k0 = 0; k0 < K; k0 += kBK) {
    if constexpr (kTrA) stage_n(sa, std::integral_constant<int, BM>(), k0, mrows, krow_a);
    else stage_k(sa, BM, k0, row_a);
    if constexpr (kTrB) stage_n(sb, std::integral_constant<int, BN>(), k0, N - n0, krow_b);
    else stage_k(sb, BN, k0, row_b);
    __syncthreads();
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
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
    }
    __syncthreads();
  }

  finish<T, KIND, BM, BN, WM, WN, false>(x, acc, reinterpret_cast<float*>(smem), e, m0, mrows, n0,
                                         row0);
}

// ------------------------------------------------------------------ aligned operands ----

// 16 zero bytes that lanes load where an operand has no more k
__device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};

// 16 bytes a lane from its address to LDS offset `at` + 16 lane, without a register between.
// The compiler does not count these loads: await_loads() does (with the builtin of this load the
// compiler waits for all of them before every read of LDS, as it cannot tell the buffers apart).
// m0 is a reserved register, which the compiler sets right before an instruction that reads it;
// no other instruction of these kernels does.
__device__ __forceinline__ void load_to_lds(const void* p, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(at), "v"(p)
               : "memory");
}
// Waits until they and this wave's reads of LDS are done.
__device__ __forceinline__ void await_loads() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}

// The tile's place in the XCD that runs it: workgroups go round the 8 XCDs, so each XCD takes a
// contiguous eighth of the tiles, whose operands then stay in its own L2.
__device__ __forceinline__ int32_t spread(int32_t total) {
  const int32_t per = (total + 7) / 8;
  const int32_t in = blockIdx.x >> 3, id = (blockIdx.x & 7) * per + in;
  return in < per && id < total ? id : -1;
}

// One tile of BM x BN by WM x WN waves.  Rows of every operand start at a multiple of 16 bytes
// and hold a multiple of 16 bytes.
template <typename T, Kind KIND, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN* kWave) void ex_tiles(Experts x) {
  constexpr int kThr = WM * WN * kWave, kWaves = WM * WN;
  constexpr int kE = 16 / sizeof(T);          // elements of a chunk
  constexpr int kBK = kRowBytes / sizeof(T);  // k staged at a time
  constexpr bool kWeightsKind = KIND == kWeightsIn || KIND == kWeightsOut;
  constexpr bool kTrA = kWeightsKind;
  constexpr bool kTrB = kWeightsKind || KIND == kBackwardGate || KIND == kBackwardIn;
  constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
  constexpr int LA = BM * 8 / kThr, LB = BN * 8 / kThr;  // chunks a lane loads of each operand
  constexpr int kStage = (BM + BN) * kRowBytes;
  __shared__ __attribute__((aligned(1024))) char smem[2 * kStage];

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
    int32_t id = spread(x.experts * tiles_m * tiles_n);
    if (id < 0) return;
    n0 = id % tiles_n * BN;
    id /= tiles_n;
    m0 = id % tiles_m * BM;
    e = id / tiles_m;
    mrows = M - m0;
    row0 = x.plan.offsets[e];
    K = x.plan.offsets[e + 1] - static_cast<int32_t>(row0);
  } else {
    constexpr int kParts = kPlanRows / BM;
    int32_t id = spread(*x.plan.tile_count * kParts * tiles_n);
    if (id < 0) return;
    n0 = id % tiles_n * kCols;
    id /= tiles_n;
    const int2 t = x.plan.tiles[id / kParts];
    e = t.x;
    m0 = 0;
    row0 = t.y + id % kParts * BM;
    mrows = x.plan.offsets[e + 1] - static_cast<int32_t>(row0);
    if (mrows <= 0) return;
    K = KIND == kForwardGate || KIND == kBackwardGate ? D : KIND == kForwardOut ? F : 2 * F;
  }

  // What this lane loads.  k contiguous: chunk (row, c) of the staged rows, at a pointer that
  // moves on by 128 bytes; rows past the last load the last one (their results are not stored).
  // k as rows: chunk c of row k, at a pointer that moves on by kBK rows, or of a gathered row.
  const char* pa[LA];
  const char* pb[LB];
  int32_t ka[LA], kb[LB];  // k of the chunk in the first stage
  const char* const zeros = reinterpret_cast<const char*>(kZeros);
#pragma unroll
  for (int j = 0; j < LA; ++j) {
    const int i = (j * kWaves + wave) * kWave + lane;
    if constexpr (!kTrA) {
      const int r = i >> 3, c = chunk_k(r, i & 7);
      const int64_t row = row0 + (r < mrows ? r : mrows - 1);
      const T* p;
      if constexpr (KIND == kForwardGate)
        p = static_cast<const T*>(x.x) + x.plan.token[row] * x.x_stride;
      else if constexpr (KIND == kForwardOut)
        p = static_cast<const T*>(x.act) + row * F;
      else if constexpr (KIND == kBackwardGate)
        p = static_cast<const T*>(x.dout) + static_cast<int64_t>(x.plan.token[row]) * D;
      else
        p = static_cast<const T*>(x.dpre) + row * 2 * F;
      ka[j] = c * kE;
      pa[j] = reinterpret_cast<const char*>(p + c * kE);
    } else {
      constexpr int kC = BM / kE;
      const int r = i / kC, c = chunk_n<T>(r, i % kC);
      ka[j] = r;
      const int32_t m = m0 + c * kE;
      // past the last column: no k (zeros)
      if (c * kE >= mrows) ka[j] = INT32_MAX / 2;
      if constexpr (KIND == kWeightsIn)
        pa[j] = reinterpret_cast<const char*>(static_cast<const T*>(x.dpre) + (row0 + r) * 2 * F +
                                              m);
      else
        pa[j] = reinterpret_cast<const char*>(static_cast<const T*>(x.dout) + m);
    }
  }
#pragma unroll
  for (int j = 0; j < LB; ++j) {
    const int i = (j * kWaves + wave) * kWave + lane;
    if constexpr (!kTrB) {
      const int r = i >> 3, c = chunk_k(r, i & 7);
      const T* p;
      if constexpr (KIND == kForwardGate) {
        constexpr int kW = BN / WN, kHalf = kW / 2;
        int32_t f = n0 + r / kW * kHalf + r % kHalf;
        if (f >= F) f = F - 1;
        p = static_cast<const T*>(x.w1) +
            (static_cast<int64_t>(e) * 2 * F + r % kW / kHalf * F + f) * D;
      } else {
        const int32_t n = n0 + r < D ? n0 + r : D - 1;
        p = static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + n) * F;
      }
      kb[j] = c * kE;
      pb[j] = reinterpret_cast<const char*>(p + c * kE);
    } else {
      constexpr int kC = BN / kE;
      const int r = i / kC, c = chunk_n<T>(r, i % kC);
      kb[j] = r;
      const int32_t n = n0 + c * kE;
      if (n >= N) kb[j] = INT32_MAX / 2;
      const T* p;
      if constexpr (KIND == kWeightsIn) p = static_cast<const T*>(x.x) + n;
      else if constexpr (KIND == kWeightsOut)
        p = static_cast<const T*>(x.wact) + (row0 + r) * F + n;
      else if constexpr (KIND == kBackwardGate)
        p = static_cast<const T*>(x.w2) + (static_cast<int64_t>(e) * D + r) * F + n;
      else
        p = static_cast<const T*>(x.w1) + (static_cast<int64_t>(e) * 2 * F + r) * D + n;
      pb[j] = reinterpret_cast<const char*>(p);
    }
  }
  // bytes from one stage to the next
  const int64_t step_a = !kTrA ? kRowBytes : int64_t{kBK} * 2 * F * sizeof(T);
  const int64_t step_b = !kTrB ? kRowBytes
                         : KIND == kBackwardIn ? int64_t{kBK} * D * sizeof(T)
                                               : int64_t{kBK} * F * sizeof(T);
  const uint32_t lds = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem));

  // Rows gathered as k: the tokens of the next stage to load are read one stage before.
  constexpr int LG = KIND == kWeightsIn ? LB : KIND == kWeightsOut ? LA : 1;
  int32_t token[LG];
  const auto gather = [&](int32_t k0) {
    if constexpr (kWeightsKind) {
#pragma unroll
      for (int j = 0; j < LG; ++j) {
        const int32_t k = k0 + (KIND == kWeightsIn ? kb[j] : ka[j]);
        token[j] = k < K ? x.plan.token[row0 + k] : 0;
      }
    }
  };
  const int64_t row_bytes =
      (KIND == kWeightsIn ? x.x_stride : static_cast<int64_t>(D)) * static_cast<int>(sizeof(T));
  const auto issue = [&](int32_t k0, int buf) {
    const uint32_t at = lds + buf * kStage + wave * (kWave * 16);
    const char* p[LA + LB];
#pragma unroll
    for (int j = 0; j < LA; ++j) {
      p[j] = zeros;
      if constexpr (KIND == kWeightsOut) {
        if (k0 + ka[j] < K) p[j] = pa[j] + token[j] * row_bytes;
      } else {
        if (k0 + ka[j] < K) p[j] = pa[j];
        pa[j] += step_a;
      }
    }
#pragma unroll
    for (int j = 0; j < LB; ++j) {
      p[LA + j] = zeros;
      if constexpr (KIND == kWeightsIn) {
        if (k0 + kb[j] < K) p[LA + j] = pb[j] + token[j] * row_bytes;
      } else {
        if (k0 + kb[j] < K) p[LA + j] = pb[j];
        pb[j] += step_b;
      }
    }
#pragma unroll
    for (int j = 0; j < LA; ++j) load_to_lds(p[j], at + j * (kThr * 16));
#pragma unroll
    for (int j = 0; j < LB; ++j)
      load_to_lds(p[LA + j], at + BM * kRowBytes + j * (kThr * 16));
    gather(k0 + kBK);
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  gather(0);
  if (K > 0) issue(0, 0);
  int buf = 0;
  for (int32_t k0 = 0; k0 < K; k0 += kBK, buf ^= 1) {
    await_loads();
    __builtin_amdgcn_s_barrier();
    if (k0 + kBK < K) issue(k0 + kBK, buf ^ 1);
    const char* const sa = smem + buf * kStage;
    const char* const sb = sa + BM * kRowBytes;
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
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
    }
  }
  if constexpr (KIND == kBackwardGate) __syncthreads();
  finish<T, KIND, BM, BN, WM, WN, true>(x, acc, reinterpret_cast<float*>(smem), e, m0, mrows, n0,
                                        row0);
}
// out[t] = sum_k weight[t, k] y[row of (t, k)], k ascending, in binary32, rounded once
template <typename T, bool WEIGHTED>
__global__ __launch_bounds__(256) void ex_join(Experts x, const float* __restrict__ y,
                                               T* __restrict__ out) {
  const int64_t t = blockIdx.x;
  for (int32_t d = threadIdx.x; d < x.dim; d += 256) {
    float s = 0.0f;
    for (int k = 0; k < x.top; ++k) {
      const int64_t j = t * x.top + k;
      const int32_t r = x.plan.pos[j];
      if (r < 0) continue;
      const float v = y[static_cast<int64_t>(r) * x.dim + d];
      s += WEIGHTED ? x.weights[j] * v : v;
    }
    out[t * x.dim + d] = from_float<T>(s);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void ex_dots(Experts x) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (j >= x.pairs) return;
  const int32_t r = x.plan.pos[j];
  float s = 0.0f;
  if (r >= 0)
    for (int i = 0; i < x.dot_tiles; ++i) s += x.dots[static_cast<int64_t>(r) * x.dot_tiles + i];
  x.dweights[j] = s;
}

inline uint32_t blocks_of(int64_t n, int64_t per) {
  return static_cast<uint32_t>((n + per - 1) / per);
}

// Whether rows and their starts are multiples of 16 bytes.
template <typename T>
bool aligned(const Experts& x) {
  constexpr int kE = 16 / sizeof(T);
  return x.dim % kE == 0 && x.hidden % kE == 0 && x.x_stride % kE == 0 && aligned16(x.x) &&
         aligned16(x.w1) && aligned16(x.w2) && aligned16(x.out) && aligned16(x.dout) &&
         aligned16(x.dx) && aligned16(x.dw1) && aligned16(x.dw2);
}

template <typename T, Kind KIND>
void product(Experts x, hipStream_t st) {
  if (aligned<T>(x)) {
    constexpr int BM = EX_BM, BN = EX_BN;
    x.dot_tiles = static_cast<int32_t>(blocks_of(x.hidden, BN));
    const uint32_t n = blocks_of(KIND == kForwardGate || KIND == kBackwardGate ||
                                 KIND == kWeightsOut ? x.hidden : x.dim,
                                 KIND == kForwardGate ? BN / 2 : BN);
    uint32_t grid = KIND == kWeightsIn    ? x.experts * blocks_of(2 * x.hidden, BM) * n
                    : KIND == kWeightsOut ? x.experts * blocks_of(x.dim, BM) * n
                                          : x.plan.most_tiles * (kPlanRows / BM) * n;
    grid = (grid + 7) / 8 * 8;
    ex_tiles<T, KIND, BM, BN, EX_WM, EX_WN><<<grid, EX_WM * EX_WN * kWave, 0, st>>>(x);
    return;
  }
  constexpr int BM = 128, BN = 128;
  constexpr int kCols = KIND == kForwardGate ? BN / 2 : BN;
  uint32_t grid;
  if constexpr (KIND == kWeightsIn)
    grid = x.experts * blocks_of(2 * x.hidden, BM) * blocks_of(x.dim, BN);
  else if constexpr (KIND == kWeightsOut)
    grid = x.experts * blocks_of(x.dim, BM) * blocks_of(x.hidden, BN);
  else
    grid = x.plan.most_tiles * (kPlanRows / BM) *
           blocks_of(KIND == kForwardGate || KIND == kBackwardGate
                                             ? x.hidden : x.dim, kCols);
  if (grid > 0) ex_product<T, KIND, BM, BN, 2, 2><<<grid, 256, 0, st>>>(x);
}

}  // namespace

template <typename T>
hipError_t launch_experts(const Experts& x, hipStream_t st) {
  const hipError_t e = launch_plan(x, st);
  if (e != hipSuccess) return e;
  product<T, kForwardGate>(x, st);
  product<T, kForwardOut>(x, st);
  ex_join<T, true><<<static_cast<uint32_t>(x.tokens), 256, 0, st>>>(x, x.y,
                                                                    static_cast<T*>(x.out));
  return hipGetLastError();
}

template <typename T>
hipError_t launch_experts_backward(const Experts& x, hipStream_t st) {
  if (x.pairs > 0) {
    product<T, kBackwardGate>(x, st);
    Experts d = x;
    if (aligned<T>(x)) d.dot_tiles = static_cast<int32_t>(blocks_of(x.hidden, EX_BN));
    if (x.dweights) ex_dots<T><<<blocks_of(x.pairs, 256), 256, 0, st>>>(d);
  }
  if (x.dx && x.tokens > 0) {
    product<T, kBackwardIn>(x, st);
    ex_join<T, false><<<static_cast<uint32_t>(x.tokens), 256, 0, st>>>(x, x.dxr,
                                                                       static_cast<T*>(x.dx));
  }
  if (x.dw1) product<T, kWeightsIn>(x, st);
  if (x.dw2) product<T, kWeightsOut>(x, st);
  return hipGetLastError();
}

}  // namespace gsn
