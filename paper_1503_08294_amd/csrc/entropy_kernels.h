// Kernels of the softmax cross entropy for one type of element, included by one source a type.
//
//   l(t, c) = x[t] . w[c] over the valid classes c,  loss = log sum exp(l) - l(target)
//   d = dloss (exp(l) / sum exp(l) - [c = target]),  dx = d w,  dw = d^T x
// The logits are not kept: a tile of them is reduced to its rows' largest value and sum of
// exponentials, and the backward pass makes them again, a piece of the classes at a time, as d.
//
// Logits of binary32 operands in two values (TWO): the matrix cores multiply float16 at 9 times the
// rate that they multiply binary32 at (1.43 and 0.153 PFLOP/s in large library products).  A row of
// x or w is kept times a power of two, which takes its largest element to 2^14 to 2^15, as hi =
// float16(v) and lo = float16(v - hi): 22 bits of every element down to 2^-18 of the largest, 2^-40
// of it below.  A product is hi lo + lo hi + hi hi, three products of one binary32 sum.  What a
// logit loses so is small beside the row's others, and in pieces of the classes for which it is not
// they are made in binary32 (two_will_do()).  The gradients' products take binary32 operands:
// a class that every token finds improbable has a row of dw that is a sum of small terms alone, and
// a token's or a feature's may be, so that no one scale has room for all of them in float16.
//
// Bound by the products.  8,192 tokens, 131,072 classes of 2,048, bfloat16: logits reduced 4.0 ms,
// made again as d 4.7 (in four pieces, 2.1 GB written), dx 3.9, dw 3.9; joins, sums and copies
// 0.05.  1,777 tokens, 10,007 classes of 501, binary32, logits in two values: 78, 84, 189 and 200 us,
// 90 for splitting into two values, copies and joins, and for launches that end at once.  (With d, w
// and x in two values as well dx and dw took 67 and 104, and lost classes whose probabilities are
// below some 2^-24 of the largest.)
#pragma once

#include "entropy.h"
#include "few.h"
#include "product.h"

namespace gsn {
namespace {

// What gradients of logits that are kept in float16 are at most.
constexpr float kMostKept = 0x1p15f;

// A token's target, -1 where there is none: out of range, or a class that is not valid.
__device__ __forceinline__ int32_t target_of(const Entropy& x, int64_t t) {
  const int32_t c = x.targets[t];
  if (c < 0 || c >= x.classes) return -1;
  return x.valid && !x.valid[c] ? -1 : c;
}

// e^v of a difference to the largest logit (or to the sum's logarithm).
template <typename T>
__device__ __forceinline__ float power(float v) {
  // (__expf's error grows with -v, to some (|v| + 3) 2^-24: too much for results of 32 bits)
  if constexpr (sizeof(T) == 4) return expf(v);
  else return __expf(v);
}

// Of a lane's columns n + 16 j + q: bit 4 j + q for one that is no valid class.
template <int NT>
__device__ __forceinline__ uint32_t shut_columns(const uint8_t* valid, int32_t classes, int32_t n) {
  uint32_t shut = 0;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int32_t c = n + 16 * j + q;
      const bool out = c >= classes || (valid && !valid[c]);
      shut |= out ? 1u << (4 * j + q) : 0u;
    }
  return shut;
}

// (largest, sum of exp(. - largest)) of two sets of logits.
__device__ __forceinline__ float2 merged(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  const float base = m == -INFINITY ? 0.0f : m;
  return float2{m, a.y * expf(a.x - base) + b.y * expf(b.x - base)};
}

// The logits of rows and columns that were kept times powers of two (which may be too small for
// binary32 themselves).
template <int MT, int NT>
__device__ __forceinline__ void unscale(const Entropy& x, f32x4 (&acc)[MT][NT], int64_t m,
                                        int32_t n, int lane) {
  i32x4 cols[NT];
  // (columns past the last class are not used, but read: ew has room for them)
#pragma unroll
  for (int j = 0; j < NT; ++j)
    cols[j] = *reinterpret_cast<const i32x4*>(x.ew + n + 16 * j + (lane >> 4) * 4);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t t = m + 16 * i + (lane & 15);
    const int32_t row = x.ex[t < x.tokens ? t : x.tokens - 1];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[i][j][q] = ldexpf(acc[i][j][q], row + cols[j][q]);
  }
}

// Whether a piece's logits are made of two values.  An element that is kept so is off by 2^-23 of
// itself or by 2^-39 of its row's largest, X or W, so that beside the errors of binary32 a logit
// has one of 2^-39 (X sum |w| + W sum |x|).  It is at most 2^-24, a rounding of a number near 1, or
// the logits are made in binary32: rows may hold a number far larger than the others, by which a
// feature shuts classes out for some tokens, say, and infinities and NaN.
__device__ __forceinline__ bool two_will_do(const Entropy& x, int32_t index) {
  const uint32_t* const w = x.sizes + 2 * (1 + index);
  return __uint_as_float(x.sizes[0]) * __uint_as_float(w[1]) +
             __uint_as_float(w[0]) * __uint_as_float(x.sizes[1]) <= 0x1p15f;
}
// Whether these logits are the ones to make.
template <typename T, bool TWO>
__device__ __forceinline__ bool logits_wanted(const Entropy& x, int32_t index) {
  if constexpr (sizeof(T) == 4) return !x.two || two_will_do(x, index) == TWO;
  else return true;
}

// A tile of the logits -> (largest, sum) of each row, and the target's logit.
template <typename T, bool TWO>
struct Reduce {
  Entropy x;
  int32_t first, index;  // the piece's first class, and its number

  __device__ __forceinline__ bool wanted() const { return logits_wanted<T, TWO>(x, index); }

  template <class TILE, int MT, int NT>
  __device__ __forceinline__ void tile(f32x4 (&acc)[MT][NT], const Place& at, int mw, int nw,
                                       int lane, char* smem) const {
    constexpr int BM = TILE::BM, BN = TILE::BN;
    const int li = lane & 15, lg = (lane >> 4) * 4;
    float2* const rows = reinterpret_cast<float2*>(smem);  // [2][BM]
    const int32_t n = first + at.n0 + nw + lg;
    const uint32_t shut = shut_columns<NT>(x.valid, x.classes, n);
    if constexpr (TWO) unscale(x, acc, int64_t{at.m0} + mw, at.n0 + nw, lane);
    if (__any(shut != 0))
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (shut >> (4 * j + q) & 1) acc[i][j][q] = -INFINITY;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t t = at.m0 + mw + 16 * i + li;
      const int32_t place = (t < x.tokens ? x.targets[t] : -1) - n;
      if (__any(place >= 0 && place < 16 * NT)) {  // (few tiles hold a target)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (place == 16 * j + q) x.chosen[t] = acc[i][j][q];
      }
      float top = acc[i][0][0];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) top = fmaxf(top, acc[i][j][q]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float base = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) sum += power<T>(acc[i][j][q] - base);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (lane < 16) rows[nw / (BN / 2) * BM + mw + 16 * i + li] = float2{top, sum};
    }
    __syncthreads();
    for (int m = threadIdx.x; m < BM; m += kProductThreads) {
      const int64_t t = int64_t{at.m0} + m;
      if (t >= x.tokens) break;
      x.part[at.n0 / BN * x.tokens + t] = merged(rows[m], rows[BM + m]);
    }
  }
};

// The same of a few tokens' logits.
struct ReduceFew {
  Entropy x;
  __device__ __forceinline__ void few(int32_t m, int32_t n, f32x4 v) const {
    const int32_t target = x.targets[m];
    float top = -INFINITY;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (n + q >= x.classes || (x.valid && !x.valid[n + q])) v[q] = -INFINITY;
      else if (n + q == target) x.chosen[m] = v[q];
      top = fmaxf(top, v[q]);
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += expf(v[q] - base);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor(sum, o);
    if ((n & 31) == 0) x.part[n / kFewCols * x.tokens + m] = float2{top, sum};
  }
};

// The parts of a piece, and of the pieces before it, joined; after the last piece the losses.
__device__ __forceinline__ void finish_token(const Entropy& x, int64_t t, float2 v, bool last) {
  if (last) {
    const int32_t target = target_of(x, t);
    // (the logarithm of the sum and the difference to the largest are each small: their difference
    // keeps the digits that one to the logarithm of all would lose)
    x.loss[t] = target < 0 ? 0.0f : logf(v.y) - (x.chosen[t] - v.x);
    if (target < 0) v = float2{0.0f, 1.0f};
  }
  x.stats[t] = v.x;
  x.stats[x.tokens + t] = v.y;
}

// A piece's parts, of logits in two values and of others, and whether it is the first and the last.
struct Parts {
  int32_t two, one, index, begin, last;
  __device__ __forceinline__ int32_t of(const Entropy& x) const {
    return x.two && two_will_do(x, index) ? two : one;
  }
};
// A workgroup a token, where there are few tokens.
constexpr int kFewJoin = 512;
__global__ __launch_bounds__(kFewJoin) void ce_join_few(Entropy x, Parts p) {
  __shared__ float2 some[kFewJoin / kWave];
  const int tid = threadIdx.x;
  const int64_t t = blockIdx.x;
  const int32_t parts = p.of(x);
  float2 v{-INFINITY, 0.0f};
#pragma unroll 4
  for (int32_t i = tid; i < parts; i += kFewJoin) v = merged(v, x.part[i * x.tokens + t]);
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1)
    v = merged(v, float2{__shfl_xor(v.x, o), __shfl_xor(v.y, o)});
  if (tid % kWave == 0) some[tid / kWave] = v;
  __syncthreads();
  if (tid > 0) return;
  v = some[0];
  for (int w = 1; w < kFewJoin / kWave; ++w) v = merged(v, some[w]);
  if (!p.begin) v = merged(float2{x.stats[t], x.stats[x.tokens + t]}, v);
  finish_token(x, t, v, p.last);
}
constexpr int kJoinTokens = 64, kJoinWaves = 16;
__global__ __launch_bounds__(kJoinTokens* kJoinWaves) void ce_join(Entropy x, Parts p) {
  __shared__ float2 some[kJoinWaves][kJoinTokens];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kJoinTokens + lane;
  const int32_t parts = p.of(x);
  float2 v{-INFINITY, 0.0f};
  if (t < x.tokens) {
#pragma unroll 4
    for (int32_t i = wave; i < parts; i += kJoinWaves) v = merged(v, x.part[i * x.tokens + t]);
  }
  some[wave][lane] = v;
  __syncthreads();
  if (wave > 0 || t >= x.tokens) return;
  if (!p.begin) v = merged(float2{x.stats[t], x.stats[x.tokens + t]}, v);
  for (int w = 1; w < kJoinWaves; ++w) v = merged(v, some[w][lane]);
  finish_token(x, t, v, p.last);
}

// 16 rows from t0 on of the logits' gradients, columns n0 on, in 2- or 4-byte elements.
template <typename E, int NT>
__device__ __forceinline__ void store_rows(const Entropy& x, void* d, const f32x4 (&v)[NT],
                                           int64_t t0, int32_t n0, int lane, char* room) {
  using Lines = Turn<E, 16 * NT>;
  const Lines turn{room};
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const float some[4] = {v[j][0], v[j][1], v[j][2], v[j][3]};
    turn.put(lane & 15, 16 * j + (lane >> 4) * 4, some);
  }
  wave_fence();
  const int64_t left = x.tokens - t0;
  turn.out(static_cast<E*>(d) + t0 * x.piece + n0, x.piece,
           static_cast<int32_t>(left < 16 ? left : 16), x.piece - n0, lane);
  wave_fence();
}

// The same as two 2-byte values each, of which the second ones come behind all of the first.
template <typename E, int NT>
__device__ __forceinline__ void store_two(const Entropy& x, void* d, f32x4 (&v)[NT], int64_t t0,
                                          int32_t n0, int lane, char* room) {
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) v[j][q] = settled(v[j][q]);
  store_rows<E>(x, d, v, t0, n0, lane, room);
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) v[j][q] -= to_float(from_float<E>(v[j][q]));
  store_rows<E>(x, static_cast<E*>(d) + x.tokens * x.piece, v, t0, n0, lane, room);
}

// A tile of the logits -> their gradients, as the operand of the two products that take them:
// rounded to the operands' type (two_d: to two values of it).
template <typename T, bool TWO>
struct Gradient {
  Entropy x;
  int32_t first, index;  // the piece's first class, and its number

  __device__ __forceinline__ bool wanted() const { return logits_wanted<T, TWO>(x, index); }

  template <class TILE, int MT, int NT>
  __device__ __forceinline__ void tile(f32x4 (&acc)[MT][NT], const Place& at, int mw, int nw,
                                       int lane, char* smem) const {
    const int li = lane & 15, lg = (lane >> 4) * 4;
    const int32_t n = at.n0 + nw + lg;
    const uint32_t shut = shut_columns<NT>(x.valid, x.classes, first + n);
    constexpr bool kScaled = __is_same(T, f16_t);
    const float factor = kScaled ? x.factor[0] : 1.0f;
    const bool masked = __any(shut != 0);
    char* const room = smem + threadIdx.x / kWave * (TILE::kLds / 4);
    static_assert(Turn<T, 16 * NT>::kBytes <= TILE::kLds / 4);
    if constexpr (TWO) unscale(x, acc, int64_t{at.m0} + mw, at.n0 + nw, lane);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t t0 = at.m0 + mw + 16 * i, t = t0 + li;
      if (t0 >= x.tokens) break;
      const int64_t tt = t < x.tokens ? t : x.tokens - 1;
      const int32_t target = target_of(x, tt);
      const int32_t place = target - first - n;
      const float top = x.stats[tt], g = x.dloss[tt] * factor;
      const float each = g / x.stats[x.tokens + tt];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[i][j][q] = power<T>(acc[i][j][q] - top) * each;
      if (__any(place >= 0 && place < 16 * NT)) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (place == 16 * j + q) acc[i][j][q] -= g;
      }
      if (masked || __any(target < 0)) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (target < 0 || (shut >> (4 * j + q) & 1)) acc[i][j][q] = 0.0f;
      }
      if constexpr (sizeof(T) == 2) {
        if (x.two_d) {
          store_two<T>(x, x.d, acc[i], t0, at.n0 + nw, lane, room);
          continue;
        }
      }
      store_rows<T>(x, x.d, acc[i], t0, at.n0 + nw, lane, room);
    }
  }
};

// A tile of sums of 32 bits in memory, added to what is there or not.
struct Partial {
  float* to;
  int64_t split;  // elements from a split to the next
  int32_t rows, pitch;
  int32_t add;

  template <class TILE, int MT, int NT>
  __device__ __forceinline__ void tile(f32x4 (&acc)[MT][NT], const Place& at, int mw, int nw,
                                       int lane, char*) const {
    const int32_t n = at.n0 + nw + (lane >> 4) * 4;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int32_t m = at.m0 + mw + 16 * i + (lane & 15);
      if (m >= rows) break;
      float* const row = to + at.split * split + static_cast<int64_t>(m) * pitch;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (n + 16 * j >= pitch) break;
        f32x4* const p = reinterpret_cast<f32x4*>(row + n + 16 * j);
        *p = add ? acc[i][j] + *p : acc[i][j];
      }
    }
  }
};

// A tile of dw, rounded to its type.
template <typename T>
struct Weights {
  Entropy x;
  int32_t first, count;

  template <class TILE, int MT, int NT>
  __device__ __forceinline__ void tile(f32x4 (&acc)[MT][NT], const Place& at, int mw, int nw,
                                       int lane, char*) const {
    const int32_t n = at.n0 + nw + (lane >> 4) * 4;
    const float factor = __is_same(T, f16_t) ? x.factor[1] : 1.0f;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int32_t m = at.m0 + mw + 16 * i + (lane & 15);
      if (m >= count) break;
      const bool shut = x.valid && !x.valid[first + m];
      T* const row = static_cast<T*>(x.dw) + static_cast<int64_t>(first + m) * x.dim;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = shut ? 0.0f : acc[i][j][q] * factor;
        if (n + 16 * j < x.dim) store4(row, n + 16 * j, x.dim, v);
      }
    }
  }
};

// The splits' sums, and their one rounding.  Rows without a target, or that are no valid class, are
// zeros.
template <typename T, bool OF_TOKENS>
__global__ __launch_bounds__(256) void ce_sum(Entropy x, const float* __restrict__ part,
                                              int32_t splits, int64_t rows, int32_t first,
                                              int64_t split, T* __restrict__ out) {
  const float factor = __is_same(T, f16_t) ? x.factor[1] : 1.0f;
  const int32_t each = (x.dim + 3) / 4;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < rows * each;
       at += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t r = at / each;
    const int32_t d = static_cast<int32_t>(at - r * each) * 4;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    const bool live = OF_TOKENS ? target_of(x, r) >= 0 : !(x.valid && !x.valid[first + r]);
    // (the loads of many parts are under way together: one token, 64 parts, 14 us less)
    if (live)
#pragma unroll 16
      for (int32_t i = 0; i < splits; ++i)
        s += *reinterpret_cast<const f32x4*>(part + i * split + r * x.pitch + d);
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = s[q] * factor;
    store4(out + (first + r) * x.dim, d, x.dim, v);
  }
}

// Rows of x (OF_TOKENS) or of w from `first` on, in rows of `pitch`, with zeros at their ends.
// DEAD: rows of zeros where a token has no target or a class is not valid.  index >= 0: not if the
// logits of this piece are made of two values.
template <typename T, bool OF_TOKENS, bool DEAD>
__global__ __launch_bounds__(256) void ce_rows(Entropy x, int64_t rows, int32_t first,
                                               int32_t index, T* __restrict__ out) {
  if (index >= 0 && two_will_do(x, index)) return;
  constexpr int kE = 16 / sizeof(T);
  const T* const from = static_cast<const T*>(OF_TOKENS ? x.x : x.w);
  const int64_t stride = OF_TOKENS ? x.x_stride : x.w_stride;
  const int32_t each = x.pitch / kE;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < rows * each;
       at += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t r = at / each;
    const int32_t k = static_cast<int32_t>(at - r * each) * kE;
    const bool live =
        !DEAD || (OF_TOKENS ? target_of(x, r) >= 0 : !(x.valid && !x.valid[first + r]));
    Frag f;
    f.u = u32x4{0, 0, 0, 0};
    if (live) f = row_chunk<false>(from + (first + r) * stride, k, x.dim);
    *reinterpret_cast<u32x4*>(out + r * x.pitch + k) = f.u;
    if (OF_TOKENS && x.two_d) *reinterpret_cast<u32x4*>(out + (rows + r) * x.pitch + k) = f.u;
  }
}

// Rows of x (OF_TOKENS) or of w in two values, a wave a row, with zeros at their ends and for
// tokens without a target and classes that are not valid; the exponent of the power of two that
// gives the row back; and the rows' sizes (as bits of numbers that are not negative, whose largest
// is the same in any order, and NaN's are larger).
template <bool OF_TOKENS>
__global__ __launch_bounds__(256) void ce_pairs(Entropy x, int64_t rows, int32_t first,
                                                f16_t* __restrict__ out,
                                                int32_t* __restrict__ exponent,
                                                uint32_t* __restrict__ sizes) {
  const float* const from = static_cast<const float*>(OF_TOKENS ? x.x : x.w);
  const int64_t stride = OF_TOKENS ? x.x_stride : x.w_stride;
  const int lane = threadIdx.x % kWave;
  const int64_t other = (OF_TOKENS ? x.tokens : int64_t{x.piece}) * x.pitch;
  __shared__ uint32_t some[2][4];
  uint32_t largest = 0, longest = 0;
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave; r < rows;
       r += static_cast<int64_t>(gridDim.x) * 4) {
    const bool live = OF_TOKENS ? target_of(x, r) >= 0 : !(x.valid && !x.valid[first + r]);
    const float* const row = from + (first + r) * stride;
    float top = 0.0f, sum = 0.0f;
    if (live)
      for (int32_t k = lane * 4; k < x.dim; k += kWave * 4) {
        float v[4];
        load4(row, k, x.dim, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          top = fmaxf(top, fabsf(v[q]));
          sum += fabsf(v[q]);
        }
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      top = fmaxf(top, __shfl_xor(top, o));
      sum += __shfl_xor(sum, o);
    }
    largest = max(largest, __float_as_uint(top));
    longest = max(longest, __float_as_uint(sum) & 0x7fffffffu);
    int down = 15;  // (what is not finite stays so)
    if (top > 0.0f && top < INFINITY) frexpf(top, &down);
    const int up = 15 - down;
    for (int32_t k = lane * 8; k < x.pitch; k += kWave * 8) {
      float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      if (live) {
        load4(row, k, x.dim, v);
        load4(row, k + 4, x.dim, v + 4);
      }
      Vec<f16_t, 8> hi, lo;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float w = settled(ldexpf(v[q], up));
        hi.v[q] = from_float<f16_t>(w);
        lo.v[q] = from_float<f16_t>(w - to_float(hi.v[q]));
      }
      f16_t* const to = out + r * x.pitch + k;
      *reinterpret_cast<Vec<f16_t, 8>*>(to) = hi;
      *reinterpret_cast<Vec<f16_t, 8>*>(to + other) = lo;
    }
    if (lane == 0) exponent[r] = -up;
  }
  if (lane == 0) {
    some[0][threadIdx.x / kWave] = largest;
    some[1][threadIdx.x / kWave] = longest;
  }
  __syncthreads();
  if (threadIdx.x > 1) return;
  const uint32_t* const s = some[threadIdx.x];
  largest = max(max(s[0], s[1]), max(s[2], s[3]));
  // (most workgroups have nothing larger to tell: 10,007 rows took 118 us when all did)
  uint32_t* const to = sizes + threadIdx.x;
  if (largest > __hip_atomic_load(to, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))
    atomicMax(to, largest);
}
__global__ __launch_bounds__(256) void ce_begin(Entropy x) {
  for (int32_t i = threadIdx.x; i < 2 * (1 + x.pieces); i += 256) x.sizes[i] = 0;
}

// Gradients of the logits in float16 are kept times 2^15 / max |dloss|: at most 2^15, and those of
// small probabilities are not lost (2^-29 of the largest dloss still has all of its 11 bits).  A
// dloss that is not finite is its own token's matter.
__global__ __launch_bounds__(1024) void ce_factor(Entropy x) {
  __shared__ float some[16];
  float m = 0.0f;
  for (int64_t t = threadIdx.x; t < x.tokens; t += 1024) {
    if (target_of(x, t) < 0) continue;
    const float v = fabsf(x.dloss[t]);
    if (v < INFINITY) m = fmaxf(m, v);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if (threadIdx.x % kWave == 0) some[threadIdx.x / kWave] = m;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int w = 1; w < 16; ++w) m = fmaxf(m, some[w]);
  const float base = fmaxf(m, 0x1p-100f);
  x.factor[0] = kMostKept / base;
  x.factor[1] = base / kMostKept;
}

// A wave a row; few enough workgroups that they have little to tell each other (ce_pairs).
inline uint32_t row_blocks(int64_t rows) {
  return static_cast<uint32_t>(rows < 4 ? 1 : rows < 4096 ? rows / 4 : 1024);
}
inline uint32_t some_blocks(int64_t threads) {
  const int64_t n = (threads + 255) / 256;
  return static_cast<uint32_t>(n < 1 ? 1 : n < (1 << 16) ? n : 1 << 16);
}

template <typename T>
Operand operand_of(const void* p, int64_t ld, int64_t rows) {
  constexpr int64_t kSize = sizeof(T);
  return Operand{static_cast<const char*>(p), {0, 0}, ld * kSize, 0, static_cast<int32_t>(rows)};
}

// An operand in two values: of the terms hi lo, lo hi, hi hi (the small ones first: fewer roundings
// of a large sum), where `lo` is `other` elements behind hi.
inline Operand pair_of(const void* p, int64_t ld, int64_t rows, int64_t other, bool first) {
  const int64_t lo = 2 * other;
  return Operand{static_cast<const char*>(p) + (first ? 0 : lo),
                 {first ? lo : -lo, first ? -lo : 0}, 2 * ld, 0, static_cast<int32_t>(rows)};
}

// A product's parts of k: `splits` of them, whole stages (of any tile).
template <typename E>
void split(Product* p, int32_t splits) {
  constexpr int32_t kBK = kRowBytes / sizeof(E);
  p->splits = splits;
  p->part = ((p->k + splits - 1) / splits + kBK - 1) / kBK * kBK;
}

// x or its copy by w from class `first` on or its copy (or both in two values).
template <typename T, bool TWO>
Product logits_of(const Entropy& x, int32_t first, int32_t count) {
  Product p{};
  if constexpr (TWO) {
    p.a = pair_of(x.x2, x.pitch, x.tokens, x.tokens * x.pitch, true);
    p.b = pair_of(x.w2, x.pitch, count, int64_t{x.piece} * x.pitch, false);
    p.terms = 3;
  } else {
    p.a = x.copy_x ? operand_of<T>(x.xc, x.pitch, x.tokens)
                   : operand_of<T>(x.x, x.x_stride, x.tokens);
    p.b = x.copy_w ? operand_of<T>(x.wc, x.pitch, count)
                   : operand_of<T>(static_cast<const T*>(x.w) + first * x.w_stride, x.w_stride,
                                   count);
    p.terms = 1;
  }
  p.batch = 1;
  p.k = x.dim;
  split<T>(&p, 1);
  return p;
}

// The copies of x and of a piece of w; index as of ce_rows().
template <typename T, bool DEAD>
void copy_tokens(const Entropy& x, int32_t index, hipStream_t st) {
  const int64_t row = x.pitch / (16 / sizeof(T));
  ce_rows<T, true, DEAD><<<some_blocks(x.tokens * row), 256, 0, st>>>(x, x.tokens, 0, index,
                                                                      static_cast<T*>(x.xc));
}
template <typename T, bool DEAD>
void copy_classes(const Entropy& x, int32_t first, int32_t count, int32_t index, hipStream_t st) {
  const int64_t row = x.pitch / (16 / sizeof(T));
  ce_rows<T, false, DEAD><<<some_blocks(count * row), 256, 0, st>>>(x, count, first, index,
                                                                    static_cast<T*>(x.wc));
}
// The same in two values.
inline void pair_tokens(const Entropy& x, hipStream_t st) {
  ce_begin<<<1, 256, 0, st>>>(x);
  ce_pairs<true><<<row_blocks(x.tokens), 256, 0, st>>>(x, x.tokens, 0, static_cast<f16_t*>(x.x2),
                                                       x.ex, x.sizes);
}
inline void pair_classes(const Entropy& x, int32_t first, int32_t count, int32_t index,
                         hipStream_t st) {
  ce_pairs<false><<<row_blocks(count), 256, 0, st>>>(x, count, first, static_cast<f16_t*>(x.w2),
                                                     x.ew, x.sizes + 2 * (1 + index));
}

template <typename T, bool TWO>
void forward(const Entropy& x, hipStream_t st) {
  if constexpr (TWO) pair_tokens(x, st);
  else if (x.copy_x) copy_tokens<T, false>(x, -1, st);
  for (int32_t first = 0; first < x.classes; first += x.piece) {
    const int32_t count = x.classes - first < x.piece ? x.classes - first : x.piece;
    const int32_t index = first / x.piece;
    Parts parts{0, 0, index, first == 0, first + count == x.classes};
    if constexpr (TWO) {
      pair_classes(x, first, count, index, st);
      Product p = logits_of<T, true>(x, first, count);
      p.eighths = 1;
      with_tile<f16_t, false, false>(p, [&](auto tile) { parts.two = tiles_of(count, tile.BN); });
      run_product<f16_t, false, false>(p, Reduce<T, true>{x, first, index}, st);
      // (of pieces whose logits are made in binary32 after all)
      if (x.copy_x) copy_tokens<T, false>(x, index, st);
    }
    if (x.copy_w) copy_classes<T, false>(x, first, count, TWO ? index : -1, st);
    Product p = logits_of<T, false>(x, first, count);
    p.eighths = 1;
    with_tile<T, false, false>(p, [&](auto tile) { parts.one = tiles_of(count, tile.BN); });
    run_product<T, false, false>(p, Reduce<T, false>{x, first, index}, st);
    // (of 64 tokens, 782 parts: 10.5 us by lanes)
    if (x.tokens <= 1024)
      ce_join_few<<<static_cast<uint32_t>(x.tokens), kFewJoin, 0, st>>>(x, parts);
    else
      ce_join<<<static_cast<uint32_t>((x.tokens + kJoinTokens - 1) / kJoinTokens),
                kJoinTokens * kJoinWaves, 0, st>>>(x, parts);
  }
}

template <typename T, bool TWO>
void backward(const Entropy& x, hipStream_t st) {
  if (__is_same(T, f16_t)) ce_factor<<<1, 1024, 0, st>>>(x);
  copy_tokens<T, true>(x, -1, st);
  if constexpr (TWO) pair_tokens(x, st);
  for (int32_t first = 0; first < x.classes; first += x.piece) {
    const int32_t count = x.classes - first < x.piece ? x.classes - first : x.piece;
    const int32_t index = first / x.piece;
    if (x.copy_w) copy_classes<T, true>(x, first, count, -1, st);
    if constexpr (TWO) {
      pair_classes(x, first, count, index, st);
      run_product<f16_t, false, false>(logits_of<T, true>(x, first, count),
                                       Gradient<T, true>{x, first, index}, st);
    }
    run_product<T, false, false>(logits_of<T, false>(x, first, count),
                                 Gradient<T, false>{x, first, index}, st);
    // (second values of d are tokens of their own in both products: two terms would read w once
    // more, and take a stage more for dw)
    const int64_t rows = x.two_d ? 2 * x.tokens : x.tokens;
    if (x.dx) {
      Product p = logits_of<T, false>(x, first, count);
      p.a = operand_of<T>(x.d, x.piece, rows);
      p.b.rows = x.dim;
      p.k = count;
      split<T>(&p, x.splits_x);
      run_product<T, false, true>(
          p, Partial{x.dxp, rows * x.pitch, static_cast<int32_t>(rows), x.pitch, first > 0}, st);
    }
    if (x.dw) {
      Product p{};
      p.a = operand_of<T>(x.d, x.piece, count);
      p.b = operand_of<T>(x.xc, x.pitch, x.dim);
      p.terms = p.batch = 1;
      p.k = static_cast<int32_t>(rows);
      split<T>(&p, x.splits_w);
      if (x.splits_w > 1) {
        const int64_t each = int64_t{x.piece} * x.pitch;
        run_product<T, true, true>(p, Partial{x.dwp, each, count, x.pitch, 0}, st);
        ce_sum<T, false><<<some_blocks(int64_t{count} * ((x.dim + 3) / 4)), 256, 0, st>>>(
            x, x.dwp, x.splits_w, count, first, each, static_cast<T*>(x.dw));
      } else {
        run_product<T, true, true>(p, Weights<T>{x, first, count}, st);
      }
    }
  }
  if (x.dx)
    ce_sum<T, true><<<some_blocks(x.tokens * ((x.dim + 3) / 4)), 256, 0, st>>>(
        x, x.dxp, x.two_d ? 2 * x.splits_x : x.splits_x, x.tokens, 0, x.tokens * x.pitch,
        static_cast<T*>(x.dx));
}

}  // namespace

template <typename T>
hipError_t launch_entropy(const Entropy& x, hipStream_t st) {
  if (x.few) {
    run_few<T>(Few{x.x, x.x_stride, x.w, x.w_stride, static_cast<int32_t>(x.tokens), x.classes,
                   x.dim}, ReduceFew{x}, st);
    ce_join_few<<<static_cast<uint32_t>(x.tokens), kFewJoin, 0, st>>>(
        x, Parts{0, (x.classes + kFewCols - 1) / kFewCols, 0, 1, 1});
    return hipGetLastError();
  }
  if constexpr (sizeof(T) == 4)
    if (x.two) {
      forward<T, true>(x, st);
      return hipGetLastError();
    }
  forward<T, false>(x, st);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_entropy_backward(const Entropy& x, hipStream_t st) {
  if constexpr (sizeof(T) == 4)
    if (x.two) {
      backward<T, true>(x, st);
      return hipGetLastError();
    }
  backward<T, false>(x, st);
  return hipGetLastError();
}

}  // namespace gsn
