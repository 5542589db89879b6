// Orthogonalised matrices, and updates of weights by them.
//
//   X = x / (norm(x) + eps);  A = X X^T,  B = a I + b A + c A A,  X <- B X    `steps` times
// (of a matrix with more rows than columns A = X^T X, X <- X B: the same without a transposition).
// A and A A are symmetric: half of their tiles are made, and stored twice.  a I is a part of B, so
// that X <- B X reads X once.
//
// The products take float16 operands, the only ones of 11 bits that the matrix cores multiply at
// their full rate (binary32 at a sixteenth).  A value v is kept times 2^11 as hi = float16(v) and,
// where one is too few, lo = float16(v - hi): 22 bits, and a product of two is hi lo + lo hi + hi
// hi, three products of one sum.  Error of the result after 5 steps (2-norm, relative, matrices of
// Gaussian entries and of a few strong directions, 256 to 1,024 a side, sums in 64 bits; binary32
// throughout 2e-6 to 6e-6): one value 2e-4 to 3e-3, two 5e-7 to 7e-7, bfloat16 in their place 1e-2
// to 8e-2.  With the matrix cores' binary32 sums two values give 3e-6 to 7e-6.
// 2^11: entries are at most 5 (28 in B), a float16 holds 65,504; what is lost below its smallest
// step is 2^-36 of a largest singular value of 1.
//
// Bound by the products: 64 matrices of 2,048 x 1,024, one value: A 196 us a step,
// B 126, X 330 (0.83 PFLOP/s); the norm and the copy, bound by memory, 448 of 3,630 us.
#include <algorithm>
#include <cmath>

#include "product.h"

namespace gsn {
namespace {

constexpr float kScale = 2048.0f;

struct Orthogonal {
  int64_t batch;
  int32_t rows, cols;    // of a matrix
  int32_t rows8, cols8;  // of its copies: up to multiples of 8, zeros there
  int32_t blocks;        // parts of a matrix's norm
  int32_t steps, values;  // values: 1 or 2 a number
  float a, b, c, eps;
  // update
  const void* x;  // the matrices, or the gradients
  const float* momentum;
  float* new_momentum;
  const void* weights;
  float rate, beta, keep;  // keep: 1 - decay
  int32_t nesterov;
  void* out;
  // workspace
  double* norms;   // [batch][blocks] sums of squares
  f16_t* now[2];   // X: [values][batch][rows8][cols8], this step's and the next
  f16_t* gram;     // A: [values][batch][short8][short8]
  f16_t* poly;     // B
};

// Eight elements of a row from column c on, of which those inside are used.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int32_t c, int32_t cols, float* v) {
  load4(row, c, cols, v);
  load4(row, c + 4, cols, v + 4);
}

// What is orthogonalised, at eight elements of a row of all matrices.  The momentum is new_momentum
// by then.
template <typename T, bool UPDATE>
__device__ __forceinline__ void input8(const Orthogonal& x, int64_t row, int32_t c, float* v) {
  load8(static_cast<const T*>(x.x) + row * x.cols, c, x.cols, v);
  if constexpr (UPDATE) {
    float m[8];
    load8(x.new_momentum + row * x.cols, c, x.cols, m);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = x.nesterov ? v[q] + x.beta * m[q] : m[q];
  }
}

// Sums of squares in 64 bits (squares of binary32 leave its range), a part of a matrix a workgroup;
// and the momentum.  Bound by memory.
constexpr int kNormThreads = 256;
template <typename T, bool UPDATE>
__global__ __launch_bounds__(kNormThreads) void or_norm(Orthogonal x) {
  __shared__ double some[kNormThreads / kWave];
  const int64_t pair = blockIdx.x / x.blocks;
  const uint32_t part = static_cast<uint32_t>(blockIdx.x - pair * x.blocks);
  const uint32_t each = static_cast<uint32_t>(x.cols8) / 8, n = each * x.rows;
  double s = 0.0;
  for (uint32_t i = part * kNormThreads + threadIdx.x; i < n; i += x.blocks * kNormThreads) {
    const uint32_t r = i / each;
    const int32_t c = static_cast<int32_t>(i - r * each) * 8;
    const int64_t row = pair * x.rows + r;
    float v[8];
    if constexpr (UPDATE) {
      float m[8];
      load8(static_cast<const T*>(x.x) + row * x.cols, c, x.cols, v);
      load8(x.momentum + row * x.cols, c, x.cols, m);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        m[q] = x.beta * m[q] + v[q];
        v[q] = x.nesterov ? v[q] + x.beta * m[q] : m[q];
      }
      store4(x.new_momentum + row * x.cols, c, x.cols, m);
      store4(x.new_momentum + row * x.cols, c + 4, x.cols, m + 4);
    } else {
      input8<T, false>(x, row, c, v);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) s += static_cast<double>(v[q]) * v[q];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (threadIdx.x % kWave == 0) some[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int w = 1; w < kNormThreads / kWave; ++w) s += some[w];
  x.norms[blockIdx.x] = s;
}

// v -> 2^11 v / norm, by a power of two before where the quotient would leave binary32's range (an
// eps of 0).  A matrix of zeros without an eps stays one; an infinite norm gives NaN.
struct Inverse {
  float before, factor;
  __device__ __forceinline__ explicit Inverse(double norm) {
    before = norm < 0x1p-100 ? 0x1p60f : norm > 0x1p120 ? 0x1p-40f : 1.0f;
    factor = norm > 0.0 ? norm < INFINITY ? static_cast<float>(kScale / (norm * before)) : NAN
                        : norm != norm ? NAN : 0.0f;
  }
  __device__ __forceinline__ float of(float v) const { return v * before * factor; }
};

// X of the first step, times 2^11, as one or two float16 values a number.
template <typename T, bool UPDATE>
__global__ __launch_bounds__(256) void or_begin(Orthogonal x) {
  __shared__ double some[4];
  const int64_t pair = blockIdx.x / x.blocks;
  const uint32_t part = static_cast<uint32_t>(blockIdx.x - pair * x.blocks);
  const int tid = threadIdx.x;
  double s = tid < x.blocks ? x.norms[pair * x.blocks + tid] : 0.0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (tid % kWave == 0) some[tid / kWave] = s;
  __syncthreads();
  s = some[0] + some[1] + some[2] + some[3];
  const double norm = sqrt(s) + static_cast<double>(x.eps);
  const Inverse inverse(norm);
  const uint32_t each = static_cast<uint32_t>(x.cols8) / 8, n = each * x.rows8;
  const int64_t other = x.batch * (int64_t{8} * n);
  for (uint32_t i = part * 256 + tid; i < n; i += x.blocks * 256) {
    const uint32_t r = i / each;
    const int32_t c = static_cast<int32_t>(i - r * each) * 8;
    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (static_cast<int32_t>(r) < x.rows) input8<T, UPDATE>(x, pair * x.rows + r, c, v);
    Vec<f16_t, 8> hi, lo;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float w = settled(inverse.of(v[q]));
      hi.v[q] = from_float<f16_t>(w);
      lo.v[q] = from_float<f16_t>(w - to_float(hi.v[q]));
    }
    f16_t* const to = x.now[0] + (pair * n + i) * 8;
    *reinterpret_cast<Vec<f16_t, 8>*>(to) = hi;
    if (x.values > 1) *reinterpret_cast<Vec<f16_t, 8>*>(to + other) = lo;
  }
}

// Tiles of A, of B and of X, as one or two float16 values a number, by way of LDS to whole lines of
// memory (a lane's own results would go out in pieces of 8 bytes, and those of the transposed half
// of A and of B in pieces of 2).
enum Made { kGram, kPoly, kNext };
template <Made MADE>
struct Keep {
  f16_t* to;
  const f16_t* gram;
  int64_t other;  // elements from a number's first value to its second
  int32_t rows, cols, values;
  float a, b, c;

  template <class TILE, int MT, int NT>
  __device__ __forceinline__ void tile(f32x4 (&acc)[MT][NT], const Place& at, int mw, int nw,
                                       int lane, char* smem) const {
    constexpr int BM = 16 * MT, BN = 16 * NT;  // of a wave
    const int li = lane & 15, lg = (lane >> 4) * 4;
    const int32_t m0 = at.m0 + mw, n0 = at.n0 + nw;
    const int64_t first = at.pair * (static_cast<int64_t>(rows) * cols);
    char* const room = smem + threadIdx.x / kWave * (TILE::kLds / 4);
    static_assert(Turn<f16_t, BN>::kBytes <= TILE::kLds / 4 &&
                  Turn<f16_t, BM>::kBytes <= TILE::kLds / 4);
    if (m0 >= rows || n0 >= cols) return;
    // a wave's part is above the diagonal, or below it and left to its mirror image, or on it
    const bool above = MADE == kNext || n0 >= m0 + BM - 1;
    if (MADE != kNext && n0 + BN <= m0) return;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int32_t m = m0 + 16 * i + li, n = n0 + 16 * j + lg;
        if constexpr (MADE == kPoly) {
          Vec<f16_t, 4> hi{}, lo{};
          const f16_t* const p = gram + first + static_cast<int64_t>(m) * cols + n;
          if (m < rows && n < cols) {
            hi = *reinterpret_cast<const Vec<f16_t, 4>*>(p);
            if (values > 1) lo = *reinterpret_cast<const Vec<f16_t, 4>*>(p + other);
          }
#pragma unroll
          for (int q = 0; q < 4; ++q)
            acc[i][j][q] = c * (acc[i][j][q] * (1.0f / kScale)) +
                           (b * (to_float(hi.v[q]) + to_float(lo.v[q])) +
                            (m == n + q ? a * kScale : 0.0f));
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[i][j][q] *= 1.0f / kScale;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[i][j][q] = settled(acc[i][j][q]);
      }
    for (int part = 0; part < values; ++part) {
      f16_t* const out = to + first + (part ? other : 0);
      if (above) {
        const Turn<f16_t, BN> turn{room};
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            turn.put(li, 16 * j + lg, v);
          }
          wave_fence();
          const int32_t m = m0 + 16 * i;
          turn.out(out + static_cast<int64_t>(m) * cols + n0, cols, rows - m, cols - n0, lane);
          wave_fence();
        }
        if constexpr (MADE != kNext) {
          // rows n of the transposed tile: columns m, 16 rows at a time
          using Mirror = Turn<f16_t, BM>;
          const Mirror turned{room};
#pragma unroll
          for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
              for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f16_t*>(room + (lg + q) * Mirror::kRow + (16 * i + li) * 2) =
                    from_float<f16_t>(acc[i][j][q]);
            wave_fence();
            const int32_t n = n0 + 16 * j;
            turned.out(out + static_cast<int64_t>(n) * cols + m0, cols, rows - n, cols - m0, lane);
            wave_fence();
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int32_t m = m0 + 16 * i + li, n = n0 + 16 * j + lg + q;
              if (m >= rows || n >= cols || n < m) continue;
              const f16_t v = from_float<f16_t>(acc[i][j][q]);
              out[static_cast<int64_t>(m) * cols + n] = v;
              out[static_cast<int64_t>(n) * cols + m] = v;
            }
      }
      // what the first value leaves
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            acc[i][j][q] = settled(acc[i][j][q] - to_float(from_float<f16_t>(acc[i][j][q])));
    }
  }
};

// Tiles of the last X: the result, or the weights' update.
template <typename T, bool UPDATE>
struct Finish {
  const T* weights;
  T* out;
  int32_t rows, cols;
  float rate, keep;

  template <class TILE, int MT, int NT>
  __device__ __forceinline__ void tile(f32x4 (&acc)[MT][NT], const Place& at, int mw, int nw,
                                       int lane, char*) const {
    const int32_t n = at.n0 + nw + (lane >> 4) * 4;
    const int64_t first = at.pair * (static_cast<int64_t>(rows) * cols);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int32_t m = at.m0 + mw + 16 * i + (lane & 15);
      if (m >= rows) break;
      const int64_t row = first + static_cast<int64_t>(m) * cols;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int32_t n1 = n + 16 * j;
        if (n1 >= cols) break;
        float v[4];
        if constexpr (UPDATE) load4(weights + row, n1, cols, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float o = acc[i][j][q] * (1.0f / (kScale * kScale));
          v[q] = UPDATE ? keep * v[q] - rate * o : o;
        }
        store4(out + row, n1, cols, v);
      }
    }
  }
};

// A small matrix by one workgroup, all steps in LDS: X, A and B as above, with S (the short side)
// rows and L columns.  A wave takes tiles of 16 x 16 of A and of B, and columns of 16 of X, which
// it alone reads and writes.  Bound by latency: 15 products that wait for each other, with a barrier
// after each; one matrix of 64 x 192 in two values 34 us, 88 as launches.
constexpr int kSmallThreads = 1024;
constexpr int kSmallLds = 152 * 1024;
constexpr int small_side(int values) { return values == 1 ? 128 : 96; }  // of S at most
struct SmallSizes {
  int32_t s, l;        // sides
  int32_t rows_x;      // S up to a multiple of 32
  int32_t x, a;        // elements of a row of X, and of A and B: up to a multiple of 32, and 8
  int32_t many_x, many_a;  // elements of X, of A
  __host__ __device__ SmallSizes(int32_t rows, int32_t cols) {
    s = rows < cols ? rows : cols;
    l = rows < cols ? cols : rows;
    rows_x = (s + 31) / 32 * 32;
    x = (l + 31) / 32 * 32 + 8;
    a = rows_x + 8;
    many_x = rows_x * x;
    many_a = rows_x * a;
  }
  __host__ __device__ int64_t bytes(int32_t values) const {
    return int64_t{2} * values * (many_x + 2 * many_a);
  }
};

template <typename T, bool UPDATE, int VALUES>
__global__ __launch_bounds__(kSmallThreads) void or_small(Orthogonal x) {
  constexpr int kWaves = kSmallThreads / kWave;
  __shared__ __attribute__((aligned(16))) char smem[kSmallLds];
  __shared__ double some[kWaves];
  const SmallSizes z(x.rows, x.cols);
  const bool wide = x.rows <= x.cols;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = lane >> 4, li = lane & 15, lg = g * 4;
  f16_t* const xs = reinterpret_cast<f16_t*>(smem);
  f16_t* const as = xs + VALUES * z.many_x;
  f16_t* const bs = as + VALUES * z.many_a;
  const int64_t pair = blockIdx.x;
  const int32_t n = x.rows * x.cols;
  const int64_t first = pair * n;

  for (int32_t i = tid; i < VALUES * (z.many_x + 2 * z.many_a) / 8; i += kSmallThreads)
    reinterpret_cast<u32x4*>(smem)[i] = u32x4{0, 0, 0, 0};
  // four elements at a time, whatever rows they belong to
  const T* const from = static_cast<const T*>(x.x) + first;
  double sum = 0.0;
#pragma unroll 2
  for (int32_t i = 4 * tid; i < n; i += 4 * kSmallThreads) {
    float v[4];
    load4(from, i, n, v);
    if constexpr (UPDATE) {
      float m[4];
      load4(x.momentum + first, i, n, m);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        m[q] = x.beta * m[q] + v[q];
        v[q] = x.nesterov ? v[q] + x.beta * m[q] : m[q];
      }
      store4(x.new_momentum + first, i, n, m);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += static_cast<double>(v[q]) * v[q];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) some[wave] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += some[w];
  const double norm = sqrt(sum) + static_cast<double>(x.eps);
  const Inverse inverse(norm);
  // one or two float16 values of v at element i of X, A or B
  const auto keep = [&](f16_t* to, int32_t other, int32_t i, float v) {
    v = settled(v);
    const f16_t hi = from_float<f16_t>(v);
    to[i] = hi;
    if constexpr (VALUES > 1) to[i + other] = from_float<f16_t>(v - to_float(hi));
  };
#pragma unroll 2
  for (int32_t i = 4 * tid; i < n; i += 4 * kSmallThreads) {
    float v[4];
    load4(from, i, n, v);
    if constexpr (UPDATE) {
      float m[4];
      load4(x.new_momentum + first, i, n, m);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = x.nesterov ? v[q] + x.beta * m[q] : m[q];
    }
    int32_t r = i / x.cols, c = i - r * x.cols;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (i + q < n) keep(xs, z.many_x, wide ? r * z.x + c : c * z.x + r, inverse.of(v[q]));
      if (++c == x.cols) {
        c = 0;
        ++r;
      }
    }
  }
  __syncthreads();

  // products of 16 rows of p (from row r0) and of q (from row r1), k contiguous in both
  const auto rows = [&](const f16_t* p, const f16_t* q, int32_t r0, int32_t r1, int32_t ld,
                        int32_t other, int32_t k_end) {
    // (the small products in sums of their own, which do not wait for each other)
    f32x4 acc[VALUES > 1 ? 3 : 1] = {};
    const f16_t* const a = p + (r0 + li) * ld + 8 * g;
    const f16_t* const b = q + (r1 + li) * ld + 8 * g;
#pragma unroll 2
    for (int32_t k = 0; k < k_end; k += 32) {
      Frag fa[VALUES], fb[VALUES];
#pragma unroll
      for (int u = 0; u < VALUES; ++u) {
        fa[u].u = *reinterpret_cast<const u32x4*>(a + u * other + k);
        fb[u].u = *reinterpret_cast<const u32x4*>(b + u * other + k);
      }
      acc[0] = multiply<f16_t>(fb[0], fa[0], acc[0], 0);
      if constexpr (VALUES > 1) {
        acc[1] = multiply<f16_t>(fb[1], fa[0], acc[1], 0);
        acc[2] = multiply<f16_t>(fb[0], fa[1], acc[2], 0);
      }
    }
    if constexpr (VALUES > 1) return acc[0] + (acc[1] + acc[2]);
    else return acc[0];
  };
  const int32_t tiles = (z.s + 15) / 16, columns = (z.l + 15) / 16;
  const auto symmetric = [&](const auto& make, f16_t* to) {
    for (int32_t t = wave; t < tiles * (tiles + 1) / 2; t += kWaves) {
      int32_t c = 0;
      while ((c + 1) * (c + 2) / 2 <= t) ++c;
      const int32_t m0 = 16 * (t - c * (c + 1) / 2), n0 = 16 * c;
      const f32x4 v = make(m0, n0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int32_t m = m0 + li, nn = n0 + lg + q;
        if (nn < m) continue;
        keep(to, z.many_a, m * z.a + nn, v[q]);
        keep(to, z.many_a, nn * z.a + m, v[q]);
      }
    }
    __syncthreads();
  };
  for (int32_t step = 0; step < x.steps; ++step) {
    symmetric([&](int32_t m0, int32_t n0) {
      return rows(xs, xs, m0, n0, z.x, z.many_x, z.x - 8) * (1.0f / kScale);
    }, as);
    symmetric([&](int32_t m0, int32_t n0) {
      f32x4 v = rows(as, as, m0, n0, z.a, z.many_a, z.rows_x) * (1.0f / kScale);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int32_t i = (m0 + li) * z.a + n0 + lg + q;
        float a = to_float(as[i]);
        if constexpr (VALUES > 1) a += to_float(as[i + z.many_a]);
        v[q] = x.c * v[q] + (x.b * a + (m0 + li == n0 + lg + q ? x.a * kScale : 0.0f));
      }
      return v;
    }, bs);
    const bool last = step + 1 == x.steps;
    for (int32_t c = wave; c < columns; c += kWaves) {
      constexpr int kMost = small_side(VALUES) / 16;
      f32x4 acc[kMost] = {}, small[kMost] = {};
      for (int32_t k = 0; k < z.rows_x; k += 32) {
        // rows of k, 16 columns wide, transposed on the way
        Frag fx[VALUES];
#pragma unroll
        for (int u = 0; u < VALUES; ++u)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            fx[u].s[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(
                    xs + u * z.many_x + (k + 8 * g + 4 * j + (li >> 2)) * z.x + 16 * c +
                    (li & 3) * 4));
#pragma unroll
        for (int i = 0; i < kMost; ++i) {
          if (i >= tiles) break;
          Frag fb[VALUES];
#pragma unroll
          for (int u = 0; u < VALUES; ++u)
            fb[u].u = *reinterpret_cast<const u32x4*>(bs + u * z.many_a + (16 * i + li) * z.a + k +
                                                      8 * g);
          acc[i] = multiply<f16_t>(fx[0], fb[0], acc[i], 0);
          if constexpr (VALUES > 1) {
            small[i] = multiply<f16_t>(fx[1], fb[0], small[i], 0);
            small[i] = multiply<f16_t>(fx[0], fb[1], small[i], 0);
          }
        }
      }
      if constexpr (VALUES > 1)
#pragma unroll
        for (int i = 0; i < kMost; ++i) acc[i] += small[i];
      wave_fence();
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        if (i >= tiles) break;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int32_t m = 16 * i + li, l = 16 * c + lg + q;
          if (m >= z.s || l >= z.l) continue;
          if (last) {
            const int64_t at = first + (wide ? m * x.cols + l : l * x.cols + m);
            const float o = acc[i][q] * (1.0f / (kScale * kScale));
            T* const out = static_cast<T*>(x.out);
            if constexpr (UPDATE)
              out[at] = from_float<T>(x.keep * to_float(static_cast<const T*>(x.weights)[at]) -
                                      x.rate * o);
            else
              out[at] = from_float<T>(o);
          } else {
            keep(xs, z.many_x, m * z.x + l, acc[i][q] * (1.0f / kScale));
          }
        }
      }
    }
    __syncthreads();
  }
}

bool small_matrix(const Orthogonal& x) {
  const SmallSizes z(x.rows, x.cols);
  return z.s <= small_side(x.values) && z.bytes(x.values) <= kSmallLds;
}

template <typename T, bool UPDATE>
hipError_t launch(const Orthogonal& x, hipStream_t st) {
  if (small_matrix(x)) {
    const uint32_t grid = static_cast<uint32_t>(x.batch);
    if (x.values == 2) or_small<T, UPDATE, 2><<<grid, kSmallThreads, 0, st>>>(x);
    else or_small<T, UPDATE, 1><<<grid, kSmallThreads, 0, st>>>(x);
    return hipGetLastError();
  }
  const uint32_t blocks = static_cast<uint32_t>(x.batch * x.blocks);
  or_norm<T, UPDATE><<<blocks, kNormThreads, 0, st>>>(x);
  or_begin<T, UPDATE><<<blocks, 256, 0, st>>>(x);
  const bool wide = x.rows <= x.cols;
  const int32_t side = wide ? x.rows8 : x.cols8;
  const int64_t all = static_cast<int64_t>(x.rows8) * x.cols8;
  const int64_t square = static_cast<int64_t>(side) * side;
  const auto operand = [&](const f16_t* p, bool first, int32_t cols, int64_t each, int32_t rows) {
    // terms: hi lo, lo hi, hi hi (the small ones first: fewer roundings of a large sum)
    const int64_t lo = x.values == 2 ? 2 * x.batch * each : 0;
    return Operand{reinterpret_cast<const char*>(p) + (first ? 0 : lo),
                   {first ? lo : -lo, first ? -lo : 0}, int64_t{2} * cols, 2 * each, rows};
  };
  Product p{};
  p.terms = x.values == 2 ? 3 : 1;
  p.batch = static_cast<int32_t>(x.batch);
  p.splits = 1;
  p.eighths = 1;
  for (int32_t s = 0; s < x.steps; ++s) {
    const f16_t* const now = x.now[s & 1];
    p.symmetric = 1;
    p.a = operand(now, true, x.cols8, all, side);
    p.b = operand(now, false, x.cols8, all, side);
    p.k = p.part = wide ? x.cols8 : x.rows8;
    const Keep<kGram> gram{x.gram, nullptr, x.batch * square, side, side, x.values, x.a, x.b, x.c};
    if (wide) run_product<f16_t, false, false>(p, gram, st);
    else run_product<f16_t, true, true>(p, gram, st);
    p.a = operand(x.gram, true, side, square, side);
    p.b = operand(x.gram, false, side, square, side);
    p.k = p.part = side;
    run_product<f16_t, false, false>(p, Keep<kPoly>{x.poly, x.gram, x.batch * square, side, side,
                                                    x.values, x.a, x.b, x.c}, st);
    p.symmetric = 0;
    if (wide) {
      p.a = operand(x.poly, true, side, square, side);
      p.b = operand(now, false, x.cols8, all, x.cols8);
    } else {
      p.a = operand(now, true, x.cols8, all, x.rows8);
      p.b = operand(x.poly, false, side, square, side);
    }
    const auto last = [&](const auto& epi) {
      run_product<f16_t, false, true>(p, epi, st);  // (B = B^T)
    };
    if (s + 1 < x.steps)
      last(Keep<kNext>{x.now[~s & 1], nullptr, x.batch * all, x.rows8, x.cols8, x.values, x.a,
                       x.b, x.c});
    else
      last(Finish<T, UPDATE>{static_cast<const T*>(x.weights), static_cast<T*>(x.out), x.rows,
                             x.cols, x.rate, x.keep});
  }
  return hipGetLastError();
}

// Whether every value on the way fits float16 times 2^11.
bool coefficients_ok(const gsn_orthogonal_params& p) {
  if (!std::isfinite(p.a) || !std::isfinite(p.b) || !std::isfinite(p.c)) return false;
  double most = 1.0;
  for (int32_t s = 0; s < p.steps; ++s) {
    double next = 0.0;
    for (int i = 0; i <= 512; ++i) {
      const double v = most * i / 512, q = p.a + (p.b + p.c * v * v) * v * v;
      if (!(std::fabs(q) <= 28.0)) return false;
      next = std::max(next, std::fabs(v * q));
    }
    if (!(next <= 5.0)) return false;
    most = next * 1.01;
  }
  return true;
}

bool params_ok(const gsn_orthogonal_params* p) {
  return p && p->dtype >= GSN_F32 && p->dtype <= GSN_F16 && p->rows >= 1 && p->cols >= 1 &&
         p->rows <= (1 << 15) && p->cols <= (1 << 15) && p->batch >= 0 && p->batch <= (1 << 20) &&
         p->steps >= 1 && p->steps <= 64 && p->eps >= 0.0f && std::isfinite(p->eps) &&
         coefficients_ok(*p);
}

Orthogonal orthogonal_of(const gsn_orthogonal_params& p, bool update) {
  Orthogonal x{};
  x.batch = p.batch;
  x.rows = p.rows;
  x.cols = p.cols;
  x.rows8 = (p.rows + 7) / 8 * 8;
  x.cols8 = (p.cols + 7) / 8 * 8;
  const int64_t n = int64_t{p.rows} * p.cols;
  x.blocks = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(256, n / 8192)));
  x.steps = p.steps;
  // An update is a small part of the weights: in 2-byte weights its error of 3e-3 at most is below
  // their own rounding.
  x.values = update && p.dtype != GSN_F32 ? 1 : 2;
  x.a = p.a;
  x.b = p.b;
  x.c = p.c;
  x.eps = p.eps;
  return x;
}

size_t carve(void* base, Orthogonal* x) {
  size_t used = 0;
  const auto take = [&](size_t n) {
    char* const p = base ? static_cast<char*>(base) + used : nullptr;
    used += (n + 255) / 256 * 256;
    return static_cast<void*>(p);
  };
  const size_t batch = static_cast<size_t>(x->batch);
  const size_t all = batch * x->rows8 * x->cols8 * 2 * x->values;
  const size_t side = std::min(x->rows8, x->cols8), square = batch * side * side * 2 * x->values;
  x->norms = static_cast<double*>(take(batch * x->blocks * 8));
  x->now[0] = static_cast<f16_t*>(take(all));
  x->now[1] = static_cast<f16_t*>(take(all));
  x->gram = static_cast<f16_t*>(take(square));
  x->poly = static_cast<f16_t*>(take(square));
  return used;
}

// Whether the grids stay below 2^32 threads of 256.
bool grids_ok(const Orthogonal& x) {
  const int64_t tiles = int64_t{tiles_of(x.rows8, kMiddleRows)} * tiles_of(x.cols8, kMiddleRows);
  return x.batch * std::max<int64_t>(tiles, x.blocks) < (1 << 23);
}

int call(const gsn_orthogonal_params* p, bool update, Orthogonal x, void* workspace,
         size_t workspace_bytes, hipStream_t st) {
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return GSN_E_INVAL;
  if (workspace_bytes < gsn_orthogonal_workspace_bytes(p, update)) return GSN_E_CAPACITY;
  if (!grids_ok(x)) return GSN_E_CAPACITY;
  carve(workspace, &x);
  hipError_t e;
  if (update)
    e = p->dtype == GSN_F32    ? launch<float, true>(x, st)
        : p->dtype == GSN_BF16 ? launch<bf16_t, true>(x, st)
                               : launch<f16_t, true>(x, st);
  else
    e = p->dtype == GSN_F32    ? launch<float, false>(x, st)
        : p->dtype == GSN_BF16 ? launch<bf16_t, false>(x, st)
                               : launch<f16_t, false>(x, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

}  // namespace
}  // namespace gsn

extern "C" {

size_t gsn_orthogonal_workspace_bytes(const gsn_orthogonal_params* p, int32_t update) {
  if (!gsn::params_ok(p)) return 0;
  gsn::Orthogonal x = gsn::orthogonal_of(*p, update != 0);
  return gsn::carve(nullptr, &x) + 256;
}

int gsn_orthogonalise(const gsn_orthogonal_params* p, const void* x, void* out, void* workspace,
                      size_t workspace_bytes, void* stream) {
  if (!gsn::params_ok(p)) return GSN_E_INVAL;
  if (p->batch == 0) return GSN_OK;
  if (!x || !out) return GSN_E_INVAL;
  gsn::Orthogonal a = gsn::orthogonal_of(*p, false);
  a.x = x;
  a.out = out;
  return gsn::call(p, false, a, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

int gsn_orthogonal_step(const gsn_orthogonal_params* p, const void* weights, const void* gradient,
                        const float* momentum, float rate, float beta, float decay,
                        int32_t nesterov, void* new_weights, float* new_momentum, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (!gsn::params_ok(p) || !std::isfinite(rate) || !std::isfinite(beta) || !std::isfinite(decay))
    return GSN_E_INVAL;
  if (p->batch == 0) return GSN_OK;
  if (!weights || !gradient || !momentum || !new_weights || !new_momentum) return GSN_E_INVAL;
  // (the new momentum is written while both are still read, the new weights after it is)
  if (new_momentum == gradient || new_momentum == weights || new_weights == new_momentum ||
      new_weights == momentum)
    return GSN_E_INVAL;
  gsn::Orthogonal a = gsn::orthogonal_of(*p, true);
  a.x = gradient;
  a.momentum = momentum;
  a.new_momentum = new_momentum;
  a.weights = weights;
  a.rate = rate;
  a.beta = beta;
  a.keep = 1.0f - decay;
  a.nesterov = nesterov;
  a.out = new_weights;
  return gsn::call(p, true, a, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

}  // extern "C"
