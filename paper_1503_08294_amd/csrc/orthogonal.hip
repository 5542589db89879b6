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
// Gaussian entries and of a few strong directions, 256 to 1,024 a side; binary32 throughout 2e-6 to
// 6e-6): one value 2e-4 to 3e-3, two 5e-7 to 7e-7; bfloat16 in their place 1e-2 to 8e-2.
// 2^11: entries are at most 5 (28 in B), a float16 holds 65,504; what is lost below its smallest
// step is 2^-36 of a largest singular value of 1.
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

// What is orthogonalised, at element i of all matrices.  The momentum is new_momentum by then.
template <typename T, bool UPDATE>
__device__ __forceinline__ float input(const Orthogonal& x, int64_t i) {
  const float g = to_float(static_cast<const T*>(x.x)[i]);
  if constexpr (!UPDATE) return g;
  const float m = x.new_momentum[i];
  return x.nesterov ? g + x.beta * m : m;
}

// Sums of squares in 64 bits (squares of binary32 leave its range), a part of a matrix a workgroup;
// and the momentum.  Bound by memory.
constexpr int kNormThreads = 256;
template <typename T, bool UPDATE>
__global__ __launch_bounds__(kNormThreads) void or_norm(Orthogonal x) {
  __shared__ double some[kNormThreads / kWave];
  const int64_t pair = blockIdx.x / x.blocks;
  const int32_t part = static_cast<int32_t>(blockIdx.x - pair * x.blocks);
  const int64_t n = static_cast<int64_t>(x.rows) * x.cols;
  double s = 0.0;
  for (int64_t i = static_cast<int64_t>(part) * kNormThreads + threadIdx.x; i < n;
       i += static_cast<int64_t>(x.blocks) * kNormThreads) {
    const int64_t at = pair * n + i;
    if constexpr (UPDATE)
      x.new_momentum[at] =
          x.beta * x.momentum[at] + to_float(static_cast<const T*>(x.x)[at]);
    const double v = input<T, UPDATE>(x, at);
    s += v * v;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (threadIdx.x % kWave == 0) some[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int w = 1; w < kNormThreads / kWave; ++w) s += some[w];
  x.norms[blockIdx.x] = s;
}

// v (times 2^11) as one or two float16 values at element i.
__device__ __forceinline__ void keep2(f16_t* to, int64_t other, int32_t values, int64_t i,
                                      float v) {
  const f16_t hi = from_float<f16_t>(v);
  to[i] = hi;
  if (values > 1) to[other + i] = from_float<f16_t>(v - to_float(hi));
}

// X of the first step.
template <typename T, bool UPDATE>
__global__ __launch_bounds__(256) void or_begin(Orthogonal x) {
  __shared__ float factor;
  const int64_t pair = blockIdx.x / x.blocks;
  const int32_t part = static_cast<int32_t>(blockIdx.x - pair * x.blocks);
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int32_t i = 0; i < x.blocks; ++i) s += x.norms[pair * x.blocks + i];
    const double norm = sqrt(s) + static_cast<double>(x.eps);
    // (a matrix of zeros without an eps; infinities become NaN below)
    factor = norm > 0.0 ? static_cast<float>(kScale / norm) : s != s ? NAN : 0.0f;
  }
  __syncthreads();
  const int64_t n = static_cast<int64_t>(x.rows) * x.cols;
  const int64_t all = static_cast<int64_t>(x.rows8) * x.cols8;
  for (int64_t i = static_cast<int64_t>(part) * 256 + threadIdx.x; i < all;
       i += static_cast<int64_t>(x.blocks) * 256) {
    const int32_t r = static_cast<int32_t>(i / x.cols8);
    const int32_t c = static_cast<int32_t>(i - static_cast<int64_t>(r) * x.cols8);
    float v = 0.0f;
    if (r < x.rows && c < x.cols)
      v = input<T, UPDATE>(x, pair * n + static_cast<int64_t>(r) * x.cols + c) * factor;
    keep2(x.now[0], x.batch * all, x.values, pair * all + i, v);
  }
}

// Four values of a row as one or two float16 values each.
__device__ __forceinline__ void keep4(f16_t* to, int64_t other, int32_t values, int64_t i,
                                      const float* v) {
  Vec<f16_t, 4> hi, lo;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    hi.v[q] = from_float<f16_t>(v[q]);
    lo.v[q] = from_float<f16_t>(v[q] - to_float(hi.v[q]));
  }
  *reinterpret_cast<Vec<f16_t, 4>*>(to + i) = hi;
  if (values > 1) *reinterpret_cast<Vec<f16_t, 4>*>(to + other + i) = lo;
}

// Tiles of A, of B and of X.
enum Made { kGram, kPoly, kNext };
template <Made MADE>
struct Keep {
  f16_t* to;
  const f16_t* gram;
  int64_t other;  // elements from a number's first value to its second
  int32_t rows, cols, values;
  float a, b, c;

  template <int SIDE, int WN, int MT, int NT>
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
        if constexpr (MADE == kPoly) {
          const Vec<f16_t, 4> hi = *reinterpret_cast<const Vec<f16_t, 4>*>(gram + row + n1);
          Vec<f16_t, 4> lo{};
          if (values > 1) lo = *reinterpret_cast<const Vec<f16_t, 4>*>(gram + other + row + n1);
#pragma unroll
          for (int q = 0; q < 4; ++q)
            v[q] = c * (acc[i][j][q] * (1.0f / kScale)) +
                   (b * (to_float(hi.v[q]) + to_float(lo.v[q])) +
                    (m == n1 + q ? a * kScale : 0.0f));
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = acc[i][j][q] * (1.0f / kScale);
        }
        keep4(to, other, values, row + n1, v);
        if (MADE != kNext && at.n0 > at.m0)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            keep2(to, other, values, first + static_cast<int64_t>(n1 + q) * cols + m, v[q]);
      }
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

  template <int SIDE, int WN, int MT, int NT>
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

template <bool TRA, bool TRB, class EPI>
void product(Product p, const EPI& epi, hipStream_t st) {
  p.splits = 1;
  p.part = p.k;
  const int64_t m = tiles_of(p.a.rows, kMiddleRows), n = tiles_of(p.b.rows, kMiddleRows);
  // (tiles of 128 from one a CU on)
  if ((p.symmetric ? m * (m + 1) / 2 : m * n) * p.batch >= 256)
    run_product<f16_t, TRA, TRB, kMiddleRows>(p, epi, st);
  else
    run_product<f16_t, TRA, TRB, kSmallRows>(p, epi, st);
}

template <typename T, bool UPDATE>
hipError_t launch(const Orthogonal& x, hipStream_t st) {
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
  for (int32_t s = 0; s < x.steps; ++s) {
    const f16_t* const now = x.now[s & 1];
    p.symmetric = 1;
    p.a = operand(now, true, x.cols8, all, side);
    p.b = operand(now, false, x.cols8, all, side);
    p.k = wide ? x.cols8 : x.rows8;
    const Keep<kGram> gram{x.gram, nullptr, x.batch * square, side, side, x.values, x.a, x.b, x.c};
    if (wide) product<false, false>(p, gram, st);
    else product<true, true>(p, gram, st);
    p.a = operand(x.gram, true, side, square, side);
    p.b = operand(x.gram, false, side, square, side);
    p.k = side;
    product<false, false>(p, Keep<kPoly>{x.poly, x.gram, x.batch * square, side, side, x.values,
                                         x.a, x.b, x.c}, st);
    p.symmetric = 0;
    if (wide) {
      p.a = operand(x.poly, true, side, square, side);
      p.b = operand(now, false, x.cols8, all, x.cols8);
    } else {
      p.a = operand(now, true, x.cols8, all, x.rows8);
      p.b = operand(x.poly, false, side, square, side);
    }
    const auto last = [&](const auto& epi) {
      if (wide) product<false, true>(p, epi, st);
      else product<false, false>(p, epi, st);
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
  x.blocks = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(256, n / 4096)));
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
