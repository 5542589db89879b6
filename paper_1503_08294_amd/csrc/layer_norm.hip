// Layer norm over the rows of a matrix, and its backward pass.
//
//   mean = sum x / D,  var = sum (x - mean)^2 / D,  r = 1 / sqrt(var + eps)
//   n = (x - mean) r,  y = n w + b
//   g = dy w,  dx = r (g - mean(g) - n mean(g n)),  dw = sum_rows dy n,  db = sum_rows dy
//
// A row stays in the registers of the lanes that read it, so x (and dy) is read once and the
// variance is that of the centred values (no difference of large sums).  All sums are binary32;
// results are rounded to their type once.
#include "mixture.h"

#pragma clang fp contract(fast)

namespace gsn {
namespace {

constexpr int kThreads = 256;

struct NormArgs {
  int64_t rows;
  int32_t dim;
  const void* x;
  int64_t x_stride;
  const void* w;
  const void* b;
  int p32;  // weight and bias are binary32 (else of x's type)
  float eps;
  void* y;
  int64_t y_stride;
  float* stats;  // [2][rows]: mean, r
};

template <typename T>
__device__ __forceinline__ float param(const void* p, int p32, int32_t i) {
  return p32 ? static_cast<const float*>(p)[i] : to_float(static_cast<const T*>(p)[i]);
}

// sum over the TPR lanes (a wave, or the workgroup) that hold a row
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum(v);
  if (TPR == kWave) return v;
  const int w = threadIdx.x / kWave;
  __syncthreads();
  if (threadIdx.x % kWave == 0) red[w] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void ln_forward(NormArgs a) {
  __shared__ float red[kThreads / kWave];
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / TPR) + threadIdx.x / TPR;
  if (TPR == kWave && row >= a.rows) return;
  const int lane = threadIdx.x % TPR;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  T* y = static_cast<T*>(a.y) + row * a.y_stride;
  float s = 0.0f;
  for (int32_t i = lane; i < a.dim; i += TPR) s += to_float(x[i]);
  const float mean = row_sum<TPR>(s, red) / a.dim;
  float q = 0.0f;
  for (int32_t i = lane; i < a.dim; i += TPR) {
    const float d = to_float(x[i]) - mean;
    q += d * d;
  }
  const float r = 1.0f / sqrtf(row_sum<TPR>(q, red) / a.dim + a.eps);
  if (lane == 0 && a.stats) {
    a.stats[row] = mean;
    a.stats[a.rows + row] = r;
  }
  for (int32_t i = lane; i < a.dim; i += TPR) {
    float v = (to_float(x[i]) - mean) * r;
    if (a.w) v *= param<T>(a.w, a.p32, i);
    if (a.b) v += param<T>(a.b, a.p32, i);
    y[i] = from_float<T>(v);
  }
}

struct NormBackArgs {
  int64_t rows;
  int32_t dim;
  const void* dy;
  int64_t dy_stride;
  const void* x;
  int64_t x_stride;
  const void* w;
  int p32;
  const float* stats;
  void* dx;
  int64_t dx_stride;
};

template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void ln_backward(NormBackArgs a) {
  __shared__ float red[kThreads / kWave];
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / TPR) + threadIdx.x / TPR;
  if (TPR == kWave && row >= a.rows) return;
  const int lane = threadIdx.x % TPR;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
  T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
  const float mean = a.stats[row], r = a.stats[a.rows + row];
  float sg = 0.0f, sgn = 0.0f;
  for (int32_t i = lane; i < a.dim; i += TPR) {
    const float n = (to_float(x[i]) - mean) * r;
    const float g = to_float(dy[i]) * (a.w ? param<T>(a.w, a.p32, i) : 1.0f);
    sg += g;
    sgn += g * n;
  }
  const float mg = row_sum<TPR>(sg, red) / a.dim;
  const float mgn = row_sum<TPR>(sgn, red) / a.dim;
  for (int32_t i = lane; i < a.dim; i += TPR) {
    const float n = (to_float(x[i]) - mean) * r;
    const float g = to_float(dy[i]) * (a.w ? param<T>(a.w, a.p32, i) : 1.0f);
    dx[i] = from_float<T>(r * (g - mg - n * mgn));
  }
}

// part[2][parts][dim]: sums of dy n and of dy over the rows of one part
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_columns(NormBackArgs a, int32_t parts,
                                                       float* __restrict__ part) {
  const int32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.dim) return;
  const int64_t per = (a.rows + parts - 1) / parts;
  const int64_t r0 = per * blockIdx.y, r1 = r0 + per < a.rows ? r0 + per : a.rows;
  float sw = 0.0f, sb = 0.0f;
  for (int64_t row = r0; row < r1; ++row) {
    const float d = to_float((static_cast<const T*>(a.dy) + row * a.dy_stride)[i]);
    const float v = to_float((static_cast<const T*>(a.x) + row * a.x_stride)[i]);
    sw += d * ((v - a.stats[row]) * a.stats[a.rows + row]);
    sb += d;
  }
  part[static_cast<int64_t>(blockIdx.y) * a.dim + i] = sw;
  part[static_cast<int64_t>(parts + blockIdx.y) * a.dim + i] = sb;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void ln_join(int32_t dim, int32_t parts, int p32,
                                                    const float* __restrict__ part, void* dw,
                                                    void* db) {
  const int32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= dim) return;
  void* out = blockIdx.y == 0 ? dw : db;
  if (!out) return;
  const float* p = part + static_cast<int64_t>(blockIdx.y) * parts * dim;
  float s = 0.0f;
  for (int32_t k = 0; k < parts; ++k) s += p[static_cast<int64_t>(k) * dim + i];
  if (p32) static_cast<float*>(out)[i] = s;
  else static_cast<T*>(out)[i] = from_float<T>(s);
}

int32_t norm_parts(int64_t rows) {
  const int64_t p = (rows + 31) / 32;
  return static_cast<int32_t>(p < 1 ? 1 : p > 512 ? 512 : p);
}

template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t st) {
  if (a.dim <= 1024)
    ln_forward<T, kWave><<<static_cast<uint32_t>((a.rows + 3) / 4), kThreads, 0, st>>>(a);
  else
    ln_forward<T, kThreads><<<static_cast<uint32_t>(a.rows), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const NormBackArgs& a, void* dw, void* db, float* part, hipStream_t st) {
  if (a.dx && a.rows > 0) {
    if (a.dim <= 1024)
      ln_backward<T, kWave><<<static_cast<uint32_t>((a.rows + 3) / 4), kThreads, 0, st>>>(a);
    else
      ln_backward<T, kThreads><<<static_cast<uint32_t>(a.rows), kThreads, 0, st>>>(a);
  }
  if (dw || db) {
    const int32_t parts = norm_parts(a.rows);
    const uint32_t nb = (a.dim + kThreads - 1) / kThreads;
    ln_columns<T><<<dim3(nb, parts), kThreads, 0, st>>>(a, parts, part);
    ln_join<T><<<dim3(nb, 2), kThreads, 0, st>>>(a.dim, parts, a.p32, part, dw, db);
  }
  return hipGetLastError();
}

bool types_ok(int32_t dtype, int32_t param_dtype) {
  return dtype >= GSN_F32 && dtype <= GSN_F16 &&
         (param_dtype == GSN_F32 || param_dtype == dtype);
}

// rows are a grid's x dimension (or a quarter of it)
constexpr int64_t kMostRows = INT32_MAX;

}  // namespace
}  // namespace gsn

extern "C" {

int gsn_layer_norm(int32_t dtype, int32_t param_dtype, int64_t rows, int32_t dim, const void* x,
                   int64_t x_stride, const void* weight, const void* bias, float eps, void* y,
                   int64_t y_stride, float* stats, void* stream) {
  if (!gsn::types_ok(dtype, param_dtype) || rows < 0 || rows > gsn::kMostRows || dim < 1 ||
      !(eps >= 0.0f))
    return GSN_E_INVAL;
  if (rows == 0) return GSN_OK;
  if (!x || !y || x_stride < dim || y_stride < dim) return GSN_E_INVAL;
  const gsn::NormArgs a{rows, dim, x, x_stride, weight, bias, param_dtype == GSN_F32, eps, y,
                        y_stride, stats};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = dtype == GSN_F32    ? gsn::forward<float>(a, st)
                       : dtype == GSN_BF16 ? gsn::forward<gsn::bf16_t>(a, st)
                                           : gsn::forward<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

size_t gsn_layer_norm_workspace_bytes(int64_t rows, int32_t dim) {
  if (rows < 0 || rows > gsn::kMostRows || dim < 1) return 0;
  return sizeof(float) * 2 * static_cast<size_t>(gsn::norm_parts(rows)) * dim;
}

int gsn_layer_norm_backward(int32_t dtype, int32_t param_dtype, int64_t rows, int32_t dim,
                            const void* dy, int64_t dy_stride, const void* x, int64_t x_stride,
                            const void* weight, const float* stats, void* dx, int64_t dx_stride,
                            void* dweight, void* dbias, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (!gsn::types_ok(dtype, param_dtype) || rows < 0 || rows > gsn::kMostRows || dim < 1)
    return GSN_E_INVAL;
  if (rows > 0 && (!dy || !x || !stats || dy_stride < dim || x_stride < dim ||
                   (dx && dx_stride < dim)))
    return GSN_E_INVAL;
  if (dweight || dbias) {
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return GSN_E_INVAL;
    if (workspace_bytes < gsn_layer_norm_workspace_bytes(rows, dim)) return GSN_E_CAPACITY;
  }
  const gsn::NormBackArgs a{rows, dim, dy, dy_stride, x, x_stride, weight,
                            param_dtype == GSN_F32, stats, dx, dx_stride};
  float* part = static_cast<float*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e =
      dtype == GSN_F32    ? gsn::backward<float>(a, dweight, dbias, part, st)
      : dtype == GSN_BF16 ? gsn::backward<gsn::bf16_t>(a, dweight, dbias, part, st)
                          : gsn::backward<gsn::f16_t>(a, dweight, dbias, part, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

}  // extern "C"
