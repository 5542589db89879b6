// Layer norm over the rows of a matrix, and its backward pass.
//
//   mean = sum x / D,  var = sum (x - mean)^2 / D,  r = 1 / sqrt(var + eps)
//   n = (x - mean) r,  y = n w + b
//   g = dy w,  dx = r (g - mean(g) - n mean(g n)),  dw = sum_rows dy n,  db = sum_rows dy
//
// A row stays in the registers of the lanes that read it, so x (and dy) is read once and the
// variance is that of the centred values (no difference of large sums).  All sums are binary32;
// results are rounded to their type once.
//
// Both passes are bound by memory (a large copy runs at 4.75 TB/s): 16,384 x 4,096 bfloat16
// forward in 63 us (4.2 TB/s); 16,384 x 2,048 backward in 38 us (5.3 TB/s: some of it is still in
// the last cache) and 7 us for the join of the columns' sums; 8,191 x 1,001 binary32, whose rows
// start at no multiple of 16 bytes, 15 us forward, 22 + 5 us backward.  Rows that a workgroup's
// registers do not hold are read again, an element at a time: forward beyond 8,192 elements,
// backward beyond 4,096 of binary32 and 8,192 of 2-byte types.  4,096 rows of binary32, us forward
// and backward: of 4,096 24 and 40, of 5,120 42 and 95, of 8,192 48 and 178, of 10,240 138 and 238;
// of bfloat16: of 8,192 41 and 49, of 16,384 192 and 278.
#include "mixture.h"

#include <algorithm>

#pragma clang fp contract(fast)

namespace gsn {
namespace {

constexpr int kThreads = 256;

template <typename T>
constexpr int kWidth = 16 / sizeof(T);
// 16 bytes of a row; rows start at any element, which these loads and stores take
template <typename T>
struct ChunkOf {
  typedef T type __attribute__((ext_vector_type(kWidth<T>), aligned(sizeof(T))));
};
template <typename T>
using Chunk = typename ChunkOf<T>::type;

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

// kWidth elements of a row at i, 0 past its end
template <typename T>
__device__ __forceinline__ void load_raw(const T* row, int32_t i, int32_t dim, Chunk<T>& v) {
  if (i + kWidth<T> <= dim) {
    v = *reinterpret_cast<const Chunk<T>*>(row + i);
  } else {
#pragma unroll
    for (int k = 0; k < kWidth<T>; ++k) v[k] = i + k < dim ? row[i + k] : from_float<T>(0.0f);
  }
}
// N elements as binary32, `none` past its end
template <typename T, int N>
__device__ __forceinline__ void load(const T* row, int32_t i, int32_t dim, float none,
                                     float (&v)[N]) {
  constexpr int kW = kWidth<T>;  // (binary32 parameters and sums of a 2-byte type: two accesses)
  static_assert(N % kW == 0);
  if (i + N <= dim) {
#pragma unroll
    for (int h = 0; h < N; h += kW) {
      const Chunk<T> c = *reinterpret_cast<const Chunk<T>*>(row + i + h);
#pragma unroll
      for (int k = 0; k < kW; ++k) v[h + k] = to_float(c[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = i + k < dim ? to_float(row[i + k]) : none;
  }
}
template <typename T, int N>
__device__ __forceinline__ void store(T* row, int32_t i, int32_t dim, const float (&v)[N]) {
  constexpr int kW = kWidth<T>;
  static_assert(N % kW == 0);
  if (i + N <= dim) {
#pragma unroll
    for (int h = 0; h < N; h += kW) {
      Chunk<T> c;
#pragma unroll
      for (int k = 0; k < kW; ++k) c[k] = from_float<T>(v[h + k]);
      *reinterpret_cast<Chunk<T>*>(row + i + h) = c;
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (i + k < dim) row[i + k] = from_float<T>(v[k]);
  }
}
template <typename T, int N>
__device__ __forceinline__ void load_param(const void* p, int p32, int32_t i, int32_t dim,
                                           float none, float (&v)[N]) {
  if (p == nullptr) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = none;
  } else if (p32) {
    load(static_cast<const float*>(p), i, dim, none, v);
  } else {
    load(static_cast<const T*>(p), i, dim, none, v);
  }
}
template <typename T>
__device__ __forceinline__ float param(const void* p, int p32, int32_t i) {
  return p32 ? static_cast<const float*>(p)[i] : to_float(static_cast<const T*>(p)[i]);
}

// Sums over the TPR lanes (a wave, or the workgroup) that hold a row, the same in every lane.
// red: 4 N floats, which no other sum uses until a barrier after this one.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
  if constexpr (TPR != kWave) {
    static_assert(TPR == 4 * kWave);
    if (threadIdx.x % kWave == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) red[4 * k + threadIdx.x / kWave] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k)
      v[k] = (red[4 * k] + red[4 * k + 1]) + (red[4 * k + 2] + red[4 * k + 3]);
  }
}

// Rows of at most TPR * NC * kWidth elements, TPR lanes and NC chunks a lane each.
template <typename T, int TPR, int NC>
__global__ __launch_bounds__(kThreads) void ln_forward(NormArgs a) {
  constexpr int kW = kWidth<T>, kRows = kThreads / TPR;
  __shared__ float red[2][kThreads / kWave];
  const int lane = threadIdx.x % TPR;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / TPR; row < a.rows;
       row += static_cast<int64_t>(gridDim.x) * kRows) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    Chunk<T> raw[NC];  // kept in their type: half the registers of a 2-byte type
#pragma unroll
    for (int c = 0; c < NC; ++c) load_raw(x, (c * TPR + lane) * kW, a.dim, raw[c]);
    float s[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int k = 0; k < kW; ++k) s[0] += to_float(raw[c][k]);
    row_sums<TPR>(s, red[0]);
    const float mean = s[0] / a.dim;  // (a quotient: a constant row has its value as the mean)
    float q[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int32_t left = a.dim - (c * TPR + lane) * kW;
#pragma unroll
      for (int k = 0; k < kW; ++k) {
        const float d = to_float(raw[c][k]) - mean;
        q[0] += k < left ? d * d : 0.0f;
      }
    }
    row_sums<TPR>(q, red[1]);
    const float r = 1.0f / sqrtf(q[0] / a.dim + a.eps);
    if (lane == 0 && a.stats) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = r;
    }
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int32_t i = (c * TPR + lane) * kW;
      float w[kW], b[kW], v[kW];
      load_param<T>(a.w, a.p32, i, a.dim, 1.0f, w);
      load_param<T>(a.b, a.p32, i, a.dim, 0.0f, b);
#pragma unroll
      for (int k = 0; k < kW; ++k) v[k] = (to_float(raw[c][k]) - mean) * r * w[k] + b[k];
      store(y, i, a.dim, v);
    }
  }
}

// Longer rows: read three times, by a workgroup each.
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_forward_long(NormArgs a) {
  __shared__ float red[2][kThreads / kWave];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    T* y = static_cast<T*>(a.y) + row * a.y_stride;
    float s[1] = {0.0f};
    for (int32_t i = threadIdx.x; i < a.dim; i += kThreads) s[0] += to_float(x[i]);
    row_sums<kThreads>(s, red[0]);
    const float mean = s[0] / a.dim;
    float q[1] = {0.0f};
    for (int32_t i = threadIdx.x; i < a.dim; i += kThreads) {
      const float d = to_float(x[i]) - mean;
      q[0] += d * d;
    }
    row_sums<kThreads>(q, red[1]);
    const float r = 1.0f / sqrtf(q[0] / a.dim + a.eps);
    if (threadIdx.x == 0 && a.stats) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = r;
    }
    for (int32_t i = threadIdx.x; i < a.dim; i += kThreads) {
      float v = (to_float(x[i]) - mean) * r;
      if (a.w) v *= param<T>(a.w, a.p32, i);
      if (a.b) v += param<T>(a.b, a.p32, i);
      y[i] = from_float<T>(v);
    }
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
  int32_t parts;
  float* part;  // [2][parts][dim]: sums of dy n and of dy over the rows of one part, or null
  uint32_t row_blocks;  // workgroups that take rows; those after them take 64 columns of all rows
  void* dw;             // (for the latter)
  void* db;
};

// Gradients of 64 columns' parameters from few rows: four lines of rows, added in order.
template <typename T>
__device__ __forceinline__ void few_columns(const NormBackArgs& a, uint32_t block) {
  constexpr int kLines = kThreads / kWave;
  __shared__ float sums[2][kLines][kWave];
  const int lane = threadIdx.x % kWave, line = threadIdx.x / kWave;
  const int32_t i = static_cast<int32_t>(block) * kWave + lane;
  float sw = 0.0f, sb = 0.0f;
  if (i < a.dim) {
#pragma unroll 8
    for (int64_t row = line; row < a.rows; row += kLines) {
      const float d = to_float((static_cast<const T*>(a.dy) + row * a.dy_stride)[i]);
      const float v = to_float((static_cast<const T*>(a.x) + row * a.x_stride)[i]);
      sw += d * ((v - a.stats[row]) * a.stats[a.rows + row]);
      sb += d;
    }
  }
  sums[0][line][lane] = sw;
  sums[1][line][lane] = sb;
  __syncthreads();
  void* const out = line == 0 ? a.dw : a.db;
  if (line > 1 || i >= a.dim || !out) return;
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < kLines; ++k) s += sums[line][k][lane];
  if (a.p32) static_cast<float*>(out)[i] = s;
  else static_cast<T*>(out)[i] = from_float<T>(s);
}

// dx and, over the rows that this workgroup takes, the sums of dy n and dy, which stay in the
// lanes' registers and go out once (waves that took rows of their own are joined through LDS).
template <typename T, int TPR, int NC>
__global__ __launch_bounds__(kThreads) void ln_backward(NormBackArgs a) {
  if (blockIdx.x >= a.row_blocks) return few_columns<T>(a, blockIdx.x - a.row_blocks);
  constexpr int kW = kWidth<T>, kRows = kThreads / TPR;
  __shared__ float red[2][2 * kThreads / kWave];
  const int lane = threadIdx.x % TPR;
  float w[NC][kW], sw[NC][kW], sb[NC][kW];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    load_param<T>(a.w, a.p32, (c * TPR + lane) * kW, a.dim, 1.0f, w[c]);
#pragma unroll
    for (int k = 0; k < kW; ++k) sw[c][k] = sb[c][k] = 0.0f;
  }
  int odd = 0;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / TPR; row < a.rows;
       row += static_cast<int64_t>(a.row_blocks) * kRows, odd ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
    Chunk<T> xr[NC], dr[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      load_raw(x, (c * TPR + lane) * kW, a.dim, xr[c]);
      load_raw(dy, (c * TPR + lane) * kW, a.dim, dr[c]);
    }
    const float mean = a.stats[row], r = a.stats[a.rows + row];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int k = 0; k < kW; ++k) {
        const float n = (to_float(xr[c][k]) - mean) * r, d = to_float(dr[c][k]);
        sw[c][k] += d * n;  // (past the row's end dy is 0)
        sb[c][k] += d;
        s[0] += d * w[c][k];
        s[1] += d * w[c][k] * n;
      }
    if (a.dx == nullptr) continue;
    row_sums<TPR>(s, red[odd]);
    const float mg = s[0] / a.dim, mgn = s[1] / a.dim;
    T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float v[kW];
#pragma unroll
      for (int k = 0; k < kW; ++k) {
        const float n = (to_float(xr[c][k]) - mean) * r;
        v[k] = r * (to_float(dr[c][k]) * w[c][k] - mg - n * mgn);
      }
      store(dx, (c * TPR + lane) * kW, a.dim, v);
    }
  }
  if (a.part == nullptr) return;
  float* pw = a.part + static_cast<int64_t>(blockIdx.x) * a.dim;
  float* pb = a.part + (static_cast<int64_t>(a.parts) + blockIdx.x) * a.dim;
  if constexpr (TPR == kThreads) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      store(pw, (c * TPR + lane) * kW, a.dim, sw[c]);
      store(pb, (c * TPR + lane) * kW, a.dim, sb[c]);
    }
  } else {
    __shared__ float sums[2][TPR * NC * kW];
    for (int v = 0; v < kRows; ++v) {
      if (threadIdx.x / TPR == v) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int k = 0; k < kW; ++k) {
            const int i = (c * TPR + lane) * kW + k;
            sums[0][i] = v == 0 ? sw[c][k] : sums[0][i] + sw[c][k];
            sums[1][i] = v == 0 ? sb[c][k] : sums[1][i] + sb[c][k];
          }
      }
      __syncthreads();
    }
    for (int32_t i = threadIdx.x; i < a.dim; i += kThreads) {
      pw[i] = sums[0][i];
      pb[i] = sums[1][i];
    }
  }
}

// Longer rows: dx by a workgroup a row, which reads x and dy twice.
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_backward_long(NormBackArgs a) {
  __shared__ float red[2][2 * kThreads / kWave];
  int odd = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, odd ^= 1) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
    T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
    const float mean = a.stats[row], r = a.stats[a.rows + row];
    float s[2] = {0.0f, 0.0f};
    for (int32_t i = threadIdx.x; i < a.dim; i += kThreads) {
      const float n = (to_float(x[i]) - mean) * r;
      const float g = to_float(dy[i]) * (a.w ? param<T>(a.w, a.p32, i) : 1.0f);
      s[0] += g;
      s[1] += g * n;
    }
    row_sums<kThreads>(s, red[odd]);
    const float mg = s[0] / a.dim, mgn = s[1] / a.dim;
    for (int32_t i = threadIdx.x; i < a.dim; i += kThreads) {
      const float n = (to_float(x[i]) - mean) * r;
      const float g = to_float(dy[i]) * (a.w ? param<T>(a.w, a.p32, i) : 1.0f);
      dx[i] = from_float<T>(r * (g - mg - n * mgn));
    }
  }
}

// The columns' sums of longer rows, a part of the rows each.
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_columns(NormBackArgs a) {
  const int32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.dim) return;
  const int64_t per = (a.rows + a.parts - 1) / a.parts;
  const int64_t r0 = per * blockIdx.y, r1 = r0 + per < a.rows ? r0 + per : a.rows;
  float sw = 0.0f, sb = 0.0f;
  for (int64_t row = r0; row < r1; ++row) {
    const float d = to_float((static_cast<const T*>(a.dy) + row * a.dy_stride)[i]);
    const float v = to_float((static_cast<const T*>(a.x) + row * a.x_stride)[i]);
    sw += d * ((v - a.stats[row]) * a.stats[a.rows + row]);
    sb += d;
  }
  a.part[static_cast<int64_t>(blockIdx.y) * a.dim + i] = sw;
  a.part[(static_cast<int64_t>(a.parts) + blockIdx.y) * a.dim + i] = sb;
}

// The parts' sums: 16 columns a workgroup, 16 parts at a time, then the 16 partial sums in order.
constexpr int kJoinColumns = 16;
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_join(int32_t dim, int32_t parts, int p32,
                                                    const float* __restrict__ part, void* dw,
                                                    void* db) {
  __shared__ float sums[kThreads / kJoinColumns][kJoinColumns];
  void* out = blockIdx.y == 0 ? dw : db;
  if (!out) return;
  const int col = threadIdx.x % kJoinColumns, line = threadIdx.x / kJoinColumns;
  const int32_t i = blockIdx.x * kJoinColumns + col;
  float s = 0.0f;
  if (i < dim) {
    const float* p = part + static_cast<int64_t>(blockIdx.y) * parts * dim + i;
#pragma unroll 8
    for (int32_t k = line; k < parts; k += kThreads / kJoinColumns)
      s += p[static_cast<int64_t>(k) * dim];
  }
  sums[line][col] = s;
  __syncthreads();
  if (line != 0 || i >= dim) return;
  s = 0.0f;
#pragma unroll
  for (int k = 0; k < kThreads / kJoinColumns; ++k) s += sums[k][col];
  if (p32) static_cast<float*>(out)[i] = s;
  else static_cast<T*>(out)[i] = from_float<T>(s);
}

// Parts of the columns' sums: workgroups of the backward pass, four a CU at most (each writes two
// rows of sums and the last launch reads them), and eight rows or more each.  16,384 x 2,048
// bfloat16, backward and join: 97 + 5 us with 256 parts, 57 + 5 with 512, 39 + 7 with 1,024,
// 46 + 11 with 2,048.
constexpr int64_t kMostParts = 1024;
int32_t norm_parts(int64_t rows) {
  return static_cast<int32_t>(std::clamp<int64_t>((rows + 7) / 8, 1, kMostParts));
}

constexpr int64_t kMostBlocks = 1 << 20;

// Whether the memory from the first to the last element of two matrices with these strides meets.
template <typename T>
bool overlap(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows,
             int32_t dim) {
  const auto bytes = [&](int64_t stride) {
    return (static_cast<uint64_t>(rows - 1) * static_cast<uint64_t>(stride) + dim) * sizeof(T);
  };
  const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  return a && b && rows > 0 && p < q + bytes(b_stride) && q < p + bytes(a_stride);
}

// Rows up to which the columns' sums have workgroups of their own beside the rows', in one launch.
// A backward pass with a join and without, us: 27 rows of 704 16.9 and 14.0, 512 of 4,000 bfloat16
// 19.7 and 13.8, 1,024 of 2,048 binary32 16.7 and 20.3.
constexpr int64_t kFewRows = 512;

template <typename T, int TPR, int NC>
void forward_rows(const NormArgs& a, hipStream_t st) {
  constexpr int kRows = kThreads / TPR;
  const int64_t nb = std::min((a.rows + kRows - 1) / kRows, kMostBlocks);
  ln_forward<T, TPR, NC><<<static_cast<uint32_t>(nb), kThreads, 0, st>>>(a);
}

// A wave a row while its lanes hold the row in 4 chunks (no barrier), else a workgroup (16,384 x
// 4,096 bfloat16: 63 us with a workgroup and 2 chunks a lane, 130 us with a wave and 8); fewer
// rows than waves fill the chip with take a workgroup each from one chunk a lane on.
template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t st) {
  constexpr int kRow = kWave * kWidth<T>;  // elements of one chunk a lane of a wave
  const int32_t d = a.dim;
  if (d <= kRow) forward_rows<T, kWave, 1>(a, st);
  else if (d <= 2 * kRow && a.rows >= 512) forward_rows<T, kWave, 2>(a, st);
  else if (d <= 4 * kRow && a.rows >= 512) forward_rows<T, kWave, 4>(a, st);
  else if (d <= 4 * kRow) forward_rows<T, kThreads, 1>(a, st);
  else if (d <= 8 * kRow) forward_rows<T, kThreads, 2>(a, st);
  else if (d <= 16 * kRow) forward_rows<T, kThreads, 4>(a, st);
  else if (sizeof(T) == 4 && d <= 32 * kRow)
    forward_rows<T, kThreads, sizeof(T) == 4 ? 8 : 4>(a, st);
  else ln_forward_long<T><<<static_cast<uint32_t>(std::min(a.rows, kMostBlocks)), kThreads, 0,
                            st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(NormBackArgs a, void* dw, void* db, hipStream_t st) {
  constexpr int kRow = kWave * kWidth<T>;
  const int32_t d = a.dim;
  const bool sums = dw || db;
  if (!sums) a.part = nullptr;
  a.parts = norm_parts(a.rows);
  // without the columns' sums a workgroup need not take many rows
  const uint32_t nb = sums ? a.parts
                           : static_cast<uint32_t>(std::min(std::max<int64_t>(a.rows, 1),
                                                            kMostBlocks));
  // few rows: the columns' sums by workgroups of their own in the same launch, without a join; not
  // where dx goes over the dy or x that they read (else a workgroup reads all of a row before it
  // writes any of it, and takes its part of the sums from what it read)
  const bool few = sums && a.rows <= kFewRows && d <= 16 * kRow &&
                   !overlap<T>(a.dx, a.dx_stride, a.dy, a.dy_stride, a.rows, d) &&
                   !overlap<T>(a.dx, a.dx_stride, a.x, a.x_stride, a.rows, d);
  a.row_blocks = nb;
  uint32_t grid = nb;
  if (few) {
    a.part = nullptr;
    a.dw = dw;
    a.db = db;
    a.row_blocks = a.dx ? static_cast<uint32_t>(a.rows) : 0;
    grid = a.row_blocks + static_cast<uint32_t>((d + kWave - 1) / kWave);
  }
  if (d <= kRow) ln_backward<T, kWave, 1><<<grid, kThreads, 0, st>>>(a);
  else if (d <= 4 * kRow) ln_backward<T, kThreads, 1><<<grid, kThreads, 0, st>>>(a);
  else if (d <= 8 * kRow) ln_backward<T, kThreads, 2><<<grid, kThreads, 0, st>>>(a);
  else if (d <= 16 * kRow) ln_backward<T, kThreads, 4><<<grid, kThreads, 0, st>>>(a);
  else {
    if (sums)  // (first: dx may go over dy or x)
      ln_columns<T><<<dim3((d + kThreads - 1) / kThreads, a.parts), kThreads, 0, st>>>(a);
    if (a.dx && a.rows > 0)
      ln_backward_long<T><<<static_cast<uint32_t>(std::min(a.rows, kMostBlocks)), kThreads, 0,
                            st>>>(a);
  }
  if (sums && !few)
    ln_join<T><<<dim3((d + kJoinColumns - 1) / kJoinColumns, 2), kThreads, 0, st>>>(
        d, a.parts, a.p32, a.part, dw, db);
  return hipGetLastError();
}

bool types_ok(int32_t dtype, int32_t param_dtype) {
  return dtype >= GSN_F32 && dtype <= GSN_F16 &&
         (param_dtype == GSN_F32 || param_dtype == dtype);
}

constexpr int64_t kMostRows = int64_t{1} << 40;
// (32-bit places in a row, with a step past its end; 16 threads a column in the columns' join)
constexpr int32_t kMostDim = 1 << 27;

}  // namespace
}  // namespace gsn

extern "C" {

int gsn_layer_norm(int32_t dtype, int32_t param_dtype, int64_t rows, int32_t dim, const void* x,
                   int64_t x_stride, const void* weight, const void* bias, float eps, void* y,
                   int64_t y_stride, float* stats, void* stream) {
  if (!gsn::types_ok(dtype, param_dtype) || rows < 0 || rows > gsn::kMostRows || dim < 1 ||
      dim > gsn::kMostDim || !(eps >= 0.0f))
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
  if (rows < 0 || rows > gsn::kMostRows || dim < 1 || dim > gsn::kMostDim) return 0;
  return sizeof(float) * 2 * static_cast<size_t>(gsn::norm_parts(rows)) * dim;
}

int gsn_layer_norm_backward(int32_t dtype, int32_t param_dtype, int64_t rows, int32_t dim,
                            const void* dy, int64_t dy_stride, const void* x, int64_t x_stride,
                            const void* weight, const float* stats, void* dx, int64_t dx_stride,
                            void* dweight, void* dbias, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (!gsn::types_ok(dtype, param_dtype) || rows < 0 || rows > gsn::kMostRows || dim < 1 ||
      dim > gsn::kMostDim)
    return GSN_E_INVAL;
  if (rows > 0 && (!dy || !x || !stats || dy_stride < dim || x_stride < dim ||
                   (dx && dx_stride < dim)))
    return GSN_E_INVAL;
  if (dweight || dbias) {
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return GSN_E_INVAL;
    if (workspace_bytes < gsn_layer_norm_workspace_bytes(rows, dim)) return GSN_E_CAPACITY;
  }
  const gsn::NormBackArgs a{rows, dim, dy, dy_stride, x, x_stride, weight,
                            param_dtype == GSN_F32, stats, dx, dx_stride, 0,
                            static_cast<float*>(workspace), 0, nullptr, nullptr};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e =
      dtype == GSN_F32    ? gsn::backward<float>(a, dweight, dbias, st)
      : dtype == GSN_BF16 ? gsn::backward<gsn::bf16_t>(a, dweight, dbias, st)
                          : gsn::backward<gsn::f16_t>(a, dweight, dbias, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

}  // extern "C"
