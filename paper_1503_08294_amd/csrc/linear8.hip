// Products of 8-bit integers: rows quantised to 8 bits, multiplied with weights of 8 bits in sums
// of 32-bit integers, which are exact.
#include <algorithm>

#include "few.h"
#include "product.h"

namespace gsn {
namespace {

struct Linear8 {
  int64_t tokens;
  int32_t dim, out, pitch;  // pitch: bytes of a row of q and of the copy of w
  const void* x;
  int64_t x_stride;
  const int8_t* w;
  int64_t w_stride;
  const float* scales;
  void* y;
  int64_t y_stride;
  int8_t* q;        // [tokens][pitch], zeros at the rows' ends
  float* x_scales;  // [tokens]
  int8_t* wc;       // [out][pitch] w, where its rows are not at multiples of 16 bytes; many tokens
  bool lines;       // rows of y begin and end at multiples of 16 bytes
};

// v / s to the nearest integer, ties to even, as of the exact quotient, where `q` is the product
// with 1 / s rounded so: it may be one off beside a border, and an fma's sign tells on which side
// of the border v is, or that it is on it.
__device__ __forceinline__ float beside_border(float q, float v, float s) {
  const float above = fmaf(-(q + 0.5f), s, v);  // > 0: v / s > q + 0.5
  const float below = fmaf(-(q - 0.5f), s, v);  // < 0: v / s < q - 0.5
  const bool odd = (static_cast<int>(q) & 1) != 0;
  if (above > 0.0f || (above == 0.0f && odd)) return q + 1.0f;
  if (below < 0.0f || (below == 0.0f && odd)) return q - 1.0f;
  return q;
}
// Eight of them (|v / s| <= 127 but for rounding) as bytes.  The quotient goes next to 1.5 2^23,
// where binary32 values are 1 apart and their last byte is the integer's.  What is left of v after q
// s has an error of 2^-24 of itself: up to 0.4999 s no other integer is nearer, and few values are
// looked at again.
__device__ __forceinline__ uint2 quantised(const float* v, float s, float inverse) {
  constexpr float kOnes = 0x1.8p23f;
  float at[8], most = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    at[i] = fmaf(v[i], inverse, kOnes);
    most = fmaxf(most, fabsf(fmaf(kOnes - at[i], s, v[i])));
  }
  if (__any(most >= 0.4999f * s)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) at[i] = beside_border(at[i] - kOnes, v[i], s) + kOnes;
  }
  uint32_t four[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float* const a = at + 4 * h;
    const auto two = [](float lo, float hi) {  // last bytes of both, in the low half
      return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x0c0c0400u);
    };
    four[h] = __builtin_amdgcn_perm(two(a[2], a[3]), two(a[0], a[1]), 0x05040100u);
  }
  return uint2{four[0], four[1]};
}

// The largest magnitude of some elements, as bits (larger for larger numbers, largest for NaN).
template <typename T>
struct Largest {
  typedef uint16_t Two __attribute__((ext_vector_type(2)));
  uint32_t top = 0;
  __device__ __forceinline__ void take(uint32_t bits) {
    if constexpr (sizeof(T) == 4)
      top = max(top, bits & 0x7fffffffu);
    else
      top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(
                                             __builtin_bit_cast(Two, top),
                                             __builtin_bit_cast(Two, bits & 0x7fff7fffu)));
  }
  // as bits of a binary32 value
  __device__ __forceinline__ uint32_t value() const {
    if constexpr (sizeof(T) == 4) {
      return top;
    } else {
      const uint16_t one = static_cast<uint16_t>(max(top & 0xffffu, top >> 16));
      return __float_as_uint(to_float(__builtin_bit_cast(T, one)));
    }
  }
};

// Rows in 8 bits, a row by THREADS, a workgroup or a wave: the largest value, then the quotients, 8
// KEPT elements a thread kept in registers in between.  `pitch` bytes of q are written (at most up
// to the next multiple of 16 bytes), zeros past the end.  8,191 rows of 4,096: bfloat16 27 us (3.7
// TB/s), binary32 31 us (5.5 TB/s, bound by memory).
constexpr int kRowThreads = 256;
template <int THREADS, int KEPT, typename T>
__device__ __forceinline__ void quantise_rows(const T* __restrict__ x, int64_t stride,
                                              int64_t rows, int32_t dim, int8_t* __restrict__ q,
                                              int64_t q_stride, int32_t pitch,
                                              float* __restrict__ scales, int64_t block,
                                              int64_t blocks) {
  // (elements go in eights; up to 7 that are left, and the zeros behind them, are one a thread:
  // eights that may all end early take registers for twice the waves, 35 us in place of 27)
  constexpr int kE = 16 / static_cast<int>(sizeof(T)), kParts = 8 / kE;
  struct Eight {
    Frag f[kParts];
  };
  __shared__ uint32_t some[THREADS / kWave];
  const int tid = threadIdx.x % THREADS;
  const int32_t chunks = dim / 8, rest = dim - 8 * chunks;
  for (int64_t r = block; r < rows; r += blocks) {
    const T* const row = x + r * stride;
    Eight kept[KEPT];
    Largest<T> most;
    const auto load = [&](int32_t c) {
      Eight v;
#pragma unroll
      for (int h = 0; h < kParts; ++h) {
        if (c < chunks) v.f[h] = row_chunk<true>(row, c * 8 + h * kE, dim);
        else v.f[h].u = u32x4{0, 0, 0, 0};
      }
      return v;
    };
    const auto largest = [&](const Eight& v) {
#pragma unroll
      for (int h = 0; h < kParts; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) most.take(v.f[h].u[i]);
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i)
      if (i * THREADS < chunks) kept[i] = load(i * THREADS + tid);
    const float left = tid < rest ? to_float(row[8 * chunks + tid]) : 0.0f;
#pragma unroll
    for (int i = 0; i < KEPT; ++i)
      if (i * THREADS < chunks) largest(kept[i]);
    for (int32_t c = KEPT * THREADS + tid; c < chunks; c += THREADS) largest(load(c));
    uint32_t top = max(most.value(), __float_as_uint(left) & 0x7fffffffu);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o));
    if constexpr (THREADS > kWave) {
      __syncthreads();
      if (tid % kWave == 0) some[tid / kWave] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < THREADS / kWave; ++w) top = max(top, some[w]);
    }
    const bool bad = top >= 0x7f800000u;
    const float s = fmaxf(__uint_as_float(bad ? 0 : top) / 127.0f, 0x1p-126f), inverse = 1.0f / s;
    int8_t* const to = q + r * q_stride;
    const auto store = [&](int32_t c, const Eight& v) {
      if (c >= chunks) return;
      float f[8];
#pragma unroll
      for (int h = 0; h < kParts; ++h) {
        const Vec<T, kE> e = __builtin_bit_cast(Vec<T, kE>, v.f[h].u);
#pragma unroll
        for (int i = 0; i < kE; ++i) f[h * kE + i] = bad ? 0.0f : to_float(e.v[i]);
      }
      const uint2 o = quantised(f, s, inverse);
      typedef uint32_t Loose __attribute__((ext_vector_type(2), aligned(1)));
      *reinterpret_cast<Loose*>(to + 8 * c) = Loose{o.x, o.y};
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i)
      if (i * THREADS < chunks) store(i * THREADS + tid, kept[i]);
    for (int32_t c = KEPT * THREADS + tid; c < chunks; c += THREADS) store(c, load(c));
    if (8 * chunks + tid < pitch) {
      const float v = bad ? 0.0f : left;
      to[8 * chunks + tid] =
          static_cast<int8_t>(static_cast<int>(beside_border(rintf(v * inverse), v, s)));
    }
    if (tid == 0) scales[r] = bad ? NAN : s;
  }
}

template <typename T, int THREADS, int KEPT>
__global__ __launch_bounds__(kRowThreads) void q8_rows(const T* x, int64_t stride, int64_t rows,
                                                       int32_t dim, int8_t* q, int64_t q_stride,
                                                       float* scales) {
  constexpr int kRows = kRowThreads / THREADS;
  quantise_rows<THREADS, KEPT>(x, stride, rows, dim, q, q_stride, dim, scales,
                               int64_t{blockIdx.x} * kRows + threadIdx.x / THREADS,
                               int64_t{gridDim.x} * kRows);
}

// x in 8 bits by the first `blocks` workgroups, and by the others w in rows of `pitch` bytes with
// zeros at their ends.
template <typename T, int THREADS, int KEPT>
__global__ __launch_bounds__(kRowThreads) void q8_begin(Linear8 x, uint32_t blocks) {
  constexpr int kRows = kRowThreads / THREADS;  // of a workgroup at a time
  if (blockIdx.x < blocks)
    return quantise_rows<THREADS, KEPT>(
        static_cast<const T*>(x.x), x.x_stride, x.tokens, x.dim, x.q, x.pitch, x.pitch,
        x.x_scales, int64_t{blockIdx.x} * kRows + threadIdx.x / THREADS, int64_t{blocks} * kRows);
  const int32_t each = x.pitch / 16;
  const int64_t all = static_cast<int64_t>(x.out) * each;
  for (int64_t i = static_cast<int64_t>(blockIdx.x - blocks) * kRowThreads + threadIdx.x; i < all;
       i += static_cast<int64_t>(gridDim.x - blocks) * kRowThreads) {
    const int64_t r = i / each;
    const int32_t k = static_cast<int32_t>(i - r * each) * 16;
    *reinterpret_cast<u32x4*>(x.wc + i * 16) =
        row_chunk<false>(x.w + r * x.w_stride, k, x.dim).u;
  }
}

// A sum times two scales.  Where one of them is `far` from 1, the sum times it may leave binary32's
// range though the result does not: then numbers from 1/2 to 1 are multiplied and the powers of two
// added.  (8,191 tokens through 4,096 x 8,192 in bfloat16: 265 us without a look at the scales, 268
// with one for a wave's part of a tile, 274 with one for each of its 16 rows.)
__device__ __forceinline__ bool far(float scale) {
  return !(fabsf(scale) >= 0x1p-60f && fabsf(scale) <= 0x1p60f);
}
__device__ __forceinline__ float times(int32_t sum, float a, float b) {
  return static_cast<float>(sum) * a * b;
}
__device__ __forceinline__ float times_far(int32_t sum, float a, float b) {
  int ea = 0, eb = 0;
  const float ma = isfinite(a) ? frexpf(a, &ea) : a, mb = isfinite(b) ? frexpf(b, &eb) : b;
  return ldexpf(times(sum, ma, mb), ea + eb);
}

template <typename T>
struct Scaled {
  Linear8 x;

  __device__ __forceinline__ void few(int32_t m, int32_t n, i32x4 sums) const {
    if (n >= x.out) return;
    float v[4];
    load4(x.scales, n, x.out, v);
    const float s = x.x_scales[m];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      v[q] = far(s) || far(v[q]) ? times_far(sums[q], s, v[q]) : times(sums[q], s, v[q]);
    store4(static_cast<T*>(x.y) + m * x.y_stride, n, x.out, v);
  }

  template <int MT, int NT>
  __device__ __forceinline__ void tile_far(const i32x4 (&acc)[MT][NT], int64_t m, int32_t n,
                                           int lane, const float (&cols)[NT][4],
                                           const float (&rows)[MT]) const {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t t = m + 16 * i + (lane & 15);
      if (t >= x.tokens) return;
      T* const row = static_cast<T*>(x.y) + t * x.y_stride;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = times_far(acc[i][j][q], rows[i], cols[j][q]);
        if (n + 16 * j < x.out) store4(row, n + 16 * j, x.out, v);
      }
    }
  }

  template <class TILE, int MT, int NT>
  __device__ __forceinline__ void tile(i32x4 (&acc)[MT][NT], const Place& at, int mw, int nw,
                                       int lane, char* smem) const {
    const int32_t n0 = at.n0 + nw, n = n0 + (lane >> 4) * 4;
    using Lines = Turn<T, 16 * NT>;
    static_assert(Lines::kBytes <= TILE::kLds / 4);
    const Lines turn{smem + threadIdx.x / kWave * (TILE::kLds / 4)};
    float cols[NT][4], rows[MT];
    bool any_far = false;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      load4(x.scales, n + 16 * j, x.out, cols[j]);
#pragma unroll
      for (int q = 0; q < 4; ++q) any_far |= n + 16 * j + q < x.out && far(cols[j][q]);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t t = at.m0 + mw + 16 * i + (lane & 15);
      rows[i] = x.x_scales[t < x.tokens ? t : x.tokens - 1];
      any_far |= far(rows[i]);
    }
    if (__any(any_far)) return tile_far(acc, int64_t{at.m0} + mw, n, lane, cols, rows);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t t0 = at.m0 + mw + 16 * i, t = t0 + (lane & 15);
      if (t0 >= x.tokens) break;
      T* const row = static_cast<T*>(x.y) + t * x.y_stride;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = times(acc[i][j][q], rows[i], cols[j][q]);
        if (x.lines) turn.put(lane & 15, 16 * j + (lane >> 4) * 4, v);
        else if (t < x.tokens && n + 16 * j < x.out) store4(row, n + 16 * j, x.out, v);
      }
      if (!x.lines) continue;
      wave_fence();
      const int64_t left = x.tokens - t0;
      turn.out(static_cast<T*>(x.y) + t0 * x.y_stride + n0, x.y_stride,
               static_cast<int32_t>(left < 16 ? left : 16), x.out - n0, lane);
      wave_fence();
    }
  }
};

// One or two tokens in one launch: every workgroup brings the tokens to 8 bits for itself, in LDS,
// while its first rows of w are on their way, and takes 32 columns as few_rows() does.  One token
// through 4,096 x 16,384: 13.0 us, 15.7 as two launches (67 MB at 5.2 TB/s).
constexpr int64_t kTokensAlone = 2;
constexpr int32_t kDimAlone = 16384;
template <typename T>
__global__ __launch_bounds__(256) void q8_alone(Linear8 x) {
  constexpr int kStep = kRowBytes, GT = kFewCols / 16;
  __shared__ __attribute__((aligned(16))) int8_t q[kTokensAlone * kDimAlone];
  __shared__ float scale[kTokensAlone];
  __shared__ i32x4 part[4][GT][kWave];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = lane >> 4, i = lane & 15;
  const int32_t n0 = blockIdx.x * kFewCols, dim = x.dim;
  const int8_t* w[GT];
#pragma unroll
  for (int t = 0; t < GT; ++t) {
    const int32_t n = n0 + 16 * t + i;
    w[t] = x.w + (n < x.out ? n : x.out - 1) * x.w_stride;
  }
  const int32_t steps = (dim + kStep - 1) / kStep, per = (steps + 3) / 4;
  const int32_t k_begin = wave * per * kStep;
  const int32_t k_end = k_begin + per * kStep < dim ? k_begin + per * kStep : dim;
  Frag fw[2][GT];
  const auto load = [&](auto inside, int32_t k0) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < GT; ++t)
        fw[h][t] = row_chunk<decltype(inside)::value>(w[t], k0 + (4 * h + g) * 16, dim);
  };
  const bool whole = k_begin + kStep <= k_end;
  if (whole) load(std::true_type(), k_begin);
  const int32_t pitch = x.pitch;
  quantise_rows<kRowThreads, 4>(static_cast<const T*>(x.x), x.x_stride, x.tokens, dim, q, pitch,
                                pitch, scale, 0, 1);
  __syncthreads();

  i32x4 acc[GT] = {};
  const bool live = i < x.tokens;
  const auto multiply_these = [&](const Frag (&a)[2][GT], int32_t k0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int32_t k = k0 + (4 * h + g) * 16;
      Frag f;
      f.u = u32x4{0, 0, 0, 0};
      if (live && k < pitch) f.u = *reinterpret_cast<const u32x4*>(q + i * pitch + k);
#pragma unroll
      for (int t = 0; t < GT; ++t) acc[t] = multiply_any<int8_t>(a[h][t], f, acc[t], 0);
    }
  };
  int32_t k0 = k_begin;
  if (whole) {
    for (; k0 + 2 * kStep <= k_end; k0 += kStep) {
      Frag a[2][GT];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < GT; ++t) a[h][t] = fw[h][t];
      load(std::true_type(), k0 + kStep);
      multiply_these(a, k0);
    }
    multiply_these(fw, k0);
    k0 += kStep;
  }
  if (k0 < k_end) {
    load(std::false_type(), k0);
    multiply_these(fw, k0);
  }
#pragma unroll
  for (int t = 0; t < GT; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  const int m = tid >> 3, c = tid & 7, n = n0 + 4 * c;
  if (m >= x.tokens || n >= x.out) return;
  i32x4 sum = {};
#pragma unroll
  for (int u = 0; u < 4; ++u) sum += part[u][c >> 2][(c & 3) * 16 + m];
  float v[4];
  load4(x.scales, n, x.out, v);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    v[e] = far(scale[m]) || far(v[e]) ? times_far(sum[e], scale[m], v[e])
                                      : times(sum[e], scale[m], v[e]);
  store4(static_cast<T*>(x.y) + m * x.y_stride, n, x.out, v);
}

// Rows by a wave each, where they fit its registers and there are enough: no wait for other waves.
// By workgroups and by waves, us, bfloat16: 65,536 rows of 64 76 and 22, 8,191 of 1,001 15.1 and
// 9.4, 2,048 of 1,024 5.9 and 4.6, 1,024 of 1,024 3.9 and 3.9; 16,384 of 2,048 34 and 26, 4,096 of
// 2,048 10.4 and 9.6, 2,048 of 2,048 6.6 and 7.1; 16,384 of 4,096 48.6 and 47.7, 8,191 27 and 31.
constexpr int32_t kWaveDim = 2048;
bool by_waves(int64_t rows, int32_t dim) {
  return dim <= kWaveDim && rows >= 2 * std::max(dim, 1024);
}
uint32_t row_blocks(int64_t rows, bool waves) {
  return static_cast<uint32_t>(std::min<int64_t>(waves ? (rows + 3) / 4 : rows, 1 << 16));
}

template <typename T>
hipError_t launch(const Linear8& x, hipStream_t st) {
  // A few tokens: w is read once, as it is.  Otherwise its rows have to begin and end at multiples
  // of 16 bytes.
  const bool aligned = aligned16(x.w) && x.w_stride % 16 == 0 && x.dim % 16 == 0;
  const bool few = x.tokens <= few_at_most(false, aligned);
  const bool copy = !few && !aligned;
  if (x.tokens <= kTokensAlone && x.pitch <= kDimAlone) {
    q8_alone<T><<<static_cast<uint32_t>((x.out + kFewCols - 1) / kFewCols), 256, 0, st>>>(x);
    return hipGetLastError();
  }
  const bool waves = by_waves(x.tokens, x.dim);
  const uint32_t blocks = row_blocks(x.tokens, waves);
  const int64_t copies =
      (static_cast<int64_t>(x.out) * (x.pitch / 16) + kRowThreads - 1) / kRowThreads;
  const uint32_t grid =
      blocks + (copy ? static_cast<uint32_t>(std::min<int64_t>(copies, 1 << 14)) : 0);
  if (waves) q8_begin<T, kWave, kWaveDim / 512><<<grid, kRowThreads, 0, st>>>(x, blocks);
  else q8_begin<T, kRowThreads, 4><<<grid, kRowThreads, 0, st>>>(x, blocks);
  if (few) {
    run_few<int8_t>(Few{x.q, x.pitch, x.w, x.w_stride, static_cast<int32_t>(x.tokens), x.out,
                        x.dim}, Scaled<T>{x}, st);
    return hipGetLastError();
  }
  Product p{};
  p.a = Operand{reinterpret_cast<const char*>(x.q), {0, 0}, x.pitch, 0,
                static_cast<int32_t>(x.tokens)};
  p.b = Operand{reinterpret_cast<const char*>(copy ? x.wc : x.w), {0, 0},
                copy ? x.pitch : x.w_stride, 0, x.out};
  p.terms = p.batch = p.splits = 1;
  p.k = p.part = x.dim;
  run_product<int8_t, false, false>(p, Scaled<T>{x}, st);
  return hipGetLastError();
}

bool params_ok(const gsn_linear_params* p) {
  // (a sum of 2^17 - 1 products of -128 and -128 is the last below 2^31)
  return p && p->dtype >= GSN_F32 && p->dtype <= GSN_F16 && p->tokens >= 0 &&
         p->tokens <= (1 << 24) && p->dim >= 1 && p->dim < (1 << 17) && p->out >= 1 &&
         p->out <= (1 << 28);
}

Linear8 linear8_of(const gsn_linear_params& p) {
  Linear8 x{};
  x.tokens = p.tokens;
  x.dim = p.dim;
  x.out = p.out;
  x.pitch = (p.dim + 15) / 16 * 16;
  return x;
}

size_t carve(void* base, Linear8* x) {
  size_t used = 0;
  const auto take = [&](size_t n) {
    char* const p = base ? static_cast<char*>(base) + used : nullptr;
    used += (n + 255) / 256 * 256;
    return static_cast<void*>(p);
  };
  const size_t pitch = static_cast<size_t>(x->pitch);
  x->q = static_cast<int8_t*>(take(static_cast<size_t>(x->tokens) * pitch));
  x->x_scales = static_cast<float*>(take(4 * static_cast<size_t>(x->tokens)));
  // (launch() copies w for no fewer tokens)
  if (x->tokens > few_at_most(false, false))
    x->wc = static_cast<int8_t*>(take(static_cast<size_t>(x->out) * pitch));
  return used;
}

}  // namespace
}  // namespace gsn

extern "C" {

int gsn_quantise(int32_t dtype, int64_t rows, int32_t dim, const void* x, int64_t x_stride,
                 int8_t* q, int64_t q_stride, float* scales, void* stream) {
  if (dtype < GSN_F32 || dtype > GSN_F16 || rows < 0 || dim < 1 || dim > (1 << 27))
    return GSN_E_INVAL;
  if (rows == 0) return GSN_OK;
  if (!x || !q || !scales || x_stride < dim || q_stride < dim) return GSN_E_INVAL;
  if (q == x || scales == x || q == static_cast<const void*>(scales)) return GSN_E_INVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool waves = gsn::by_waves(rows, dim);
  const uint32_t blocks = gsn::row_blocks(rows, waves);
  const auto run = [&](auto* p) {
    using T = std::remove_const_t<std::remove_pointer_t<decltype(p)>>;
    if (waves)
      gsn::q8_rows<T, gsn::kWave, gsn::kWaveDim / 512><<<blocks, gsn::kRowThreads, 0, st>>>(
          p, x_stride, rows, dim, q, q_stride, scales);
    else
      gsn::q8_rows<T, gsn::kRowThreads, 4><<<blocks, gsn::kRowThreads, 0, st>>>(
          p, x_stride, rows, dim, q, q_stride, scales);
  };
  if (dtype == GSN_F32) run(static_cast<const float*>(x));
  else if (dtype == GSN_BF16) run(static_cast<const gsn::bf16_t*>(x));
  else run(static_cast<const gsn::f16_t*>(x));
  return hipGetLastError() == hipSuccess ? GSN_OK : GSN_E_HIP;
}

size_t gsn_linear_quantised_workspace_bytes(const gsn_linear_params* p) {
  if (!gsn::params_ok(p)) return 0;
  gsn::Linear8 x = gsn::linear8_of(*p);
  return gsn::carve(nullptr, &x) + 256;
}

int gsn_linear_quantised(const gsn_linear_params* p, const void* x, int64_t x_stride,
                         const int8_t* w, int64_t w_stride, const float* scales, void* y,
                         int64_t y_stride, void* workspace, size_t workspace_bytes,
                         void* stream) {
  if (!gsn::params_ok(p)) return GSN_E_INVAL;
  if (p->tokens == 0) return GSN_OK;
  if (!x || !w || !scales || !y || x_stride < p->dim || w_stride < p->dim || y_stride < p->out ||
      !workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return GSN_E_INVAL;
  if (workspace_bytes < gsn_linear_quantised_workspace_bytes(p)) return GSN_E_CAPACITY;
  if (int64_t{gsn::tiles_of(p->tokens, gsn::kMiddleRows)} *
          gsn::tiles_of(p->out, gsn::kMiddleRows) >= (1 << 23))
    return GSN_E_CAPACITY;
  if (y == x || y == w || y == scales) return GSN_E_INVAL;
  gsn::Linear8 a = gsn::linear8_of(*p);
  a.x = x;
  a.x_stride = x_stride;
  a.w = w;
  a.w_stride = w_stride;
  a.scales = scales;
  a.y = y;
  a.y_stride = y_stride;
  const int64_t elements = 16 / static_cast<int64_t>(gsn::size_of(p->dtype));
  a.lines = gsn::aligned16(y) && y_stride % elements == 0 && p->out % elements == 0;
  gsn::carve(workspace, &a);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = p->dtype == GSN_F32    ? gsn::launch<float>(a, st)
                       : p->dtype == GSN_BF16 ? gsn::launch<gsn::bf16_t>(a, st)
                                              : gsn::launch<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

}  // extern "C"
