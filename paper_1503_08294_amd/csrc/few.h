// Products of a few rows with a large matrix, read once: y(m, n) = sum over k of x(m, k) w(n, k).
//
// Bound by reading w.  No staging: a wave loads 32 rows of w straight into fragments, the next 128
// bytes of k while it multiplies these, with 16 MT rows of x.  The four waves of a workgroup take a
// quarter of k each, joined through LDS.  Rows start at any element.  One token against 65,536
// classes of 2,048, bfloat16: 0.27 GB in 50 us (5.4 TB/s; a large copy 4.9); through 4,096 x 16,384
// in 8 bits 67 MB in 13 us.
#pragma once

#include "product.h"

namespace gsn {

struct Few {
  const void* x;
  int64_t x_stride;  // elements
  const void* w;
  int64_t w_stride;
  int32_t rows, cols, k;  // of x, rows of w
};

// Rows of x up to which this is taken in place of tiles, which read x once a tile from LDS.  The
// two in us: 50,001 classes of 1,024, bfloat16, 16 rows 28 and 28, 24 rows 32 and 28, 64 rows 48
// and 28; 60,000 of 1,024, binary32, 32 rows 70 and 88, 33 rows 102 and 88.  Tiles of a w whose
// rows do not begin at multiples of 16 bytes take a copy of it, which is twice its bytes more to
// move.
constexpr int64_t few_at_most(bool binary32, bool aligned) {
  return !aligned ? 64 : binary32 ? 32 : 16;
}
constexpr int32_t kFewCols = 32;  // columns of a workgroup

namespace {

// What becomes of the results: EPI::few(m, n, v) with row m's columns n to n + 3 (some of them past
// the last one), by 8 lanes that follow each other for each row.
template <typename T, int MT, class EPI>
__global__ __launch_bounds__(256) void few_rows(Few p, EPI epi) {
  constexpr int kE = 16 / static_cast<int>(sizeof(T)), kStep = 8 * kE, GT = kFewCols / 16;
  using Acc = AccOf<T>;
  __shared__ Acc part[4][GT][MT][kWave];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = lane >> 4, i = lane & 15;
  const int32_t n0 = blockIdx.x * kFewCols;
  const T* w[GT];
#pragma unroll
  for (int t = 0; t < GT; ++t) {
    const int32_t n = n0 + 16 * t + i;
    w[t] = static_cast<const T*>(p.w) + (n < p.cols ? n : p.cols - 1) * p.w_stride;
  }
  const T* x[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int32_t r = 16 * m + i;
    x[m] = static_cast<const T*>(p.x) + (r < p.rows ? r : p.rows - 1) * p.x_stride;
  }
  const int32_t steps = (p.k + kStep - 1) / kStep, per = (steps + 3) / 4;
  const int32_t k_begin = wave * per * kStep;
  const int32_t k_end = k_begin + per * kStep < p.k ? k_begin + per * kStep : p.k;

  Acc acc[GT][MT];
#pragma unroll
  for (int t = 0; t < GT; ++t)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[t][m] = Acc{0, 0, 0, 0};
  Frag fw[2][GT], fx[2][MT];
  const auto load = [&](auto inside, int32_t k0) {
    constexpr bool kIn = decltype(inside)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int32_t k = k0 + (4 * h + g) * kE;
#pragma unroll
      for (int t = 0; t < GT; ++t) fw[h][t] = row_chunk<kIn>(w[t], k, p.k);
#pragma unroll
      for (int m = 0; m < MT; ++m) fx[h][m] = row_chunk<kIn>(x[m], k, p.k);
    }
  };
  const auto multiply_these = [&](const Frag (&aw)[2][GT], const Frag (&ax)[2][MT]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < kParts<T>; ++q)
#pragma unroll
        for (int t = 0; t < GT; ++t)
#pragma unroll
          for (int m = 0; m < MT; ++m)
            acc[t][m] = multiply_any<T>(aw[h][t], ax[h][m], acc[t][m], q);
  };
  int32_t k0 = k_begin;
  if (k0 + kStep <= k_end) {
    load(std::true_type(), k0);
    for (; k0 + 2 * kStep <= k_end; k0 += kStep) {
      Frag aw[2][GT], ax[2][MT];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < GT; ++t) aw[h][t] = fw[h][t];
#pragma unroll
        for (int m = 0; m < MT; ++m) ax[h][m] = fx[h][m];
      }
      load(std::true_type(), k0 + kStep);
      multiply_these(aw, ax);
    }
    multiply_these(fw, fx);
    k0 += kStep;
  }
  if (k0 < k_end) {
    load(std::false_type(), k0);
    multiply_these(fw, fx);
  }
#pragma unroll
  for (int t = 0; t < GT; ++t)
#pragma unroll
    for (int m = 0; m < MT; ++m) part[wave][t][m][lane] = acc[t][m];
  __syncthreads();
  const int c = tid & 7;
  for (int m = tid >> 3; m < 16 * MT && m < p.rows; m += 32) {
    Acc v = part[0][c >> 2][m >> 4][(c & 3) * 16 + (m & 15)];
#pragma unroll
    for (int u = 1; u < 4; ++u) v += part[u][c >> 2][m >> 4][(c & 3) * 16 + (m & 15)];
    epi.few(m, n0 + 4 * c, v);
  }
}

template <typename T, class EPI>
void run_few(const Few& p, const EPI& epi, hipStream_t st) {
  static_assert(few_at_most(false, false) <= 64);
  const uint32_t grid = static_cast<uint32_t>((p.cols + kFewCols - 1) / kFewCols);
  if (p.rows <= 16) few_rows<T, 1><<<grid, 256, 0, st>>>(p, epi);
  else if (p.rows <= 32) few_rows<T, 2><<<grid, 256, 0, st>>>(p, epi);
  else few_rows<T, 4><<<grid, 256, 0, st>>>(p, epi);
}

}  // namespace
}  // namespace gsn
