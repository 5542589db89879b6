// Products of matrices of any sizes in tiles, with a functor for what becomes of a tile's results.
//
//   C(m, n) = sum over terms s and k of A_s(m, k) B_s(n, k)    for every pair of a batch
//
// An operand lies in memory with k contiguous (its rows are m or n) or with m or n contiguous (its
// rows are k, TR).  Rows start at multiples of 16 bytes.  With k contiguous what follows k = K up
// to the next multiple of 16 bytes is read as well: both operands have zeros there.  With k as the
// row the columns' ends are read, and nothing is used of them.
#pragma once

#include <type_traits>

#include "experts_rule.h"
#include "tiles.h"

namespace gsn {

// One operand: of each term the matrix of the batch's first pair, all with the same steps.
struct Operand {
  const char* p;
  int64_t next[2];  // bytes from a term to the next
  int64_t ld;       // bytes from row to row
  int64_t batch;    // bytes from pair to pair
  int32_t rows;     // m or n that there are
};

struct Product {
  Operand a, b;
  int32_t terms, k, batch;
  int32_t splits;  // parts of k, each summed by a workgroup of its own
  int32_t part;    // k of a part, a multiple of a stage's
  int32_t tiles_m, tiles_n;
  int32_t symmetric;  // C = C^T: tiles with n0 >= m0 alone
};

// A tile: its pair of the batch, its first row and column, its part of k.
struct Place {
  int32_t pair, m0, n0, split;
};

inline int32_t tiles_of(int64_t n, int32_t side) {
  return static_cast<int32_t>((n + side - 1) / side);
}
inline int64_t tiles_of(const Product& p) {
  const int64_t t = p.symmetric ? int64_t{p.tiles_m} * (p.tiles_m + 1) / 2
                                : int64_t{p.tiles_m} * p.tiles_n;
  return t * p.batch * p.splits;
}

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

template <typename T>
using AccOf = std::conditional_t<sizeof(T) == 1, i32x4, f32x4>;

template <typename T>
__device__ __forceinline__ AccOf<T> multiply_any(const Frag& n, const Frag& m, AccOf<T> acc,
                                                 int q) {
  if constexpr (sizeof(T) == 1)
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, n.u),
                                                 __builtin_bit_cast(i32x4, m.u), acc, 0, 0, 0);
  else
    return multiply<T>(n, m, acc, q);
}

// Fragments of an operand of 8-bit elements: the bytes lie as those of wider elements with k
// contiguous do.
template <typename T, bool TR, int R>
__device__ __forceinline__ Frag fragment_any(const char* tile, int r0, int s, int lane) {
  if constexpr (sizeof(T) == 1) {
    static_assert(!TR);
    return fragment<float, false, R>(tile, r0, s, lane);
  } else {
    return fragment<T, TR, R>(tile, r0, s, lane);
  }
}

// What this lane loads of one operand's stages: of stage h the chunks j THR + thread for j = 0, 1,
// ..., SIDE rows (or columns) of 128 bytes of k in all.
template <typename T, bool TR, int SIDE, int THR>
struct Feed {
  static constexpr int kE = 16 / static_cast<int>(sizeof(T));
  static constexpr int kBK = kRowBytes / static_cast<int>(sizeof(T));
  static constexpr int kC = TR ? SIDE / kE : 8;  // chunks of a row
  static constexpr int kLoads = SIDE * 8 / THR;
  static constexpr int kStep = THR / kC;  // rows from one j to the next
  static_assert(THR % kC == 0 && SIDE * 8 % THR == 0);

  const char* p;   // the chunk j = 0 of the next stage
  int64_t ld, step;
  int32_t k, end;  // k of that stage (with k contiguous: of the chunk), and where k ends
  int32_t left;    // rows (columns) from this lane's on
  int r, c;

  __device__ __forceinline__ static int chunk(int row, int c) {
    if constexpr (TR) return chunk_n<T, kC>(row, c);
    else return chunk_k(row, c);
  }
  __device__ __forceinline__ void begin(const Operand& o, int32_t pair, int32_t row0, int32_t k0,
                                        int32_t k_end, int tid) {
    ld = o.ld;
    r = tid / kC;
    c = chunk(r, tid % kC);
    const char* base = o.p + pair * o.batch;
    if constexpr (TR) {
      p = base + static_cast<int64_t>(k0 + r) * ld +
          (static_cast<int64_t>(row0) + c * kE) * static_cast<int>(sizeof(T));
      step = kBK * ld;
      k = k0 + r;
      left = o.rows - row0;
    } else {
      p = base + static_cast<int64_t>(row0 + r) * ld +
          (static_cast<int64_t>(k0) + c * kE) * static_cast<int>(sizeof(T));
      step = kRowBytes;
      k = k0 + c * kE;
      left = o.rows - row0 - r;
    }
    end = k_end;
  }
  __device__ __forceinline__ void load(uint32_t at) {
    const char* const zeros = reinterpret_cast<const char*>(kZeros);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const char* from = p + j * (kStep * ld);
      bool in;
      if constexpr (TR) {
        int cj = c;
        if constexpr (kStep % 16 != 0) {  // (otherwise the chunk's place is the same for all j)
          cj = chunk(r + j * kStep, static_cast<int>(threadIdx.x) % kC);
          from += (cj - c) * 16;
        }
        in = k + j * kStep < end && cj * kE < left;
      } else {
        static_assert(kStep % 16 == 0);
        in = k < end && j * kStep < left;
      }
      load_to_lds(in ? from : zeros, at + j * (THR * 16));
    }
    p += step;
    k += kBK;
  }
  // to the next term after `stages` stages
  __device__ __forceinline__ void turn(int64_t next, int32_t stages) {
    p += next - stages * step;
    k -= stages * kBK;
  }
};

// Number of the tile in its pair -> its row and column of tiles.
__device__ __forceinline__ int2 symmetric_place(int32_t id) {
  // column c holds the tiles (0, c) .. (c, c), c (c + 1) / 2 before it
  int32_t c = static_cast<int32_t>((sqrtf(8.0f * static_cast<float>(id) + 1.0f) - 1.0f) * 0.5f);
  while (c * (c + 1) / 2 > id) --c;
  while ((c + 1) * (c + 2) / 2 <= id) ++c;
  return int2{id - c * (c + 1) / 2, c};
}

// false: no tile for this workgroup.
template <int SIDE>
__device__ __forceinline__ bool place_of(const Product& p, Place* at) {
  const int32_t each =
      p.symmetric ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
  const int32_t id = spread(blockIdx.x, each * p.batch * p.splits, tile_run(SIDE));
  if (id < 0) return false;
  const int32_t outer = id / each, in = id - outer * each;
  const int2 t = p.symmetric ? symmetric_place(in) : tile_place<4>(in, p.tiles_m, p.tiles_n);
  at->split = outer / p.batch;
  at->pair = outer - at->split * p.batch;
  at->m0 = t.x * SIDE;
  at->n0 = t.y * SIDE;
  return true;
}

// Workgroups of a product's grid.
template <int SIDE>
int64_t grid_of(const Product& p) {
  constexpr int64_t round = 8 * tile_run(SIDE);
  return (tiles_of(p) + round - 1) / round * round;
}

// Tiles of 128 or 64 a side by four waves, 2 x 2 of them.  Stages go from memory straight to LDS;
// a stage is awaited by all waves together, then a later one is sent out and this one multiplied.
template <int SIDE>
constexpr int kSlots = SIDE == kMiddleRows ? 2 : 3;
template <int SIDE>
constexpr int kProductLds = kSlots<SIDE> * 2 * SIDE * kRowBytes;
constexpr int kProductThreads = 256;

// What becomes of a tile's results is the functor's:
//   EPI::tile<SIDE, WN, MT, NT>(acc, place, mw, nw, lane, smem)
// acc[i][j][q] is C(m0 + mw + 16 i + (lane & 15), n0 + nw + 16 j + 4 (lane >> 4) + q); mw and nw
// are the wave's first row and column in the tile, of WN waves a row.  All threads of the workgroup
// come, LDS is free.
template <typename T, bool TRA, bool TRB, int SIDE, class EPI>
__global__ __launch_bounds__(kProductThreads, SIDE == kMiddleRows ? 2 : 3) void mt_product(
    Product p, EPI epi) {
  constexpr int kThr = kProductThreads, MT = SIDE / 32, NT = SIDE / 32;
  constexpr int kSlot = 2 * SIDE * kRowBytes, SLOTS = kSlots<SIDE>;
  __shared__ __attribute__((aligned(1024))) char smem[kProductLds<SIDE>];
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wm = wave >> 1, wn = wave & 1;
  Place at;
  if (!place_of<SIDE>(p, &at)) return;

  using FeedA = Feed<T, TRA, SIDE, kThr>;
  using FeedB = Feed<T, TRB, SIDE, kThr>;
  constexpr int kBK = FeedA::kBK, kLoads = FeedA::kLoads + FeedB::kLoads;
  const int32_t k0 = at.split * p.part;
  const int32_t k_end = k0 + p.part < p.k ? k0 + p.part : p.k;
  const int32_t each = k_end > k0 ? (k_end - k0 + kBK - 1) / kBK : 0;  // stages of a term
  const int32_t stages = each * p.terms;
  FeedA fa;
  FeedB fb;
  fa.begin(p.a, at.pair, at.m0, k0, k_end, tid);
  fb.begin(p.b, at.pair, at.n0, k0, k_end, tid);
  const uint32_t lds = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem)) +
      wave * (kWave * 16);
  int32_t in_term = 0, term = 0;
  const auto load = [&](int slot) {
    fa.load(lds + slot * kSlot);
    fb.load(lds + slot * kSlot + SIDE * kRowBytes);
    if (++in_term == each) {
      in_term = 0;
      fa.turn(term == 0 ? p.a.next[0] : p.a.next[1], each);
      fb.turn(term == 0 ? p.b.next[0] : p.b.next[1], each);
      ++term;
    }
  };

  AccOf<T> acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = AccOf<T>{0, 0, 0, 0};

  if (stages > 0) load(0);
  if (SLOTS > 2 && stages > 1) load(1);
  int slot = 0;
  for (int32_t h = 0; h < stages; ++h) {
    if (SLOTS > 2 && h + 1 < stages) meet_loaded<kLoads>();
    else meet_loaded<0>();
    if (h + SLOTS - 1 < stages) load(slot == 0 ? SLOTS - 1 : slot - 1);
    const char* const sa = smem + slot * kSlot;
    const char* const sb = sa + SIDE * kRowBytes;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Frag ra[MT], rb[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i)
        ra[i] = fragment_any<T, TRA, SIDE>(sa, wm * (SIDE / 2) + i * 16, s, lane);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        rb[j] = fragment_any<T, TRB, SIDE>(sb, wn * (SIDE / 2) + j * 16, s, lane);
#pragma unroll
      for (int q = 0; q < kParts<T>; ++q)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = multiply_any<T>(rb[j], ra[i], acc[i][j], q);
    }
    slot = slot + 1 == SLOTS ? 0 : slot + 1;
  }
  meet_read();
  epi.template tile<SIDE, 2, MT, NT>(acc, at, wm * (SIDE / 2), wn * (SIDE / 2), lane, smem);
}

template <typename T, bool TRA, bool TRB, int SIDE, class EPI>
void run_product(Product p, const EPI& epi, hipStream_t st) {
  p.tiles_m = tiles_of(p.a.rows, SIDE);
  p.tiles_n = tiles_of(p.b.rows, SIDE);
  const int64_t grid = grid_of<SIDE>(p);
  if (grid > 0)
    mt_product<T, TRA, TRB, SIDE, EPI>
        <<<static_cast<uint32_t>(grid), kProductThreads, 0, st>>>(p, epi);
}

}  // namespace
}  // namespace gsn
