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
  // An XCD takes an eighth of all tiles, not runs of them in turn.  With many pairs, each stays
  // with one XCD: 64 pairs, 2,048 x 1,024 by 1,024 x 1,024 of float16, 310 us in eighths and 342 in
  // runs; 4 pairs, 2,048 x 4,096 by its transposed self, three products, 315 and 356; 7 of 666 x
  // 501, 20 and 27.  One pair with few rows and very many columns: 8,192 x 131,072 x 2,048, nothing
  // written, 4.0 and 4.3 ms; but with its results written (tiles of 128) a piece of 32,768 columns
  // took 1.23 and 1.18, and 8,192 x 2,048 x 32,768 1.10 and 0.96.
  int32_t eighths;
  int32_t symmetric;  // C = C^T: tiles with n0 >= m0 alone
};

// A tile: its pair of the batch, its first row and column, its part of k.
struct Place {
  int32_t pair, m0, n0, split;
};

inline int32_t tiles_of(int64_t n, int32_t side) {
  return static_cast<int32_t>((n + side - 1) / side);
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

// Tiles of BM x BN by four waves, 2 x 2 of them: stages of 128 bytes of k, SLOTS of them in LDS,
// and WAVES of a SIMD that registers and LDS have to last for.  RUN of them at a time are an XCD's,
// in blocks TALL tiles high.  GROUPS of four waves take a part of the stages each, with SLOTS of
// their own, and add their sums up in the groups' order.
template <int BM_, int BN_, int SLOTS_, int WAVES_, int RUN_, int TALL_, int GROUPS_ = 1>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, SLOTS = SLOTS_, WAVES = WAVES_;
  static constexpr int RUN = RUN_, TALL = TALL_, GROUPS = GROUPS_;
  static constexpr int kSlot = (BM + BN) * kRowBytes;
  static constexpr int kLds = SLOTS * kSlot;  // of a group
  static constexpr int kThreads = 256 * GROUPS;
  static_assert(BN % BM == 0 && kLds * WAVES <= 160 * 1024 && WAVES % GROUPS == 0);
};

// Fragment of 16 rows at r0 and the s-th half of a stage's k; R rows, or columns, in all.  (8-bit
// elements lie as the bytes of wider ones do.)
template <typename T, bool TR, int R>
__device__ __forceinline__ Frag fragment_any(const char* tile, int r0, int s, int lane) {
  if constexpr (sizeof(T) == 1) {
    static_assert(!TR);
    return fragment<float, false, R>(tile, r0, s, lane);
  } else {
    return fragment<T, TR, R>(tile, r0, s, lane);
  }
}

// v as a binary32 value: what is made of it is made of the same one.  (Left to the compiler, a
// product may be fused with its rounding to float16, and a second value that is made of the product
// as rounded to binary32 does not belong to the first where that is a tie.)
__device__ __forceinline__ float settled(float v) {
  asm("" : "+v"(v));
  return v;
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
  // from the first stage of all to stage `in_term` of a later term
  __device__ __forceinline__ void skip(int64_t next0, int64_t next1, int32_t in_term) {
    p += next0 + next1 + in_term * step;
    k += in_term * kBK;
  }
  // to the next term after `stages` stages
  __device__ __forceinline__ void turn(int64_t next, int32_t stages) {
    p += next - stages * step;
    k -= stages * kBK;
  }
};

// Number of a tile in its pair -> its row and column of tiles, of a symmetric product those that
// hold something on or above the diagonal, a column of tiles after the other.
template <class TILE>
__device__ __forceinline__ int2 symmetric_place(int32_t id, int32_t tiles_m) {
  constexpr int32_t R = TILE::BN / TILE::BM;  // column c has the tiles 0 .. R (c + 1) - 1
  const float f = sqrtf(8.0f / R * static_cast<float>(id) + 1.0f);
  int32_t c = static_cast<int32_t>((f - 1.0f) * 0.5f);
  while (R * c * (c + 1) / 2 > id) --c;
  while (R * (c + 1) * (c + 2) / 2 <= id) ++c;
  return int2{id - R * c * (c + 1) / 2, c};
}

// Tiles of a pair.  (The last column of a symmetric product may have fewer tiles than R (c + 1):
// its number of rows.)
template <class TILE>
__host__ __device__ inline int32_t tiles_of_pair(const Product& p) {
  constexpr int32_t R = TILE::BN / TILE::BM;
  return p.symmetric ? R * (p.tiles_n - 1) * p.tiles_n / 2 + p.tiles_m : p.tiles_m * p.tiles_n;
}

// Workgroups of a product: those of a round of 8 runs are dealt out to the XCDs a run each
// (spread()), where the tiles that are worked on at a time share operands.
template <class TILE>
__host__ __device__ inline int32_t numbers_of(const Product& p) {
  constexpr int32_t round = 8 * TILE::RUN;
  const int32_t tiles = tiles_of_pair<TILE>(p) * p.batch * p.splits;
  return p.eighths || tiles < round ? (tiles + 7) / 8 * 8 : (tiles + round - 1) / round * round;
}

// false: there is no tile of this number.
template <class TILE>
__device__ __forceinline__ bool place_of(const Product& p, int32_t number, Place* at) {
  const int32_t each = tiles_of_pair<TILE>(p);
  const int32_t all = each * p.batch * p.splits;
  const int32_t id = spread(number, all, p.eighths ? (all + 7) / 8 : TILE::RUN);
  if (id < 0) return false;
  const int32_t outer = id / each, in = id - outer * each;
  const int2 t = p.symmetric ? symmetric_place<TILE>(in, p.tiles_m)
                             : tile_place<TILE::TALL>(in, p.tiles_m, p.tiles_n);
  at->split = outer / p.batch;
  at->pair = outer - at->split * p.batch;
  at->m0 = t.x * TILE::BM;
  at->n0 = t.y * TILE::BN;
  return true;
}

constexpr int kProductThreads = 256;

// A tile by four waves.  Stages go from memory straight to LDS; a stage is awaited by all waves
// together, then a later one is sent out (with one place, after this one is multiplied) and this
// one multiplied.  Two or three workgroups share a CU: one's waits, start and results hide behind
// another's products.
//
// 8,192 tokens, 131,072 classes of 2,048, bfloat16: logits at 1.10 PFLOP/s, the gradients' products
// at 1.13 (a large library product: 1.31); 8,191 through 4,096 x 8,192 in 8 bits 2.09 POP/s (2.12).
// There the matrix cores are busy for half of the cycles and LDS for a fifth: what is left is the
// wait for loads.  A k of a few stages pays for its start and results: 1,024 in float16 0.83.
//
// What becomes of the results is the functor's:
//   EPI::tile<TILE, MT, NT>(acc, place, mw, nw, lane, room)
// and, where there is a bool EPI::wanted() that is false, nothing: the product is not made.
// acc[i][j][q] is C(m0 + mw + 16 i + (lane & 15), n0 + nw + 16 j + 4 (lane >> 4) + q); mw and nw
// are the wave's first row and column in the tile.  All threads of the workgroup come; room is LDS
// that no other wave reads any more.
template <class EPI>
__device__ __forceinline__ auto wanted(const EPI& epi, int) -> decltype(epi.wanted()) {
  return epi.wanted();
}
template <class EPI>
__device__ __forceinline__ bool wanted(const EPI&, int64_t) {
  return true;
}

template <typename T, bool TRA, bool TRB, class TILE, class EPI>
__global__ __launch_bounds__(TILE::kThreads, TILE::WAVES) void mt_product(Product p, EPI epi) {
  constexpr int kThr = kProductThreads, BM = TILE::BM, BN = TILE::BN;
  constexpr int MT = BM / 32, NT = BN / 32, kSlot = TILE::kSlot, SLOTS = TILE::SLOTS;
  static_assert(SLOTS >= 1 && SLOTS <= 3);
  constexpr int GROUPS = TILE::GROUPS;
  __shared__ __attribute__((aligned(1024))) char lds_all[GROUPS * TILE::kLds];
  const int group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThr);
  char* const smem = lds_all + group * TILE::kLds;
  const int tid = threadIdx.x - group * kThr, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int mw = (wave >> 1) * (BM / 2), nw = (wave & 1) * (BN / 2);
  if (!wanted(epi, 0)) return;
  Place at;
  if (!place_of<TILE>(p, blockIdx.x, &at)) return;

  using FeedA = Feed<T, TRA, BM, kThr>;
  using FeedB = Feed<T, TRB, BN, kThr>;
  constexpr int kBK = FeedA::kBK, kLoads = FeedA::kLoads + FeedB::kLoads;
  const int32_t k0 = at.split * p.part;
  const int32_t k_end = k0 + p.part < p.k ? k0 + p.part : p.k;
  const int32_t each = k_end > k0 ? (k_end - k0 + kBK - 1) / kBK : 0;  // stages of a term
  const int32_t all = each * p.terms;
  // this group's: `most` of them or what is left
  const int32_t most = (all + GROUPS - 1) / GROUPS;
  const int32_t before = group * most < all ? group * most : all;
  const int32_t stages = all - before < most ? all - before : most;
  FeedA fa;
  FeedB fb;
  fa.begin(p.a, at.pair, at.m0, k0, k_end, tid);
  fb.begin(p.b, at.pair, at.n0, k0, k_end, tid);
  const uint32_t lds = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem)) +
      wave * (kWave * 16);
  int32_t in_term = 0, term = 0;
  if constexpr (GROUPS > 1) {
    if (each > 0) term = before / each;
    in_term = before - term * each;
    fa.skip(term > 0 ? p.a.next[0] : 0, term > 1 ? p.a.next[1] : 0, in_term);
    fb.skip(term > 0 ? p.b.next[0] : 0, term > 1 ? p.b.next[1] : 0, in_term);
  }
  const auto load = [&](int slot) {
    fa.load(lds + slot * kSlot);
    fb.load(lds + slot * kSlot + BM * kRowBytes);
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
  for (int32_t h = 0; h < most; ++h) {
    if constexpr (SLOTS == 1) {
      // (the other workgroups of the CU multiply while this one's stage is on its way)
      if (h > 0) {
        meet_read();
        if (h < stages) load(0);
      }
      meet_loaded<0>();
      if (GROUPS > 1 && h >= stages) continue;
    } else {
      if (SLOTS > 2 && h + 1 < stages) meet_loaded<kLoads>();
      else meet_loaded<0>();
      if (GROUPS > 1 && h >= stages) continue;
      if (h + SLOTS - 1 < stages) load(slot == 0 ? SLOTS - 1 : slot - 1);
    }
    const char* const sa = smem + slot * kSlot;
    const char* const sb = sa + BM * kRowBytes;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Frag ra[MT], rb[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) rb[j] = fragment_any<T, TRB, BN>(sb, nw + j * 16, s, lane);
#pragma unroll
      for (int i = 0; i < MT; ++i) ra[i] = fragment_any<T, TRA, BM>(sa, mw + i * 16, s, lane);
#pragma unroll
      for (int q = 0; q < kParts<T>; ++q)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = multiply_any<T>(rb[j], ra[i], acc[i][j], q);
    }
    if constexpr (SLOTS > 1) slot = slot + 1 == SLOTS ? 0 : slot + 1;
  }
  meet_read();
  if constexpr (GROUPS > 1) {
    constexpr int kSums = kThr * MT * NT * 16;
    static_assert(kSums <= TILE::kLds);
    auto* const sums = reinterpret_cast<AccOf<T>*>(smem);
    if (group > 0)
#pragma unroll
      for (int i = 0; i < MT * NT; ++i) sums[i * kThr + tid] = acc[i / NT][i % NT];
    meet_read();
    if (group > 0) return;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g)
#pragma unroll
      for (int i = 0; i < MT * NT; ++i)
        acc[i / NT][i % NT] +=
            *reinterpret_cast<const AccOf<T>*>(smem + g * TILE::kLds + (i * kThr + tid) * 16);
  }
  epi.template tile<TILE, MT, NT>(acc, at, mw, nw, lane, smem);
}

template <typename T, bool TRA, bool TRB, class TILE, class EPI>
void run_tiles(Product p, const EPI& epi, hipStream_t st) {
  p.tiles_m = tiles_of(p.a.rows, TILE::BM);
  p.tiles_n = tiles_of(p.b.rows, TILE::BN);
  const int32_t grid = numbers_of<TILE>(p);
  if (grid > 0)
    mt_product<T, TRA, TRB, TILE, EPI>
        <<<static_cast<uint32_t>(grid), TILE::kThreads, 0, st>>>(p, epi);
}

// Which tiles a product takes.  Of 2-byte elements, us, C of bfloat16, tiles of 128 x 256, 128 x
// 128 and 64 x 64 (two workgroups a CU of the first two, three of the last):
//   k contiguous: 8,192 x 4,096 x 1,024: 75, 84, 118; 4,096 x 4,096 (512 tiles of 128 x 256): 39,
//     44, 62; 4,096 x 2,048: 29, 24, 31; 2,048 x 2,048 (256 of 128): 24, 16, 20; 1,536 x 1,536: 24,
//     15, 13
//   n contiguous in B: 77, 87, 134; 41, 44, 67; 32, 24, 35; 25, 17, 20; 27, 16, 14
//   m and n contiguous: 76, 90, 134; 41, 46, 69; 33, 25, 34; 26, 17, 21; 28, 17, 15
//   8 bits, 4,096 x 4,096 x 4,096: 65, 76, 159
// The large tiles have one place for a stage: a workgroup waits for its loads while the other one
// multiplies, and the registers that a stage ahead would take and the half lines that two stages of
// half the size would read cost more (8,192 x 32,768 x 2,048, k contiguous: 1,007 us; 1,099 with
// three places for 64 bytes of k; tiles of 128 with two places for 128 bytes 1,130, with one 1,003;
// 8,192 x 2,048 x 32,768: 978, 957, 1,085, 1,161).  MFMAs of 32 x 32 in place of 16 x 16 were 8 to
// 12% slower.  The middle tiles have two places where all of them are on the CUs at a time, and
// one, in three workgroups a CU, where there are more (64 products of 1,024 x 1,024 x 2,048 of
// which half is made, 2,304 tiles: 212 and 196 us; 4,096 x 2,560 x 1,024, 640 tiles 34 and 33,
// 4,096 x 2,048, 512 tiles 24 and 24).  The CUs hold 512 of the large or of the middle tiles: the
// large ones are taken where their rounds, at 0.9 of the time for their size, are not the longer
// (1,777 x 10,007 x 1,512, 560 large tiles or 1,106: 484 and 408 us of a training step).
// Binary32 products are bound by the matrix cores, and small tiles fill the CUs more evenly.
// Up to about one workgroup a CU its SIMDs have a wave each, which waits for its own loads: two
// groups of waves share k.  With one group and two: tiles of 128: 2,048 x 2,048 x 2,048 (256) 28,
// 23; tiles of 64 from 8 stages on: 1,024 x 1,024 x 2,048 (256) 15, 12; 2,048 x 1,024 x 2,048 (512)
// 19, 16; 1,024 x 768 x 512 7.2, 7.2; 8 bits, 64 rows by 16,384 of 4,096 (256, memory) 14.6, 13.1.
using LargeTile = Tile<128, 256, 1, 2, 32, 8>;
using MiddleTile = Tile<128, 128, 2, 2, 16, 4>;
using MiddleMany = Tile<128, 128, 1, 3, 16, 4>;
using MiddleTwo = Tile<128, 128, 2, 2, 16, 4, 2>;
using SmallTile = Tile<64, 64, 3, 3, 1, 4>;
using SmallTwo = Tile<64, 64, 2, 4, 1, 4, 2>;      // two workgroups a CU
using SmallTwoAlone = Tile<64, 64, 3, 2, 1, 4, 2>;  // one
// Few rows: small tiles of which some are left after the 768 that the CUs take at a time; wider
// ones are one round (64 rows by 50,000 of 1,024, 782 tiles: 18 us and 22; by 49,152 19 and 18; by
// 100,000 40 and 35).
using FlatTile = Tile<64, 128, 2, 3, 1, 4>;

// f(a tile's type) for the tiles of a product.
template <typename T, bool TRA, bool TRB, class F>
void with_tile(const Product& p, const F& f) {
  const auto tiles = [&](int32_t bm, int32_t bn) {
    const int64_t m = tiles_of(p.a.rows, bm), n = tiles_of(p.b.rows, bn);
    return (p.symmetric && bm == bn ? n * (n + 1) / 2 : m * n) * p.batch * p.splits;
  };
  const int64_t middle = tiles(MiddleTile::BM, MiddleTile::BN);
  const int64_t bytes = int64_t{p.part} * p.terms * static_cast<int64_t>(sizeof(T));
  if constexpr (sizeof(T) < 4) {
    // (few rows: bound by reading the other operand, of which small tiles have more on its way: 64
    // rows by 16,384 of 4,096, 26 us and 43; of a symmetric product large tiles would hold more
    // that is below the diagonal)
    const bool few = p.a.rows <= SmallTile::BM;
    const int64_t large = tiles(LargeTile::BM, LargeTile::BN);
    const auto rounds = [](int64_t n) { return (n + 511) / 512; };
    if (!few && !p.symmetric && large >= 512 && 18 * rounds(large) <= 10 * rounds(middle))
      return f(LargeTile());
    if (!few && middle > 512) return f(MiddleMany());
    if (!few && middle > 256) return f(MiddleTile());
    if (!few && middle >= 144) return f(MiddleTwo());
  }
  const int64_t small = tiles(SmallTile::BM, SmallTile::BN);
  if (p.a.rows <= SmallTile::BM && small > 768 && small <= 1024 && sizeof(T) < 4)
    return f(FlatTile());
  if (bytes < 8 * kRowBytes || small > 512) return f(SmallTile());
  if (small <= 256) f(SmallTwoAlone());
  else f(SmallTwo());
}

template <typename T, bool TRA, bool TRB, class EPI>
void run_product(const Product& p, const EPI& epi, hipStream_t st) {
  with_tile<T, TRA, TRB>(p, [&](auto tile) { run_tiles<T, TRA, TRB, decltype(tile)>(p, epi, st); });
}

}  // namespace
}  // namespace gsn
