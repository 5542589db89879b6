// Matrix tiles: fragments and their products on the matrix cores, where operands are staged in LDS,
// loads to LDS and the waits for them, and which tile a workgroup takes.  Included by the sources
// of kernels that multiply matrices.
#pragma once

#include "mixture.h"

#pragma clang fp contract(fast)

namespace gsn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kRowBytes = 128;  // bytes of k (contiguous operands) in a stage

// 16 bytes of an operand in a lane: 8 or 4 values of k of row (lane & 15)
union Frag {
  u32x4 u;
  bf16x8 b;
  f16x8 h;
  f32x4 f;
  s16x4 s[2];
};

// acc[i] += sum over the fragment's k of n-row (lane >> 4) * 4 + i and m-row lane & 15; of a 4-byte
// type part q of four, so that products of one sum do not wait for each other.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 4 : 1;
template <typename T>
__device__ __forceinline__ f32x4 multiply(const Frag& n, const Frag& m, f32x4 acc, int q) {
  if constexpr (sizeof(T) == 4)
    return __builtin_amdgcn_mfma_f32_16x16x4f32(n.f[q], m.f[q], acc, 0, 0, 0);
  else if constexpr (__is_same(T, bf16_t))
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(n.b, m.b, acc, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(n.h, m.h, acc, 0, 0, 0);
}

// Place of 16-byte chunk c in row r of a staged operand with k contiguous (8 chunks a row): the
// 16 rows that a quarter wave reads at one k fall on different banks.
__device__ __forceinline__ int chunk_k(int r, int c) { return c ^ ((r >> 1) & 7); }
// The same with k as the row: the 4 (2-byte types) or 1 rows that 16 lanes read 32 or 64 bytes
// of, and those of the wave's other quarters, fall on different banks.
template <typename T, int CHUNKS = 16>  // CHUNKS of a row, at least
__device__ __forceinline__ int chunk_n(int k, int c) {
  if constexpr (sizeof(T) == 2 && CHUNKS < 16) return c ^ ((k & 3) << 1);
  else if constexpr (sizeof(T) == 2) return c ^ (((k & 3) | ((k >> 1) & 4)) << 1);
  else return c ^ (((k >> 2) & 3) << 2);
}

// Fragment of 16 rows at `r0` and the s-th half of a stage's k; R rows (k contiguous) or columns
// (k as the row) in all.
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
      const char* p = tile + (k * R + (chunk_n<T, R / 8>(k, col >> 3) << 3) + (col & 7)) * 2;
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

// Four results of a row at column n, N columns in all.  Rows start at any element.
template <typename T>
struct LooseOf {
  typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};
template <typename T>
__device__ __forceinline__ void store4(T* row, int32_t n, int32_t N, const float* v) {
  if (n + 4 <= N) {
    typename LooseOf<T>::type o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = from_float<T>(v[i]);
    *reinterpret_cast<typename LooseOf<T>::type*>(row + n) = o;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < N) row[n + i] = from_float<T>(v[i]);
}
template <typename T>
__device__ __forceinline__ void load4(const T* row, int32_t n, int32_t N, float* v) {
  if (n + 4 <= N) {
    const auto o = *reinterpret_cast<const typename LooseOf<T>::type*>(row + n);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_float(o[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = n + i < N ? to_float(row[n + i]) : 0.0f;
}

// 16 zero bytes that lanes load where an operand has no more k
__device__ __attribute__((aligned(16))) const uint32_t kZeros[4] = {0, 0, 0, 0};

// A lane's 16 bytes of a row of K elements at k, zeros past its end (INSIDE: there is none in
// them).  Rows start at any element.
template <bool INSIDE, typename T>
__device__ __forceinline__ Frag row_chunk(const T* row, int32_t k, int32_t K) {
  constexpr int kE = 16 / sizeof(T);
  typedef T Loose __attribute__((ext_vector_type(kE), aligned(sizeof(T))));
  Frag f;
  if (INSIDE || k + kE <= K) {
    // (said to be global: a pointer chosen between two is taken for any, whose loads LDS reads wait
    // for)
    f.u = __builtin_bit_cast(u32x4, *(const __attribute__((address_space(1))) Loose*)(row + k));
  } else {
    Vec<T, kE> v;
#pragma unroll
    for (int j = 0; j < kE; ++j) v.v[j] = k + j < K ? row[k + j] : from_float<T>(0.0f);
    f.u = __builtin_bit_cast(u32x4, v);
  }
  return f;
}

// Workgroups go round the 8 XCDs.  Runs of `run` tiles go to one XCD, where the tiles that its CUs
// work on at a time share operands through its L2; the next run goes to the next XCD.
// Fewer tiles than 8 runs are dealt out evenly.  -1: no tile for this workgroup (for any of them,
// where no pair has an expert and there are no tiles).
__device__ __forceinline__ int32_t spread(int32_t block, int32_t total, int32_t run) {
  if (total <= 0) return -1;
  if (total < 8 * run) run = (total + 7) / 8;
  const int32_t in = block >> 3;
  const int32_t id = (in / run * 8 + (block & 7)) * run + in % run;
  return id < total ? id : -1;
}
// Place of a tile in a block of tiles_m x tiles_n, taken TALL tiles of m by all of n at a time, m
// first: 32 tiles in a row, 4 x 8, have 4 + 8 tiles of operands.
template <int32_t TALL>
__device__ __forceinline__ int2 tile_place(int32_t id, int32_t tiles_m, int32_t tiles_n) {
  const int32_t g = id / (TALL * tiles_n), in = id - g * TALL * tiles_n;
  const int32_t left = tiles_m - g * TALL, tall = left < TALL ? left : TALL;
  return int2{g * TALL + in % tall, in / tall};
}
// 16 bytes a lane from its address to LDS offset `at` + 16 lane, without a register between.
// The compiler does not count these loads: meet() does (with the builtin of this load the
// compiler waits for all of them before every read of LDS, as it cannot tell the buffers apart).
// m0 is a reserved register, which asm cannot declare as written; no other instruction of these
// kernels reads it (tests/test_experts_assembly.py; putting its old value back after every load
// took up to 3% of a training step's time).
__device__ __forceinline__ void load_to_lds(const void* p, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(at), "v"(p)
               : "memory");
}
__device__ __forceinline__ void load_word_to_lds(const void* p, uint32_t at) {  // 4 bytes a lane
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(at), "v"(p)
               : "memory");
}
// Waits for the workgroup's other waves; before that until this wave's reads of LDS are done, or
// its loads too.  One block of asm each, so that no access of LDS comes between.
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }
__device__ __forceinline__ void meet_read() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
template <int LEFT>  // but for so many of the last loads
__device__ __forceinline__ void meet_loaded() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// Waits until at most LEFT of this wave's loads and stores are under way; until its reads of LDS
// are done.
template <int LEFT>
__device__ __forceinline__ void await_own() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void await_reads() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// What a wave's lanes wrote to LDS before it, they may read from each other after it.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// 16 rows of COLS results of a wave, turned round in its own LDS: a lane has four columns of one
// row, and 4 lanes of 64 share it, so stores from the lanes would go out in pieces of 32 or 64
// bytes; from here they go out in whole rows of 64 to 256 bytes.
template <typename U, int COLS>
struct Turn {
  static constexpr int kRow = COLS * static_cast<int>(sizeof(U)) + 16;  // (spreads the banks)
  static constexpr int kBytes = 16 * kRow;
  static constexpr int kW = 16 / static_cast<int>(sizeof(U));
  static constexpr int kLanes = COLS / kW;  // of a row
  static constexpr int kStores = 16 * kLanes / kWave;
  char* at;
  __device__ __forceinline__ void put(int row, int col, const float* v) const {
    Vec<U, 4> o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.v[i] = from_float<U>(v[i]);
    *reinterpret_cast<Vec<U, 4>*>(at + row * kRow + col * static_cast<int>(sizeof(U))) = o;
  }
  // rows `rows` of the 16, columns `cols` of a matrix with rows of ld elements
  __device__ __forceinline__ void out(U* to, int64_t ld, int32_t rows, int32_t cols,
                                      int lane) const {
#pragma unroll
    for (int i = 0; i < kStores; ++i) {
      const int row = i * (kWave / kLanes) + lane / kLanes, col = lane % kLanes * kW;
      const u32x4 v = *reinterpret_cast<const u32x4*>(at + row * kRow +
                                                      col * static_cast<int>(sizeof(U)));
      if (row < rows && col < cols) *reinterpret_cast<u32x4*>(to + row * ld + col) = v;
    }
  }
};

}  // namespace
}  // namespace gsn
