// The experts' products: the pairs' order by expert, buffers, and the C entry points.
#include "experts.h"

#include <algorithm>

namespace gsn {
namespace {

constexpr int kPlanThreads = 256;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanChunk = 1024;  // pairs of a workgroup, a quarter of them a wave
constexpr int kPlanEach = kPlanExperts / kPlanThreads;

int32_t plan_chunks(int64_t pairs) {
  return static_cast<int32_t>(pairs > 0 ? (pairs + kPlanChunk - 1) / kPlanChunk : 1);
}

// A stable counting sort of the pairs by expert: a first launch counts every chunk's pairs of each
// expert, a second one adds up what comes before a chunk and places its pairs.  32,764 pairs of
// 64 experts: 12 us in all, 31 us in one launch in which a workgroup an expert reads all ids twice.
// Every workgroup reads the counts of all chunks, so the second launch's time grows with the square
// of their number and with the experts: 2^20 pairs of 64 and of 1,024 experts 31 and 295 us, 2^22
// 0.25 and 3.6 ms, 2^24 3.5 and 114 ms, which is then most of the call.
// The pairs of a single chunk are counted where they are placed, without the first launch.
__global__ __launch_bounds__(kPlanThreads) void ex_count(int32_t pairs, int32_t experts,
                                                         const int32_t* __restrict__ ids,
                                                         int32_t* __restrict__ counts) {
  __shared__ int32_t count[kPlanExperts];
  for (int e = threadIdx.x; e < experts; e += kPlanThreads) count[e] = 0;
  __syncthreads();
  const int32_t i0 = blockIdx.x * kPlanChunk;
#pragma unroll
  for (int k = 0; k < kPlanChunk; k += kPlanThreads) {
    const int32_t i = i0 + k + threadIdx.x;
    const int32_t id = i < pairs ? ids[i] : -1;
    if (id >= 0 && id < experts) atomicAdd(&count[id], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += kPlanThreads)
    counts[static_cast<int64_t>(blockIdx.x) * experts + e] = count[e];
}

__global__ __launch_bounds__(kPlanThreads) void ex_place(int32_t pairs, int32_t experts,
                                                         int32_t top,
                                                         const int32_t* __restrict__ ids,
                                                         const int32_t* __restrict__ counts,
                                                         Plan plan) {
  __shared__ int32_t total[kPlanExperts], before[kPlanExperts];
  __shared__ int32_t next[kPlanWaves][kPlanExperts];  // a wave's next row of an expert
  __shared__ int32_t sums[3][kPlanWaves];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int32_t chunks = gridDim.x, chunk = blockIdx.x;
  for (int e = tid; e < experts; e += kPlanThreads) {
    total[e] = before[e] = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) next[w][e] = 0;
  }
  __syncthreads();
  // of every expert, the pairs of all chunks and of those before this one; and this chunk's by wave
  int span = 1;
  while (span < experts && span < kPlanThreads) span *= 2;
  for (int e = tid % span; chunks > 1 && e < experts; e += span) {
    int32_t all = 0, less = 0;
#pragma unroll 8
    for (int32_t c = tid / span; c < chunks; c += kPlanThreads / span) {
      const int32_t v = counts[static_cast<int64_t>(c) * experts + e];
      all += v;
      less += c < chunk ? v : 0;
    }
    if (all != 0) atomicAdd(&total[e], all);
    if (less != 0) atomicAdd(&before[e], less);
  }
  const int32_t i0 = chunk * kPlanChunk + wave * (kPlanChunk / kPlanWaves) + lane;
  int32_t id[kPlanChunk / kPlanThreads];
#pragma unroll
  for (int k = 0; k < kPlanChunk / kPlanThreads; ++k) {
    const int32_t i = i0 + k * kWave;
    id[k] = i < pairs ? ids[i] : -1;
    if (id[k] < 0 || id[k] >= experts) {
      if (i < pairs) plan.pos[i] = -1;
      id[k] = -1;
    } else {
      atomicAdd(&next[wave][id[k]], 1);
      if (chunks == 1) atomicAdd(&total[id[k]], 1);
    }
  }
  __syncthreads();
  // first rows and blocks of the experts, kPlanEach experts a thread
  const auto blocks = [](int32_t c, int32_t rows) { return (c + rows - 1) / rows; };
  int32_t mine[3] = {0, 0, 0}, first[3];  // rows, blocks, small blocks
#pragma unroll
  for (int k = 0; k < kPlanEach; ++k) {
    const int e = tid * kPlanEach + k;
    const int32_t c = e < experts ? total[e] : 0;
    mine[0] += c;
    mine[1] += blocks(c, kPlanRows);
    mine[2] += blocks(c, kSmallRows);
  }
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    first[q] = mine[q];
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int32_t v = __shfl_up(first[q], o);
      if (lane >= o) first[q] += v;
    }
    if (lane == kWave - 1) sums[q][wave] = first[q];
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    for (int w = 0; w < wave; ++w) first[q] += sums[q][w];
    first[q] -= mine[q];
  }
#pragma unroll
  for (int k = 0; k < kPlanEach; ++k) {
    const int e = tid * kPlanEach + k;
    if (e >= experts) break;
    const int32_t c = total[e], rows = first[0];
    const int32_t large = blocks(c, kPlanRows), small = blocks(c, kSmallRows);
    int32_t at = rows + before[e];
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
      const int32_t n = next[w][e];
      next[w][e] = at;
      at += n;
    }
    if (chunk == 0) {
      plan.offsets[e] = rows;
      if (e == experts - 1) {
        plan.offsets[experts] = rows + c;
        plan.tile_count[0] = first[1] + large;
        plan.tile_count[1] = first[2] + small;
      }
    }
    // (each chunk lists a part of the blocks)
    for (int32_t b = chunk; b < large; b += chunks)
      plan.tiles[first[1] + b] = int4{e, rows, first[1], large};
    for (int32_t b = chunk; b < small; b += chunks) {
      const int32_t r = b * kSmallRows;
      plan.small[first[2] + b] = int4{e, rows + r, c - r < kSmallRows ? c - r : kSmallRows, 0};
    }
    first[0] += c;
    first[1] += large;
    first[2] += small;
  }
  __syncthreads();
  // a wave's pairs in their order: the lanes that hold the same expert are found bit by bit
#pragma unroll
  for (int k = 0; k < kPlanChunk / kPlanThreads; ++k) {
    uint64_t same = __ballot(id[k] >= 0);
    for (int bit = 1; bit < experts; bit <<= 1) {
      const uint64_t m = __ballot((id[k] & bit) != 0);
      same &= (id[k] & bit) ? m : ~m;
    }
    if (id[k] >= 0) {
      const int32_t i = i0 + k * kWave;
      const int32_t r = next[wave][id[k]] + __popcll(same & ((uint64_t{1} << lane) - 1));
      plan.rows[r] = i;
      plan.token[r] = i / top;
      plan.pos[i] = r;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    if (id[k] >= 0 && (same >> lane) == 1)  // the last of them
      next[wave][id[k]] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
  }
}

constexpr size_t up(size_t n) { return (n + 255) / 256 * 256; }

struct Carver {
  char* base;
  size_t used = 0;
  void* take(size_t n) {
    void* p = base ? base + used : nullptr;
    used += up(n);
    return p;
  }
};

void carve_plan(Carver* c, Experts* x) {
  const size_t n = static_cast<size_t>(x->pairs);
  Plan& p = x->plan;
  const int64_t cut = x->pairs < x->experts ? x->pairs : x->experts;
  p.most_tiles = static_cast<int32_t>(x->pairs / kPlanRows + cut);
  p.most_small = static_cast<int32_t>(x->pairs / kSmallRows + cut);
  p.offsets = static_cast<int32_t*>(c->take(4 * (static_cast<size_t>(x->experts) + 1)));
  p.tile_count = static_cast<int32_t*>(c->take(8));
  p.tiles = static_cast<int4*>(c->take(16 * static_cast<size_t>(p.most_tiles)));
  p.small = static_cast<int4*>(c->take(16 * static_cast<size_t>(p.most_small)));
  p.rows = static_cast<int32_t*>(c->take(4 * n));
  p.token = static_cast<int32_t*>(c->take(4 * n));
  p.pos = static_cast<int32_t*>(c->take(4 * n));
  p.counts = static_cast<int32_t*>(
      c->take(4 * static_cast<size_t>(plan_chunks(x->pairs)) * x->experts));
}

// what the forward pass leaves for the backward pass
size_t carve_saved(void* base, Experts* x) {
  Carver c{static_cast<char*>(base)};
  carve_plan(&c, x);
  x->pre = static_cast<float*>(
      c.take(8 * static_cast<size_t>(x->pairs) * static_cast<size_t>(x->hidden)));
  return c.used;
}

size_t carve_forward(void* base, int32_t dtype, bool saved, Experts* x) {
  const size_t n = static_cast<size_t>(x->pairs);
  Carver c{static_cast<char*>(base)};
  if (!saved) carve_plan(&c, x);
  x->act = c.take(size_of(dtype) * n * x->hidden);
  x->y = static_cast<float*>(c.take(4 * n * x->dim));
  return c.used;
}

size_t carve_backward(void* base, int32_t dtype, Experts* x) {
  const size_t n = static_cast<size_t>(x->pairs), s = size_of(dtype);
  Carver c{static_cast<char*>(base)};
  x->dot_tiles = (x->hidden + kSmallRows - 1) / kSmallRows;
  x->dpre = c.take(2 * s * n * x->hidden);
  x->wact = c.take(s * n * x->hidden);
  x->dots = static_cast<float*>(c.take(4 * n * x->dot_tiles));
  x->dxr = static_cast<float*>(c.take(4 * n * x->dim));
  return c.used;
}

bool params_ok(const gsn_experts_params* p) {
  if (!p || p->dtype < GSN_F32 || p->dtype > GSN_F16 || p->tokens < 0 || p->experts < 1 ||
      p->experts > kPlanExperts || p->top < 1 || p->top > 64 || p->dim < 1 || p->hidden < 1 ||
      p->dim > (1 << 20) || p->hidden > (1 << 20))
    return false;
  // pairs, and workgroups of a product's grid, are counted in 31 bits; a grid has less than
  // 2^32 threads
  return p->tokens <= (int64_t{1} << 23) && p->tokens * p->top <= (int64_t{1} << 26);
}

Experts experts_of(const gsn_experts_params& p) {
  Experts x{};
  x.tokens = p.tokens;
  x.experts = p.experts;
  x.top = p.top;
  x.dim = p.dim;
  x.hidden = p.hidden;
  x.pairs = p.tokens * p.top;
  return x;
}

int32_t side_of(const Experts& x, int32_t dtype) {
  const bool aligned = x.x_stride % 8 == 0 && aligned16(x.x) && aligned16(x.w1) &&
                       aligned16(x.w2) && aligned16(x.out) && aligned16(x.dout) &&
                       aligned16(x.dx) && aligned16(x.dw1) && aligned16(x.dw2);
  return tile_side(dtype == GSN_F32, x.pairs, x.experts, x.dim, x.hidden, aligned);
}

// Whether the grids of a call's products stay below 2^32 threads: of the backward pass one for the
// gates' gradients and one for what is wanted of the others.
bool grids_ok(const Experts& x, bool backward) {
  const int64_t threads = x.side == kTileRows ? 512 : 256;
  const auto in = [&](Kind kind) { return product_blocks(kind, x); };
  const int64_t most =
      backward ? std::max(in(kBackwardGate), (x.dx ? in(kBackwardIn) : 0) +
                                                 (x.dw1 ? in(kWeightsIn) : 0) +
                                                 (x.dw2 ? in(kWeightsOut) : 0) +
                                                 (x.dweights ? x.pairs / threads + 1 : 0))
               : std::max(in(kForwardGate), in(kForwardOut));
  return most < (int64_t{1} << 32) / threads;
}

// Weights beyond the addresses of a process are no weights.
bool weights_ok(const gsn_experts_params& p) {
  const int64_t bytes = p.experts * static_cast<int64_t>(size_of(p.dtype));
  return int64_t{2} * p.hidden * p.dim <= (int64_t{1} << 47) / bytes;
}

bool workspace_ok(const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 256 == 0; }

}  // namespace

hipError_t launch_plan(const Experts& x, hipStream_t st) {
  const int32_t pairs = static_cast<int32_t>(x.pairs);
  const uint32_t chunks = static_cast<uint32_t>(plan_chunks(x.pairs));
  if (chunks > 1)
    ex_count<<<chunks, kPlanThreads, 0, st>>>(pairs, x.experts, x.ids, x.plan.counts);
  ex_place<<<chunks, kPlanThreads, 0, st>>>(pairs, x.experts, x.top, x.ids, x.plan.counts,
                                            x.plan);
  return hipGetLastError();
}

extern template hipError_t launch_experts<float>(const Experts&, hipStream_t);
extern template hipError_t launch_experts<bf16_t>(const Experts&, hipStream_t);
extern template hipError_t launch_experts<f16_t>(const Experts&, hipStream_t);
extern template hipError_t launch_experts_backward<float>(const Experts&, hipStream_t);
extern template hipError_t launch_experts_backward<bf16_t>(const Experts&, hipStream_t);
extern template hipError_t launch_experts_backward<f16_t>(const Experts&, hipStream_t);

}  // namespace gsn

extern "C" {

size_t gsn_experts_workspace_bytes(const gsn_experts_params* p, int32_t backward) {
  if (!gsn::params_ok(p)) return 0;
  gsn::Experts x = gsn::experts_of(*p);
  return (backward ? gsn::carve_backward(nullptr, p->dtype, &x)
                   : gsn::carve_forward(nullptr, p->dtype, false, &x)) + 256;
}

size_t gsn_experts_saved_bytes(const gsn_experts_params* p) {
  if (!gsn::params_ok(p)) return 0;
  gsn::Experts x = gsn::experts_of(*p);
  return gsn::carve_saved(nullptr, &x);
}

int gsn_experts(const gsn_experts_params* p, const void* x, int64_t x_stride,
                const int32_t* ids, const float* weights, const void* w1, const void* w2,
                void* out, void* saved, size_t saved_bytes, void* workspace,
                size_t workspace_bytes, void* stream) {
  if (!gsn::params_ok(p)) return GSN_E_INVAL;
  gsn::Experts a = gsn::experts_of(*p);
  if (a.tokens == 0 && !saved) return GSN_OK;
  if (!gsn::workspace_ok(workspace) || (saved && !gsn::workspace_ok(saved))) return GSN_E_INVAL;
  if (a.tokens > 0 && (!x || !ids || !weights || !w1 || !w2 || !out || x_stride < p->dim))
    return GSN_E_INVAL;
  if (workspace_bytes < gsn_experts_workspace_bytes(p, 0) ||
      (saved && saved_bytes < gsn_experts_saved_bytes(p)))
    return GSN_E_CAPACITY;
  a.x = x;
  a.x_stride = x_stride;
  a.ids = ids;
  a.weights = weights;
  a.w1 = w1;
  a.w2 = w2;
  a.out = out;
  a.side = gsn::side_of(a, p->dtype);
  if (saved) gsn::carve_saved(saved, &a);
  gsn::carve_forward(workspace, p->dtype, saved != nullptr, &a);
  if (!gsn::weights_ok(*p) || !gsn::grids_ok(a, false)) return GSN_E_CAPACITY;
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (a.tokens == 0) e = gsn::launch_plan(a, st);
  else if (p->dtype == GSN_F32) e = gsn::launch_experts<float>(a, st);
  else if (p->dtype == GSN_BF16) e = gsn::launch_experts<gsn::bf16_t>(a, st);
  else e = gsn::launch_experts<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

int gsn_experts_backward(const gsn_experts_params* p, const void* dout, const void* x,
                         int64_t x_stride, const float* weights, const void* w1, const void* w2,
                         const void* saved, size_t saved_bytes, void* dx, float* dweights,
                         void* dw1, void* dw2, void* workspace, size_t workspace_bytes,
                         void* stream) {
  if (!gsn::params_ok(p)) return GSN_E_INVAL;
  gsn::Experts a = gsn::experts_of(*p);
  if (!gsn::workspace_ok(workspace) || !gsn::workspace_ok(saved)) return GSN_E_INVAL;
  if (a.tokens > 0 && (!dout || !x || !weights || !w1 || !w2 || x_stride < p->dim))
    return GSN_E_INVAL;
  if (workspace_bytes < gsn_experts_workspace_bytes(p, 1) ||
      saved_bytes < gsn_experts_saved_bytes(p))
    return GSN_E_CAPACITY;
  a.dout = dout;
  a.x = x;
  a.x_stride = x_stride;
  a.weights = weights;
  a.w1 = w1;
  a.w2 = w2;
  a.dx = dx;
  a.dweights = dweights;
  a.dw1 = dw1;
  a.dw2 = dw2;
  a.side = gsn::side_of(a, p->dtype);
  gsn::carve_saved(const_cast<void*>(saved), &a);
  gsn::carve_backward(workspace, p->dtype, &a);
  if (!gsn::weights_ok(*p) || !gsn::grids_ok(a, true)) return GSN_E_CAPACITY;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = p->dtype == GSN_F32 ? gsn::launch_experts_backward<float>(a, st)
                       : p->dtype == GSN_BF16
                           ? gsn::launch_experts_backward<gsn::bf16_t>(a, st)
                           : gsn::launch_experts_backward<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

}  // extern "C"
