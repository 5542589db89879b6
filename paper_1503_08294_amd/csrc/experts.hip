// The experts' products: the pairs' order by expert, buffers, and the C entry points.
#include "experts.h"

#include <algorithm>

namespace gsn {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
static_assert(kPlanExperts <= kPlanThreads);

// One workgroup an expert.  Each reads all ids twice: for the pairs of every expert (where its
// own rows begin), then to place its own, each wave a stretch of the pairs in their order.  No
// workgroup waits for another, and the order is that of the pairs.
__global__ __launch_bounds__(kPlanThreads) void ex_plan(int32_t pairs, int32_t experts,
                                                        int32_t top,
                                                        const int32_t* __restrict__ ids,
                                                        Plan plan) {
  __shared__ int32_t count[kPlanExperts];
  __shared__ int32_t mine[kPlanWaves];
  __shared__ int2 sums[kPlanWaves];
  __shared__ int4 at;  // first row, rows, first tile of this expert
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int32_t e = blockIdx.x;
  if (tid < kPlanExperts) count[tid] = 0;
  __syncthreads();
  const int32_t per = ((pairs + kPlanWaves - 1) / kPlanWaves + kWave - 1) / kWave * kWave;
  const int64_t i0 = static_cast<int64_t>(per) * wave;
  const int64_t i1 = i0 + per < pairs ? i0 + per : pairs;
  int32_t found = 0;
  for (int64_t i = i0; i < i1; i += kWave) {
    const int32_t id = i + lane < i1 ? ids[i + lane] : -1;
    if (id >= 0 && id < experts) atomicAdd(&count[id], 1);
    else if (e == 0 && i + lane < i1) plan.pos[i + lane] = -1;
    found += __popcll(__ballot(id == e));
  }
  if (lane == 0) mine[wave] = found;
  __syncthreads();
  // rows and tiles before every expert
  const int32_t c = tid < experts ? count[tid] : 0;
  int32_t rows = c, tiles = (c + kPlanRows - 1) / kPlanRows;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int32_t r = __shfl_up(rows, o), t = __shfl_up(tiles, o);
    if (lane >= o) {
      rows += r;
      tiles += t;
    }
  }
  if (lane == kWave - 1) sums[wave] = int2{rows, tiles};
  __syncthreads();
  for (int w = 0; w < wave; ++w) {
    rows += sums[w].x;
    tiles += sums[w].y;
  }
  if (tid == e) at = int4{rows - c, c, tiles - (c + kPlanRows - 1) / kPlanRows, 0};
  if (e == 0) {
    if (tid < experts) plan.offsets[tid + 1] = rows;
    if (tid == 0) plan.offsets[0] = 0;
    if (tid == experts - 1) *plan.tile_count = tiles;
  }
  __syncthreads();
  const int4 a = at;
  for (int32_t k = tid; k * kPlanRows < a.y; k += kPlanThreads)
    plan.tiles[a.z + k] = int4{e, a.x, a.z, (a.y + kPlanRows - 1) / kPlanRows};
  int32_t r = a.x;
  for (int w = 0; w < wave; ++w) r += mine[w];
  for (int64_t i = i0; i < i1; i += kWave) {
    const bool hit = i + lane < i1 && ids[i + lane] == e;
    const uint64_t m = __ballot(hit);
    if (hit) {
      const int32_t at_row = r + __popcll(m & ((uint64_t{1} << lane) - 1));
      plan.rows[at_row] = static_cast<int32_t>(i + lane);
      plan.token[at_row] = static_cast<int32_t>(i + lane) / top;
      plan.pos[i + lane] = at_row;
    }
    r += __popcll(m);
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
  p.most_tiles = static_cast<int32_t>(
      x->pairs / kPlanRows + (x->pairs < x->experts ? x->pairs : x->experts));
  p.offsets = static_cast<int32_t*>(c->take(4 * (static_cast<size_t>(x->experts) + 1)));
  p.tile_count = static_cast<int32_t*>(c->take(4));
  p.tiles = static_cast<int4*>(c->take(16 * static_cast<size_t>(p.most_tiles)));
  p.rows = static_cast<int32_t*>(c->take(4 * n));
  p.token = static_cast<int32_t*>(c->take(4 * n));
  p.pos = static_cast<int32_t*>(c->take(4 * n));
}

// what the forward pass leaves for the backward pass
size_t carve_saved(void* base, Experts* x) {
  Carver c{static_cast<char*>(base)};
  carve_plan(&c, x);
  x->pre = static_cast<float*>(
      c.take(8 * static_cast<size_t>(x->pairs) * static_cast<size_t>(x->hidden)));
  return c.used;
}

// (rows past the last one may be read, for results that are not stored)
size_t carve_forward(void* base, int32_t dtype, bool saved, Experts* x) {
  const size_t n = static_cast<size_t>(x->pairs);
  Carver c{static_cast<char*>(base)};
  if (!saved) carve_plan(&c, x);
  x->act = c.take(size_of(dtype) * (n + kPlanRows) * x->hidden);
  x->y = static_cast<float*>(c.take(4 * n * x->dim));
  return c.used;
}

size_t carve_backward(void* base, int32_t dtype, Experts* x) {
  const size_t n = static_cast<size_t>(x->pairs), s = size_of(dtype);
  Carver c{static_cast<char*>(base)};
  x->dot_tiles = (x->hidden + kSmallRows - 1) / kSmallRows;
  x->dpre = c.take(2 * s * (n + kPlanRows) * x->hidden);
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

// Whether every product's grid stays below 2^32 threads.
bool grids_ok(const Experts& x) {
  const int64_t side = x.aligned ? kTileRows : kSmallRows, threads = x.aligned ? 512 : 256;
  const auto tiles = [&](int64_t n) { return (n + side - 1) / side; };
  const int64_t rows = (x.pairs / kPlanRows + x.experts) * (kPlanRows / side);
  const int64_t wide = tiles(2 * static_cast<int64_t>(x.hidden)) + 1, deep = tiles(x.dim);
  const int64_t most = std::max(std::max(rows * wide, rows * deep), x.experts * wide * deep);
  return most + 256 < (int64_t{1} << 32) / threads;
}

bool workspace_ok(const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 256 == 0; }

}  // namespace

hipError_t launch_plan(const Experts& x, hipStream_t st) {
  ex_plan<<<x.experts, kPlanThreads, 0, st>>>(static_cast<int32_t>(x.pairs), x.experts, x.top,
                                              x.ids, x.plan);
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
  a.aligned = gsn::aligned(a, p->dtype);
  if (!gsn::grids_ok(a)) return GSN_E_CAPACITY;
  if (saved) gsn::carve_saved(saved, &a);
  gsn::carve_forward(workspace, p->dtype, saved != nullptr, &a);
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
  a.aligned = gsn::aligned(a, p->dtype);
  if (!gsn::grids_ok(a)) return GSN_E_CAPACITY;
  gsn::carve_saved(const_cast<void*>(saved), &a);
  gsn::carve_backward(workspace, p->dtype, &a);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = p->dtype == GSN_F32 ? gsn::launch_experts_backward<float>(a, st)
                       : p->dtype == GSN_BF16
                           ? gsn::launch_experts_backward<gsn::bf16_t>(a, st)
                           : gsn::launch_experts_backward<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

}  // extern "C"
