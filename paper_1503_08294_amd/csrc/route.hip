// Routing of tokens to experts: scores, the choice of K of E experts, their weights, and the
// gradient of the logits.
//
// A token's logits lie in the lanes of one wave (expert lane + 64 j).  An expert's place in the
// order is one 64-bit key, the float's bits in unsigned order above the complemented index, so
// the largest key is the best expert and ties go to the lowest index; 0 is an expert shut out.
#include "mixture.h"

#pragma clang fp contract(fast)

namespace gsn {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMostExperts = 1024;
constexpr int kMostTop = 64;  // one chosen expert a lane
constexpr int kMostGroups = 64;

using u64 = unsigned long long;

struct RouteArgs {
  int32_t experts, top, groups, top_groups, best;
  bool softmax, renorm;
  float scale;
  int64_t tokens;
  const void* logits;
  int64_t stride;
  const float* balance;
  const uint8_t* valid;
  int32_t* ids;
  float* weights;
};

// unsigned order of the bits = order of the floats (-0 equals +0)
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}

__device__ __forceinline__ u64 wave_max_key(u64 k) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const u64 other = __shfl_xor(k, o);
    k = other > k ? other : k;
  }
  return k;
}

// a logit as the scores take it: NaN is shut out like -inf, +inf is the largest float
__device__ __forceinline__ float clean(float l) {
  return l == l ? fminf(l, __FLT_MAX__) : -__builtin_inff();
}

// Share of a renormalised sigmoid before the division, relative to exp(low) with low the least
// of 0 and the largest chosen logit: no chosen set underflows as a whole.
__device__ __forceinline__ float sigmoid_from(float l, float low) {
  return l > 0.0f ? sigmoid(l) : __expf(l - low) * __builtin_amdgcn_rcpf(1.0f + __expf(l));
}

template <typename T, int NPL>
__global__ __launch_bounds__(kThreads) void rt_choose(RouteArgs a) {
  __shared__ u64 keys[kWaves][NPL * kWave];
  __shared__ float pick[kWaves][NPL * kWave];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
  if (t >= a.tokens) return;
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  const float ninf = -__builtin_inff();
  float l[NPL];
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    const int e = lane + kWave * j;
    l[j] = e < a.experts ? clean(to_float(row[e])) : ninf;
  }
  if (a.valid && a.valid[t] == 0) {
#pragma unroll
    for (int j = 0; j < NPL; ++j) l[j] = ninf;
  }
  float most = ninf;
#pragma unroll
  for (int j = 0; j < NPL; ++j) most = fmaxf(most, l[j]);
  most = fmaxf(wave_max(most), -__FLT_MAX__);
  float total = 0.0f;
  if (a.softmax) {
#pragma unroll
    for (int j = 0; j < NPL; ++j) total += __expf(l[j] - most);
    total = wave_sum(total);
  }
  const float inv = total > 0.0f ? 1.0f / total : 0.0f;
  // choice: score + bias; key: the logits give the same order where there is no bias
  u64 key[NPL];
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    const int e = lane + kWave * j;
    float c = a.softmax ? __expf(l[j] - most) * inv : sigmoid(l[j]);
    float k = l[j];
    if (a.balance) {
      c += e < a.experts ? a.balance[e] : 0.0f;
      k = c;
    }
    const bool shut = !(l[j] > ninf) || !(k > ninf);
    key[j] = shut ? 0 : (static_cast<u64>(ordered(k)) << 32) | (0xffffffffu - e);
    keys[wave][e] = key[j];
    pick[wave][e] = c;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (a.groups > 1 && a.top_groups < a.groups) {
    const int width = a.experts / a.groups;
    u64 value = 0;  // of the group of this lane
    if (lane < a.groups) {
      u64 k1 = 0, k2 = 0;
      for (int i = 0; i < width; ++i) {
        const u64 k = keys[wave][lane * width + i];
        if (k > k1) {
          k2 = k1;
          k1 = k;
        } else if (k > k2) {
          k2 = k;
        }
      }
      if (k1 != 0) {
        uint32_t v = static_cast<uint32_t>(k1 >> 32);
        if (a.best == 2) {
          float s = pick[wave][0xffffffffu - static_cast<uint32_t>(k1)];
          if (k2 != 0) s += pick[wave][0xffffffffu - static_cast<uint32_t>(k2)];
          v = ordered(s);
        }
        value = (static_cast<u64>(v) << 32) | (0xffffffffu - lane);
      }
    }
    int rank = 0;
    for (int g = 0; g < a.groups; ++g) rank += __shfl(value, g) > value;
    const u64 kept = __ballot(value != 0 && rank < a.top_groups);
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      const int e = lane + kWave * j;
      if (e < a.experts && !((kept >> (e / width)) & 1)) key[j] = 0;
    }
  }
  // K rounds of the largest key; lane k holds the k-th
  int32_t id = -1;
  float logit = ninf;
  for (int k = 0; k < a.top; ++k) {
    u64 b = 0;
#pragma unroll
    for (int j = 0; j < NPL; ++j) b = key[j] > b ? key[j] : b;
    b = wave_max_key(b);
    if (b == 0) break;
    const int32_t e = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(b));
    float v = ninf;
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      if (key[j] == b) {
        key[j] = 0;
        v = l[j];
      }
    }
    v = __shfl(v, e % kWave);
    if (lane == k) {
      id = e;
      logit = v;
    }
  }
  const float top = fmaxf(wave_max(logit), -__FLT_MAX__);
  float s = 0.0f;
  if (id >= 0) {
    if (a.softmax) s = a.renorm ? __expf(logit - top) : __expf(logit - most) * inv;
    else s = a.renorm ? sigmoid_from(logit, fminf(top, 0.0f)) : sigmoid(logit);
  }
  if (a.renorm) {
    const float sum = wave_sum(s);
    s = sum > 0.0f ? s / sum : 0.0f;
  }
  if (lane < a.top) {
    a.ids[t * a.top + lane] = id;
    a.weights[t * a.top + lane] = s * a.scale;
  }
}

struct RouteBackArgs {
  int32_t experts, top;
  bool softmax, renorm;
  float scale;
  int64_t tokens;
  const float* dweights;
  const void* logits;
  int64_t stride;
  const int32_t* ids;
  void* dlogits;
  int64_t dstride;
};

// softmax: dl = s (G - sum G s), G the chosen experts' scaled gradients; renormalised, over the
// chosen alone, dl_k = p_k (g_k - sum g p).  sigmoid: dl_k = g_k s_k (1 - s_k); renormalised
// dl_k = p_k (g_k - sum g p) (1 - s_k), since d log s = (1 - s) dl.
template <typename T, int NPL>
__global__ __launch_bounds__(kThreads) void rt_backward(RouteBackArgs a) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
  if (t >= a.tokens) return;
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  T* out = static_cast<T*>(a.dlogits) + t * a.dstride;
  const float ninf = -__builtin_inff();
  int32_t id = -1;
  float g = 0.0f;
  if (lane < a.top) {
    id = a.ids[t * a.top + lane];
    if (id < 0 || id >= a.experts) id = -1;
    if (id >= 0) g = a.dweights[t * a.top + lane] * a.scale;
  }
  const float logit = id >= 0 ? clean(to_float(row[id])) : ninf;
  const bool any = __ballot(id >= 0) != 0;
  float l[NPL], most = 0.0f, inv = 0.0f;
#pragma unroll
  for (int j = 0; j < NPL; ++j) l[j] = ninf;
  if (a.softmax && !a.renorm && any) {
    most = ninf;
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      const int e = lane + kWave * j;
      if (e < a.experts) l[j] = clean(to_float(row[e]));
      most = fmaxf(most, l[j]);
    }
    most = fmaxf(wave_max(most), -__FLT_MAX__);
    float total = 0.0f;
#pragma unroll
    for (int j = 0; j < NPL; ++j) total += __expf(l[j] - most);
    total = wave_sum(total);
    inv = total > 0.0f ? 1.0f / total : 0.0f;
  }
  float back = 0.0f, mean = 0.0f;
  if (a.renorm) {
    const float top = fmaxf(wave_max(logit), -__FLT_MAX__);
    float p = 0.0f;
    if (id >= 0)
      p = a.softmax ? __expf(logit - top) : sigmoid_from(logit, fminf(top, 0.0f));
    const float sum = wave_sum(p);
    p = sum > 0.0f ? p / sum : 0.0f;
    mean = wave_sum(g * p);
    back = p * (g - mean);
    // 1 - sigmoid(l) = sigmoid(-l), without the cancellation
    if (!a.softmax) back *= sigmoid(-logit);
  } else if (a.softmax) {
    mean = wave_sum(id >= 0 ? g * (__expf(logit - most) * inv) : 0.0f);
    back = g;
  } else {
    back = g * sigmoid(logit) * sigmoid(-logit);
  }
  if (id < 0) back = 0.0f;
  float d[NPL];
#pragma unroll
  for (int j = 0; j < NPL; ++j) d[j] = 0.0f;
  for (int k = 0; k < a.top; ++k) {
    const int32_t e = __shfl(id, k);
    const float b = __shfl(back, k);
#pragma unroll
    for (int j = 0; j < NPL; ++j) d[j] += e == lane + kWave * j ? b : 0.0f;
  }
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    const int e = lane + kWave * j;
    if (a.softmax && !a.renorm)
      d[j] = l[j] > ninf ? __expf(l[j] - most) * inv * (d[j] - mean) : 0.0f;
    if (e < a.experts) out[e] = from_float<T>(d[j]);
  }
}

__global__ __launch_bounds__(kThreads) void rt_clear(int32_t n, int32_t* __restrict__ c) {
  const int32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i < n) c[i] = 0;
}

__global__ __launch_bounds__(kThreads) void rt_counts(int64_t pairs, int32_t experts,
                                                      const int32_t* __restrict__ ids,
                                                      int32_t* __restrict__ counts) {
  __shared__ int32_t mine[kMostExperts];
  for (int e = threadIdx.x; e < experts; e += kThreads) mine[e] = 0;
  __syncthreads();
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < pairs;
       i += step) {
    const int32_t e = ids[i];
    if (e >= 0 && e < experts) atomicAdd(&mine[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += kThreads)
    if (mine[e] != 0) atomicAdd(&counts[e], mine[e]);
}

// balance[e] += rate where expert e has fewer pairs than the mean, -= rate where it has more
__global__ __launch_bounds__(kThreads) void rt_balance(int32_t experts,
                                                       const int32_t* __restrict__ counts,
                                                       float rate, float* __restrict__ balance) {
  __shared__ unsigned long long total;
  if (threadIdx.x == 0) total = 0;
  __syncthreads();
  unsigned long long s = 0;
  for (int e = threadIdx.x; e < experts; e += kThreads) s += static_cast<uint32_t>(counts[e]);
  atomicAdd(&total, s);
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += kThreads) {
    const unsigned long long mine =
        static_cast<unsigned long long>(static_cast<uint32_t>(counts[e])) * experts;
    if (mine < total) balance[e] += rate;
    else if (mine > total) balance[e] -= rate;
  }
}

template <typename T>
hipError_t choose(const RouteArgs& a, hipStream_t st) {
  const uint32_t nb = static_cast<uint32_t>((a.tokens + kWaves - 1) / kWaves);
  if (a.experts <= 64) rt_choose<T, 1><<<nb, kThreads, 0, st>>>(a);
  else if (a.experts <= 256) rt_choose<T, 4><<<nb, kThreads, 0, st>>>(a);
  else rt_choose<T, 16><<<nb, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const RouteBackArgs& a, hipStream_t st) {
  const uint32_t nb = static_cast<uint32_t>((a.tokens + kWaves - 1) / kWaves);
  if (a.experts <= 64) rt_backward<T, 1><<<nb, kThreads, 0, st>>>(a);
  else if (a.experts <= 256) rt_backward<T, 4><<<nb, kThreads, 0, st>>>(a);
  else rt_backward<T, 16><<<nb, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

bool params_ok(const gsn_route_params* p) {
  if (!p || p->experts < 1 || p->experts > kMostExperts || p->top < 1 || p->top > kMostTop ||
      p->top > p->experts)
    return false;
  if (p->score != GSN_SCORE_SOFTMAX && p->score != GSN_SCORE_SIGMOID) return false;
  if (p->groups < 1 || p->groups > kMostGroups || p->experts % p->groups != 0 ||
      p->top_groups < 1 || p->top_groups > p->groups || p->best < 1 || p->best > 2)
    return false;
  if (p->top > p->top_groups * (p->experts / p->groups)) return false;
  return p->scale == p->scale && p->scale - p->scale == 0.0f;  // finite
}

constexpr int64_t kMostTokens = int64_t{1} << 25;  // a wave each, in a grid of 2^31 threads

bool dtype_ok(int32_t d) { return d >= GSN_F32 && d <= GSN_F16; }

}  // namespace
}  // namespace gsn

extern "C" {

int gsn_route(const gsn_route_params* p, int32_t dtype, int64_t tokens, const void* logits,
              int64_t stride, const float* balance, const uint8_t* valid, int32_t* ids,
              float* weights, void* stream) {
  if (!gsn::params_ok(p) || !gsn::dtype_ok(dtype) || tokens < 0 || tokens > gsn::kMostTokens)
    return GSN_E_INVAL;
  if (tokens == 0) return GSN_OK;
  if (!logits || !ids || !weights || stride < p->experts) return GSN_E_INVAL;
  const gsn::RouteArgs a{p->experts, p->top, p->groups, p->top_groups, p->best,
                         p->score == GSN_SCORE_SOFTMAX, p->renormalise != 0, p->scale, tokens,
                         logits, stride, balance, valid, ids, weights};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = dtype == GSN_F32    ? gsn::choose<float>(a, st)
                       : dtype == GSN_BF16 ? gsn::choose<gsn::bf16_t>(a, st)
                                           : gsn::choose<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

int gsn_route_backward(const gsn_route_params* p, int32_t dtype, int64_t tokens,
                       const float* dweights, const void* logits, int64_t stride,
                       const int32_t* ids, void* dlogits, int64_t dstride, void* stream) {
  if (!gsn::params_ok(p) || !gsn::dtype_ok(dtype) || tokens < 0 || tokens > gsn::kMostTokens)
    return GSN_E_INVAL;
  if (tokens == 0) return GSN_OK;
  if (!dweights || !logits || !ids || !dlogits || stride < p->experts || dstride < p->experts)
    return GSN_E_INVAL;
  const gsn::RouteBackArgs a{p->experts, p->top, p->score == GSN_SCORE_SOFTMAX,
                             p->renormalise != 0, p->scale, tokens, dweights, logits, stride,
                             ids, dlogits, dstride};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = dtype == GSN_F32    ? gsn::backward<float>(a, st)
                       : dtype == GSN_BF16 ? gsn::backward<gsn::bf16_t>(a, st)
                                           : gsn::backward<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

int gsn_route_counts(int64_t pairs, int32_t experts, const int32_t* ids, int32_t* counts,
                     void* stream) {
  if (pairs < 0 || experts < 1 || experts > gsn::kMostExperts || !counts || (pairs > 0 && !ids))
    return GSN_E_INVAL;
  if (pairs > INT32_MAX) return GSN_E_CAPACITY;
  hipStream_t st = static_cast<hipStream_t>(stream);
  gsn::rt_clear<<<(experts + gsn::kThreads - 1) / gsn::kThreads, gsn::kThreads, 0, st>>>(
      experts, counts);
  if (pairs > 0) {
    const int64_t nb = (pairs + 4 * gsn::kThreads - 1) / (4 * gsn::kThreads);
    gsn::rt_counts<<<static_cast<uint32_t>(nb < 512 ? nb : 512), gsn::kThreads, 0, st>>>(
        pairs, experts, ids, counts);
  }
  return hipGetLastError() == hipSuccess ? GSN_OK : GSN_E_HIP;
}

int gsn_route_balance(int32_t experts, const int32_t* counts, float rate, float* balance,
                      void* stream) {
  if (experts < 1 || experts > gsn::kMostExperts || !counts || !balance || !(rate >= 0.0f))
    return GSN_E_INVAL;
  gsn::rt_balance<<<1, gsn::kThreads, 0, static_cast<hipStream_t>(stream)>>>(experts, counts,
                                                                             rate, balance);
  return hipGetLastError() == hipSuccess ? GSN_OK : GSN_E_HIP;
}

}  // extern "C"
