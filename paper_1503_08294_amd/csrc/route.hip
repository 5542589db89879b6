// Routing of tokens to experts: scores, the choice of K of E experts, their weights, and the
// gradient of the logits.
//
// A token's logits lie in SUB lanes of a wave (16: four tokens a wave; 64: one), NPL experts in a
// row each.  An expert's place in the order is its float's bits in unsigned order, 0 if it is shut
// out; ties go to the lower lane and the earlier of its experts, which is the lower index.
// Every lane keeps its four best; each of the K rounds takes the largest of the lanes' first ones
// (16 lanes: four instructions that move data between lanes), and only a lane whose four are all
// taken looks through its experts again (with two kept, one of a wave's lanes did in nearly every
// round, and 16,384 tokens of 256 experts took 19 us in place of 12).
//
// Bound by instructions, and by the latency of their chain where tokens are few: 16,384 tokens of
// 256 experts, 8 chosen of 4 of 8 groups, sigmoid with a balance: 12 us a call among others, 14 in
// a trace (8 MB of logits would take 2), 1,174 vector instructions a wave, which take 77% of the
// cycles to issue; one such token 6 us; 65,536 tokens of 64 experts, 2 chosen, softmax: 8 us,
// backward 7.
#include "mixture.h"

#pragma clang fp contract(fast)

namespace gsn {
namespace {

constexpr int kThreads = 256;
constexpr int kMostExperts = 1024;
constexpr int kMostTop = 64;
constexpr int kMostGroups = 64;

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

// unsigned order of the bits = order of the floats (-0 equals +0), and back
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) {
  return __uint_as_float(k ^ (static_cast<uint32_t>(static_cast<int32_t>(~k) >> 31) | 0x80000000u));
}

// The value of a lane of this row of 16: its neighbour (lane ^ 1), lane ^ 2, and the mirror
// images in 8 and in 16 lanes; after a reduction's four steps all 16 hold the result.
template <int STEP>
__device__ __forceinline__ uint32_t other(uint32_t v) {
  constexpr int kCtrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;
  return __builtin_amdgcn_mov_dpp(static_cast<int>(v), kCtrl, 0xf, 0xf, true);
}
template <int SUB, typename F>
__device__ __forceinline__ uint32_t reduce(uint32_t v, F f) {
  v = f(v, other<0>(v));
  v = f(v, other<1>(v));
  v = f(v, other<2>(v));
  v = f(v, other<3>(v));
  if constexpr (SUB == kWave) {
    v = f(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 16)));
    v = f(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 32)));
  }
  return v;
}
template <int SUB>
__device__ __forceinline__ uint32_t max_u32(uint32_t v) {
  return reduce<SUB>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int SUB>
__device__ __forceinline__ float max_f32(float v) {
  return __uint_as_float(reduce<SUB>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
template <int SUB>
__device__ __forceinline__ float sum_f32(float v) {
  return __uint_as_float(reduce<SUB>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
// the lowest of this token's lanes where p holds, -1 for none
template <int SUB>
__device__ __forceinline__ int first_lane(bool p) {
  const uint64_t m = __ballot(p);
  if constexpr (SUB == kWave) return __ffsll(static_cast<unsigned long long>(m)) - 1;
  return __ffs(static_cast<int>((m >> ((threadIdx.x % kWave) & 48)) & 0xffff)) - 1;
}

// What a wave's lanes wrote to LDS before it, they may read from each other after it.
__device__ __forceinline__ void lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
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

// A lane's NPL elements of a row of n at i; rows start at any element.
template <typename T, int NPL>
__device__ __forceinline__ void load_row(const T* row, int i, int n, float none, float (&v)[NPL]) {
  constexpr int kW = NPL * sizeof(T) >= 16 ? 16 / sizeof(T) : NPL;
  typedef T Some __attribute__((ext_vector_type(kW), aligned(sizeof(T))));
  if (NPL > 1 && i + NPL <= n) {
#pragma unroll
    for (int h = 0; h < NPL; h += kW) {
      const Some c = *reinterpret_cast<const Some*>(row + i + h);
#pragma unroll
      for (int k = 0; k < kW; ++k) v[h + k] = to_float(c[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < NPL; ++k) v[k] = i + k < n ? to_float(row[i + k]) : none;
  }
}
template <typename T, int NPL>
__device__ __forceinline__ void store_row(T* row, int i, int n, const float (&v)[NPL]) {
  constexpr int kW = NPL * sizeof(T) >= 16 ? 16 / sizeof(T) : NPL;
  typedef T Some __attribute__((ext_vector_type(kW), aligned(sizeof(T))));
  if (NPL > 1 && i + NPL <= n) {
#pragma unroll
    for (int h = 0; h < NPL; h += kW) {
      Some c;
#pragma unroll
      for (int k = 0; k < kW; ++k) c[k] = from_float<T>(v[h + k]);
      *reinterpret_cast<Some*>(row + i + h) = c;
    }
  } else {
#pragma unroll
    for (int k = 0; k < NPL; ++k)
      if (i + k < n) row[i + k] = from_float<T>(v[k]);
  }
}

// A lane's four best after (k, at) in the order, best first; 0 where there is none.
struct Best {
  uint32_t k[4];
  int p[4];
};
template <int NPL>
__device__ __forceinline__ Best best_after(const uint32_t (&key)[NPL], uint32_t k, int at) {
  Best t{};
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    uint32_t c = key[j] < k || (key[j] == k && j > at) ? key[j] : 0;
    int p = j;
    bool up = false;
#pragma unroll
    for (int i = 0; i < 4 && i <= j; ++i) {
      up = up || c > t.k[i];  // (an equal one that came before stays before; the rest move up)
      const uint32_t ck = t.k[i];
      const int cp = t.p[i];
      t.k[i] = up ? c : ck;
      t.p[i] = up ? p : cp;
      c = up ? ck : c;
      p = up ? cp : p;
    }
  }
  return t;
}

template <typename T, int SUB, int NPL>
__global__ __launch_bounds__(kThreads) void rt_choose(RouteArgs a) {
  constexpr int kTokens = kThreads / SUB;
  __shared__ int32_t picked[kTokens][SUB];
  // the logits, where a bias keeps the keys from telling them; before that, for groups whose
  // experts are not whole lanes, the keys
  __shared__ __attribute__((aligned(16))) uint32_t words[kTokens][SUB * NPL];
  __shared__ uint32_t values[kTokens][kMostGroups];
  const int sub = threadIdx.x / SUB, lane = threadIdx.x % SUB;
  // (a token past the end is worked on like the last one, and not written)
  const int64_t mine = static_cast<int64_t>(blockIdx.x) * kTokens + sub;
  const int64_t t = mine < a.tokens ? mine : a.tokens - 1;
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  const float ninf = -__builtin_inff();
  const int e0 = lane * NPL;
  const bool live = !a.valid || a.valid[t] != 0;
  float l[NPL], b[NPL];
  load_row(row, e0, a.experts, ninf, l);
  if (a.balance) load_row(a.balance, e0, a.experts, ninf, b);
#pragma unroll
  for (int j = 0; j < NPL; ++j) l[j] = live ? clean(l[j]) : ninf;
  const bool grouped = a.groups > 1 && a.top_groups < a.groups;
  // softmax over all experts, where a bias or a group's sum or the weights take it
  float most = 0.0f, inv = 0.0f;
  if (a.softmax && (a.balance || !a.renorm || (grouped && a.best == 2))) {
    most = ninf;
#pragma unroll
    for (int j = 0; j < NPL; ++j) most = fmaxf(most, l[j]);
    most = fmaxf(max_f32<SUB>(most), -__FLT_MAX__);
    float total = 0.0f;
#pragma unroll
    for (int j = 0; j < NPL; ++j) total += __expf(l[j] - most);
    total = sum_f32<SUB>(total);
    inv = total > 0.0f ? 1.0f / total : 0.0f;
  }
  const auto score = [&](float v) { return a.softmax ? __expf(v - most) * inv : sigmoid(v); };
  uint32_t key[NPL];
  if (a.balance) {
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      const float c = score(l[j]) + b[j];
      key[j] = l[j] > ninf && c > ninf ? ordered(c) : 0;
    }
  } else {
#pragma unroll
    for (int j = 0; j < NPL; ++j) key[j] = l[j] > ninf ? ordered(l[j]) : 0;
  }
  Best top = best_after(key, 0xffffffffu, -1);

  if (grouped) {
    const int width = a.experts / a.groups;
    // the value of a group whose two best are k1, k2
    const auto value_of = [&](uint32_t k1, uint32_t k2) -> uint32_t {
      if (k1 == 0 || a.best == 1) return k1;
      float v = unordered(k1), w = unordered(k2);
      if (!a.balance) {
        v = score(v);
        w = score(w);
      }
      return ordered(k2 != 0 ? v + w : v);
    };
    const int lanes = width / NPL;
    if (lanes * NPL == width && (lanes == 1 || lanes == 2 || lanes == 4)) {
      // whole lanes: the two best of a group, then one round of the largest value for each kept
      uint32_t k1 = top.k[0], k2 = top.k[1];
      const auto join = [&](uint32_t o1, uint32_t o2) {
        const uint32_t low = k1 < o1 ? k1 : o1, high = k2 > o2 ? k2 : o2;
        k1 = k1 > o1 ? k1 : o1;
        k2 = low > high ? low : high;
      };
      if (lanes > 1) join(other<0>(k1), other<0>(k2));
      if (lanes > 2) join(other<1>(k1), other<1>(k2));
      uint32_t value = e0 < a.experts ? value_of(k1, k2) : 0;
      bool kept = false;
      for (int g = 0; g < a.top_groups; ++g) {
        const uint32_t best = max_u32<SUB>(value);
        const int first = first_lane<SUB>(best != 0 && value == best);
        if (first >= 0 && first / lanes == lane / lanes) {
          kept = true;
          value = 0;
        }
      }
#pragma unroll
      for (int j = 0; j < NPL; ++j) key[j] = kept ? key[j] : 0;
      if (!kept) top = Best{};
    } else {
#pragma unroll
      for (int j = 0; j < NPL; ++j) words[sub][e0 + j] = key[j];
      lds_fence();
      for (int g = lane; g < a.groups; g += SUB) {
        uint32_t k1 = 0, k2 = 0;
        for (int i = 0; i < width; ++i) {
          const uint32_t k = words[sub][g * width + i];
          const uint32_t low = k < k1 ? k : k1;
          k1 = k > k1 ? k : k1;
          k2 = low > k2 ? low : k2;
        }
        values[sub][g] = value_of(k1, k2);
      }
      lds_fence();
#pragma unroll
      for (int j = 0; j < NPL; ++j) {
        const int e = e0 + j;
        if (e >= a.experts) continue;
        const int g = e / width;
        const uint32_t v = values[sub][g];
        int rank = 0;
        for (int i = 0; i < a.groups; ++i) {
          const uint32_t o = values[sub][i];
          rank += o > v || (o == v && i < g);
        }
        if (rank >= a.top_groups) key[j] = 0;
      }
      top = best_after(key, 0xffffffffu, -1);
    }
  }

  // K rounds
  if (a.balance) {
#pragma unroll
    for (int j = 0; j < NPL; ++j) words[sub][e0 + j] = __float_as_uint(l[j]);
  }
  uint32_t last = 0xffffffffu, mine_key = 0;
  int last_at = -1;
  picked[sub][lane] = -1;
  lds_fence();
  for (int k = 0; k < a.top; ++k) {
    const uint32_t best = max_u32<SUB>(top.k[0]);
    const int first = first_lane<SUB>(best != 0 && top.k[0] == best);
    mine_key = lane == k ? best : mine_key;
    const bool won = first == lane;
    if (won) {
      picked[sub][k] = e0 + top.p[0];
      last = top.k[0];
      last_at = top.p[0];
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        top.k[i] = top.k[i + 1];
        top.p[i] = top.p[i + 1];
      }
      top.k[3] = 0;
    }
    if (NPL > 4 && __any(won && top.k[0] == 0)) {
      const Best next = best_after(key, last, last_at);
      if (won && top.k[0] == 0) top = next;
    }
  }
  lds_fence();
  const int32_t id = lane < a.top ? picked[sub][lane] : -1;
  const float logit = id < 0 ? ninf
                      : a.balance ? __uint_as_float(words[sub][id]) : unordered(mine_key);
  float s = 0.0f;
  if (a.renorm) {
    const float high = fmaxf(max_f32<SUB>(logit), -__FLT_MAX__);
    if (id >= 0) s = a.softmax ? __expf(logit - high) : sigmoid_from(logit, fminf(high, 0.0f));
    const float sum = sum_f32<SUB>(s);
    s = sum > 0.0f ? s / sum : 0.0f;
  } else if (id >= 0) {
    s = score(logit);
  }
  if (lane < a.top && mine < a.tokens) {
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
// dl_k = p_k (g_k - sum g p) (1 - s_k), since d log s = (1 - s) dl.  The chosen experts' values
// reach the lanes that write their places through a row in LDS.
template <typename T, int SUB, int NPL>
__global__ __launch_bounds__(kThreads) void rt_backward(RouteBackArgs a) {
  constexpr int kTokens = kThreads / SUB;
  __shared__ __attribute__((aligned(16))) float rows[kTokens][SUB * NPL];
  const int sub = threadIdx.x / SUB, lane = threadIdx.x % SUB;
  const int64_t mine = static_cast<int64_t>(blockIdx.x) * kTokens + sub;
  const int64_t t = mine < a.tokens ? mine : a.tokens - 1;
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  const float ninf = -__builtin_inff();
  const int e0 = lane * NPL;
#pragma unroll
  for (int j = 0; j < NPL; ++j) rows[sub][e0 + j] = 0.0f;
  int32_t id = -1;
  float g = 0.0f;
  if (lane < a.top) {
    id = a.ids[t * a.top + lane];
    if (id < 0 || id >= a.experts) id = -1;
    if (id >= 0) g = a.dweights[t * a.top + lane] * a.scale;
  }
  const float logit = id >= 0 ? clean(to_float(row[id])) : ninf;
  const bool any = first_lane<SUB>(id >= 0) >= 0;
  const bool dense = a.softmax && !a.renorm;  // every expert has a gradient
  float l[NPL], most = 0.0f, inv = 0.0f;
  if (dense) {
    load_row(row, e0, a.experts, ninf, l);
    most = ninf;
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      l[j] = any ? clean(l[j]) : ninf;
      most = fmaxf(most, l[j]);
    }
    most = fmaxf(max_f32<SUB>(most), -__FLT_MAX__);
    float total = 0.0f;
#pragma unroll
    for (int j = 0; j < NPL; ++j) total += __expf(l[j] - most);
    total = sum_f32<SUB>(total);
    inv = total > 0.0f ? 1.0f / total : 0.0f;
  }
  float back = 0.0f, mean = 0.0f;
  if (a.renorm) {
    const float high = fmaxf(max_f32<SUB>(logit), -__FLT_MAX__);
    float p = 0.0f;
    if (id >= 0) p = a.softmax ? __expf(logit - high) : sigmoid_from(logit, fminf(high, 0.0f));
    const float sum = sum_f32<SUB>(p);
    p = sum > 0.0f ? p / sum : 0.0f;
    mean = sum_f32<SUB>(g * p);
    back = p * (g - mean);
    // 1 - sigmoid(l) = sigmoid(-l), without the cancellation
    if (!a.softmax) back *= sigmoid(-logit);
  } else if (a.softmax) {
    mean = sum_f32<SUB>(id >= 0 ? g * (__expf(logit - most) * inv) : 0.0f);
    back = g;
  } else {
    back = g * sigmoid(logit) * sigmoid(-logit);
  }
  lds_fence();
  if (id >= 0) rows[sub][id] = back;
  lds_fence();
  float d[NPL];
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    d[j] = rows[sub][e0 + j];
    if (dense) d[j] = l[j] > ninf ? __expf(l[j] - most) * inv * (d[j] - mean) : 0.0f;
  }
  if (mine < a.tokens)
    store_row(static_cast<T*>(a.dlogits) + t * a.dstride, e0, a.experts, d);
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

// 16 lanes a token where they hold its experts and chosen ones, else a wave.  Over 128 experts a
// wave also where the tokens are too few to fill the card, so that one token's latency counts:
// 256 experts in 8 groups, 16 lanes a token and a wave, us: 1 token 7.5 and 6.4, 1024 tokens 7.5
// and 7.0, 4096 tokens 8.2 and 9.5, 65,536 tokens 35 and 78; 128 experts, 1 token: 3.5 and 3.9.
constexpr int64_t kFewTokens = 1024;
template <typename T>
hipError_t choose(const RouteArgs& a, hipStream_t st) {
  const auto blocks = [&](int sub) {
    const int per = kThreads / sub;
    return static_cast<uint32_t>((a.tokens + per - 1) / per);
  };
  if (a.top <= 16 && a.experts <= 64)
    rt_choose<T, 16, 4><<<blocks(16), kThreads, 0, st>>>(a);
  else if (a.top <= 16 && a.experts <= 128)
    rt_choose<T, 16, 8><<<blocks(16), kThreads, 0, st>>>(a);
  else if (a.top <= 16 && a.experts <= 256 && a.tokens > kFewTokens)
    rt_choose<T, 16, 16><<<blocks(16), kThreads, 0, st>>>(a);
  else if (a.experts <= 256)
    rt_choose<T, 64, 4><<<blocks(64), kThreads, 0, st>>>(a);
  else if (a.experts <= 512)
    rt_choose<T, 64, 8><<<blocks(64), kThreads, 0, st>>>(a);
  else
    rt_choose<T, 64, 16><<<blocks(64), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const RouteBackArgs& a, hipStream_t st) {
  const auto blocks = [&](int sub) {
    const int per = kThreads / sub;
    return static_cast<uint32_t>((a.tokens + per - 1) / per);
  };
  if (a.top <= 16 && a.experts <= 64)
    rt_backward<T, 16, 4><<<blocks(16), kThreads, 0, st>>>(a);
  else if (a.top <= 16 && a.experts <= 128)
    rt_backward<T, 16, 8><<<blocks(16), kThreads, 0, st>>>(a);
  else if (a.top <= 16 && a.experts <= 256)
    rt_backward<T, 16, 16><<<blocks(16), kThreads, 0, st>>>(a);
  else if (a.experts <= 256)
    rt_backward<T, 64, 4><<<blocks(64), kThreads, 0, st>>>(a);
  else if (a.experts <= 512)
    rt_backward<T, 64, 8><<<blocks(64), kThreads, 0, st>>>(a);
  else
    rt_backward<T, 64, 16><<<blocks(64), kThreads, 0, st>>>(a);
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

constexpr int64_t kMostTokens = int64_t{1} << 25;  // a wave each at most, in a grid of 2^31 threads

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
