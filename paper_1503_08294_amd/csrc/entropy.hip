// Softmax cross entropy over many classes: pieces of the classes, buffers, and the C entry points.
#include "entropy.h"

#include <algorithm>

#include "experts_rule.h"
#include "few.h"

namespace gsn {
namespace {

int64_t up_to(int64_t n, int64_t per) { return (n + per - 1) / per * per; }
size_t up(size_t n) { return (n + 255) / 256 * 256; }

// Bytes that the parts of a forward pass, the logits' gradients of a backward pass, and the copy of
// a piece of w may have each (a piece has 256 classes at least).
constexpr int64_t kPartBytes = int64_t{1} << 28;
constexpr int64_t kPieceBytes = int64_t{1} << 29;
// Workgroups that a product of few tiles is split up into, along k, where a part keeps 1,024 bytes
// of k at least.
constexpr int64_t kFill = 512;
// Tokens from which on the logits of binary32 operands are made of two float16 values, which takes
// more memory traffic and launches, and fewer cycles of the matrix cores; of a backward pass they
// are one product of three.  As they are and in two values, us: 60,000 classes of 1,024, forward
// 224 tokens 284 and 229, 256 285 and 235, 320 357 and 268, backward 849 and 790, 887 and 841,
// 1,116 and 1,034; 10,007 of 501, 256 tokens 52 and 56, backward 115 and 130, 512 tokens 70 and 65,
// 181 and 183; 2,000 of 2,048, 256 tokens 47 and 60, backward 110 and 120.
constexpr int64_t kTwoTokens = 256;

// Tokens up to which gradients of the logits are kept in two values of a 2-byte type.  In one, a
// token's dx and its class's row of dw are off by the rounding of its target's gradient, up to half
// a step all of them; over many tokens these differ, over a few they may all be large.  us of a
// backward pass in one value and in two, bfloat16: 50,001 classes of 1,024, 1 token 79 and 82, 16
// 83 and 90, 32 88 and 98, 64 96 and 110, 128 110 and 141; 10,007 of 501, 32 tokens 37 and 39.
constexpr int64_t kTwoGradients = 32;

bool params_ok(const gsn_entropy_params* p) {
  return p && p->dtype >= GSN_F32 && p->dtype <= GSN_F16 && p->tokens >= 0 &&
         p->tokens <= (1 << 24) && p->dim >= 1 && p->dim <= (1 << 16) && p->classes >= 1 &&
         p->classes <= (1 << 28);
}

struct Carver {
  char* base;
  size_t used = 0;
  void* take(size_t n) {
    void* p = base ? base + used : nullptr;
    used += up(n);
    return p;
  }
};

int32_t split_of(int64_t rows, int64_t cols, int64_t k, int32_t dtype) {
  const int64_t tiles =
      up_to(rows, kMiddleRows) / kMiddleRows * (up_to(cols, kMiddleRows) / kMiddleRows);
  const int64_t bytes = k * static_cast<int64_t>(size_of(dtype));
  return static_cast<int32_t>(std::max<int64_t>(1, std::min(kFill / tiles, bytes / 1024)));
}

Entropy entropy_of(const gsn_entropy_params& p, bool backward) {
  Entropy x{};
  const int64_t size = static_cast<int64_t>(size_of(p.dtype));
  const int64_t tokens = std::max<int64_t>(p.tokens, 1);
  x.tokens = p.tokens;
  x.classes = p.classes;
  x.dim = p.dim;
  // (rows of the copies and of d are whole lines of 128 bytes: products read rows that begin inside
  // a line up to a fifth slower)
  x.two = p.dtype == GSN_F32 && p.tokens >= kTwoTokens;
  x.two_d = backward && p.dtype != GSN_F32 && p.tokens <= kTwoGradients;
  x.pitch = static_cast<int32_t>(up_to(p.dim, 64));
  int64_t piece = kPieceBytes / (size * x.pitch);
  if (backward) piece = std::min(piece, kPieceBytes / (size * tokens * (x.two_d ? 2 : 1)));
  else piece = std::min(piece, kPartBytes / (8 * tokens) * kSmallRows);
  piece = std::max<int64_t>(piece / 256 * 256, 256);
  // A few tokens: w is read once, whatever its rows' alignment, and no piece of it is copied.
  x.few = !backward && p.tokens <= few_at_most(p.dtype == GSN_F32, true);
  x.piece = static_cast<int32_t>(std::min(piece, up_to(p.classes, 64)));
  x.pieces = (p.classes - 1) / x.piece + 1;
  const bool may_be_few = p.tokens <= few_at_most(p.dtype == GSN_F32, false);
  x.parts = static_cast<int32_t>(up_to(may_be_few ? p.classes : x.piece, kFewCols) / kFewCols);
  x.splits_x = split_of(tokens, x.pitch, x.piece, p.dtype);
  x.splits_w = split_of(x.piece, x.pitch, tokens, p.dtype);
  return x;
}

// x and w in two values (a tile reads the exponents of whole tiles).
void carve_two(Carver* c, Entropy* x) {
  const size_t t = static_cast<size_t>(x->tokens), n = static_cast<size_t>(x->piece);
  x->x2 = c->take(4 * t * x->pitch);
  x->w2 = c->take(4 * n * x->pitch);
  x->ex = static_cast<int32_t*>(c->take(4 * t));
  x->ew = static_cast<int32_t*>(c->take(4 * (n + kTileRows)));
  x->sizes = static_cast<uint32_t*>(c->take(8 * (1 + static_cast<size_t>(x->pieces))));
}

size_t carve_forward(void* base, int32_t dtype, Entropy* x) {
  Carver c{static_cast<char*>(base)};
  const size_t s = size_of(dtype), t = static_cast<size_t>(x->tokens);
  if (x->two) carve_two(&c, x);
  if (!x->few) {
    x->xc = c.take(s * t * x->pitch);
    x->wc = c.take(s * x->piece * static_cast<size_t>(x->pitch));
  }
  x->part = static_cast<float2*>(c.take(8 * t * x->parts));
  x->chosen = static_cast<float*>(c.take(4 * t));
  float* const stats = static_cast<float*>(c.take(8 * t));
  if (!x->stats) x->stats = stats;
  return c.used;
}

size_t carve_backward(void* base, int32_t dtype, Entropy* x) {
  Carver c{static_cast<char*>(base)};
  const size_t s = size_of(dtype), t = static_cast<size_t>(x->tokens);
  x->factor = static_cast<float*>(c.take(8));
  x->xc = c.take(s * t * x->pitch * (x->two_d ? 2 : 1));
  x->wc = c.take(s * x->piece * static_cast<size_t>(x->pitch));
  x->d = c.take(s * t * x->piece * (x->two_d ? 2 : 1));
  if (x->two) carve_two(&c, x);
  x->dxp = static_cast<float*>(
      c.take(4 * t * x->pitch * static_cast<size_t>(x->splits_x) * (x->two_d ? 2 : 1)));
  x->dwp = x->splits_w > 1
               ? static_cast<float*>(c.take(4 * static_cast<size_t>(x->piece) * x->pitch *
                                            static_cast<size_t>(x->splits_w)))
               : nullptr;
  return c.used;
}

// Whether the grids of a call's products stay below 2^32 threads of 256.
bool grids_ok(const Entropy& x, int32_t dtype, bool backward) {
  const int64_t side = dtype == GSN_F32 ? kSmallRows : kMiddleRows;
  const auto tiles = [&](int64_t m, int64_t n) {
    return up_to(m, side) / side * (up_to(n, side) / side);
  };
  int64_t most = tiles(x.tokens, x.piece);
  if (backward) most = std::max({most, tiles(x.tokens, x.pitch), tiles(x.piece, x.pitch)});
  return most < (1 << 23);
}

// What the kernels may read as it is: rows that start and end at multiples of 16 bytes.
bool in_place(const void* p, int64_t stride, int32_t dim, int32_t dtype) {
  const int64_t elements = 16 / static_cast<int64_t>(size_of(dtype));
  return aligned16(p) && stride % elements == 0 && dim % elements == 0;
}

// Whether an output begins where one of the inputs does.
template <class... IN>
bool over(const void* out, const IN*... in) {
  return out && ((out == in) || ...);
}

bool workspace_ok(const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 256 == 0; }

}  // namespace

extern template hipError_t launch_entropy<float>(const Entropy&, hipStream_t);
extern template hipError_t launch_entropy<bf16_t>(const Entropy&, hipStream_t);
extern template hipError_t launch_entropy<f16_t>(const Entropy&, hipStream_t);
extern template hipError_t launch_entropy_backward<float>(const Entropy&, hipStream_t);
extern template hipError_t launch_entropy_backward<bf16_t>(const Entropy&, hipStream_t);
extern template hipError_t launch_entropy_backward<f16_t>(const Entropy&, hipStream_t);

}  // namespace gsn

extern "C" {

size_t gsn_cross_entropy_workspace_bytes(const gsn_entropy_params* p, int32_t backward) {
  if (!gsn::params_ok(p)) return 0;
  gsn::Entropy x = gsn::entropy_of(*p, backward != 0);
  return (backward ? gsn::carve_backward(nullptr, p->dtype, &x)
                   : gsn::carve_forward(nullptr, p->dtype, &x)) + 256;
}

int gsn_cross_entropy(const gsn_entropy_params* p, const void* x, int64_t x_stride, const void* w,
                      int64_t w_stride, const int32_t* targets, const uint8_t* valid, float* loss,
                      float* stats, void* workspace, size_t workspace_bytes, void* stream) {
  if (!gsn::params_ok(p)) return GSN_E_INVAL;
  if (p->tokens == 0) return GSN_OK;
  if (!x || !w || !targets || !loss || x_stride < p->dim || w_stride < p->dim ||
      !gsn::workspace_ok(workspace))
    return GSN_E_INVAL;
  if (workspace_bytes < gsn_cross_entropy_workspace_bytes(p, 0)) return GSN_E_CAPACITY;
  gsn::Entropy a = gsn::entropy_of(*p, false);
  if (!gsn::grids_ok(a, p->dtype, false)) return GSN_E_CAPACITY;
  if (gsn::over(loss, x, w, targets, valid, stats) || gsn::over(stats, x, w, targets, valid))
    return GSN_E_INVAL;
  a.x = x;
  a.x_stride = x_stride;
  a.w = w;
  a.w_stride = w_stride;
  a.targets = targets;
  a.valid = valid;
  a.loss = loss;
  a.stats = stats;
  a.copy_x = !gsn::in_place(x, x_stride, p->dim, p->dtype);
  a.copy_w = !gsn::in_place(w, w_stride, p->dim, p->dtype);
  if (p->tokens <= gsn::few_at_most(p->dtype == GSN_F32, !a.copy_w)) a.few = true;
  gsn::carve_forward(workspace, p->dtype, &a);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = p->dtype == GSN_F32    ? gsn::launch_entropy<float>(a, st)
                       : p->dtype == GSN_BF16 ? gsn::launch_entropy<gsn::bf16_t>(a, st)
                                              : gsn::launch_entropy<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

int gsn_cross_entropy_backward(const gsn_entropy_params* p, const float* dloss, const void* x,
                               int64_t x_stride, const void* w, int64_t w_stride,
                               const int32_t* targets, const uint8_t* valid, const float* stats,
                               void* dx, void* dw, void* workspace, size_t workspace_bytes,
                               void* stream) {
  if (!gsn::params_ok(p)) return GSN_E_INVAL;
  if (!dx && !dw) return GSN_OK;
  if (p->tokens == 0 && !dw) return GSN_OK;
  if (!w || w_stride < p->dim || !gsn::workspace_ok(workspace)) return GSN_E_INVAL;
  if (p->tokens > 0 && (!dloss || !x || !targets || !stats || x_stride < p->dim))
    return GSN_E_INVAL;
  if (workspace_bytes < gsn_cross_entropy_workspace_bytes(p, 1)) return GSN_E_CAPACITY;
  gsn::Entropy a = gsn::entropy_of(*p, true);
  if (!gsn::grids_ok(a, p->dtype, true)) return GSN_E_CAPACITY;
  // (dx is written when all else has been read but the targets and dloss)
  if (gsn::over(dx, dw, targets, valid, dloss) ||
      gsn::over(dw, x, targets, valid, stats, dloss))
    return GSN_E_INVAL;
  a.dloss = dloss;
  a.x = x;
  a.x_stride = x_stride;
  a.w = w;
  a.w_stride = w_stride;
  a.targets = targets;
  a.valid = valid;
  a.stats = const_cast<float*>(stats);
  a.dx = p->tokens > 0 ? dx : nullptr;
  a.dw = dw;
  a.copy_x = !gsn::in_place(x, x_stride, p->dim, p->dtype);
  // (the product with w meets its classes that are not valid as zeros)
  a.copy_w = valid || !gsn::in_place(w, w_stride, p->dim, p->dtype);
  gsn::carve_backward(workspace, p->dtype, &a);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = p->dtype == GSN_F32 ? gsn::launch_entropy_backward<float>(a, st)
                       : p->dtype == GSN_BF16
                           ? gsn::launch_entropy_backward<gsn::bf16_t>(a, st)
                           : gsn::launch_entropy_backward<gsn::f16_t>(a, st);
  return e == hipSuccess ? GSN_OK : GSN_E_HIP;
}

}  // extern "C"
