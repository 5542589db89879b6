// Softmax cross entropy over many classes: what the host passes to the kernels of one type.
#pragma once

#include "mixture.h"

namespace gsn {

struct Entropy {
  int64_t tokens;
  int32_t classes, dim;
  int32_t pitch;     // elements of a row of the copies of x and w
  const void* x;
  int64_t x_stride;
  const void* w;
  int64_t w_stride;
  const int32_t* targets;
  const uint8_t* valid;  // of the classes, or null
  // pieces of the classes: of a forward and of a backward pass
  int32_t piece, parts;  // classes of a piece; tiles of its columns, at most
  bool copy_x, copy_w;
  bool few;       // tokens that read w once, as it is
  bool two;       // binary32 logits of x and w in two float16 values, of pieces that allow it
  bool two_d;     // gradients of the logits in two values of a 2-byte type, backward
  void* xc;       // [tokens][pitch] x, zeros for tokens without a target (backward) and at the
                  // ends; of two_d twice, one behind the other
  void* wc;       // [piece][pitch] a piece of w, zeros for classes that are not valid
  void* x2;       // x and a piece of w in two values, the second ones behind all of the first
  void* w2;
  int32_t* ex;    // the exponents of the powers of two that give back the rows of x2,
  int32_t* ew;    // and of w2
  int32_t pieces;
  uint32_t* sizes;  // [1 + pieces][2] of x and of each piece of w: bits of the largest magnitude
                    // and of a row's largest sum of magnitudes
  // forward
  float* loss;
  float* stats;   // [2][tokens]: the largest logit, and the sum of exp(logit - largest)
  float2* part;   // [parts][tokens] the same of every tile's columns
  float* chosen;  // [tokens] logit of the target
  // backward
  const float* dloss;
  float* factor;  // 2: what dloss is multiplied by where the logits' gradients are kept, and back
  void* d;        // [tokens][piece] gradients of the logits; of two_d the second values behind them
  int32_t splits_x, splits_w;
  float* dxp;     // [splits_x][tokens][pitch]; of two_d [splits_x][2][tokens][pitch]
  float* dwp;     // [splits_w][piece][pitch], where splits_w > 1
  void* dx;
  void* dw;
};

template <typename T>
hipError_t launch_entropy(const Entropy& x, hipStream_t st);
template <typename T>
hipError_t launch_entropy_backward(const Entropy& x, hipStream_t st);

}  // namespace gsn
