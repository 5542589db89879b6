// The experts' products: what the host passes to the kernels of one type of element.
#pragma once

#include "experts_rule.h"
#include "mixture.h"

namespace gsn {

constexpr int kPlanExperts = 1024;    // experts at most
constexpr int kPlanRows = kTileRows;  // rows of a listed block

// Pairs (token, place k), number token * top + k, sorted by expert and then by number: row r of
// the products is pair rows[r], pair j is row pos[j] (-1 for a pair without an expert), expert
// e's rows are offsets[e] .. offsets[e + 1] - 1.  Blocks of kPlanRows rows that hold one expert's
// rows alone are listed in tiles as (expert, the expert's first row, its first block, its
// blocks), expert by expert, tile_count[0] of them; blocks of kSmallRows in small as (expert,
// the block's first row, its rows), tile_count[1] of them.
struct Plan {
  int32_t* offsets;     // experts + 1
  int32_t* tile_count;  // 2
  int4* tiles;          // most_tiles
  int4* small;          // most_small
  int32_t* rows;        // pairs
  int32_t* token;       // pairs: rows[r] / top
  int32_t* pos;         // pairs
  int32_t* counts;      // pairs of each expert in each chunk of them
  int32_t most_tiles, most_small;
};

struct Experts {
  int32_t side;  // of the products' tiles
  int64_t tokens;
  int32_t experts, top, dim, hidden;
  int64_t pairs;
  const void* x;
  int64_t x_stride;
  const int32_t* ids;
  const float* weights;
  const void* w1;
  const void* w2;
  Plan plan;
  // forward
  void* out;
  float* pre;    // [pairs][2 hidden] the products with w1, kept for the backward pass, or null
  void* act;     // [pairs][hidden]
  float* y;      // [pairs][dim]
  // backward
  const void* dout;
  void* dpre;    // [pairs][2 hidden]
  void* wact;    // [pairs][hidden], the activation times the pair's weight
  float* dots;   // [pairs][dot_tiles] parts of the weights' gradients
  int32_t dot_tiles;
  float* dxr;    // [pairs][dim]
  void* dx;
  float* dweights;
  void* dw1;
  void* dw2;
};

hipError_t launch_plan(const Experts& x, hipStream_t st);

template <typename T>
hipError_t launch_experts(const Experts& x, hipStream_t st);
template <typename T>
hipError_t launch_experts_backward(const Experts& x, hipStream_t st);

enum Kind {
  kForwardGate,   // act (and pre) from x, w1
  kForwardOut,    // y from act, w2
  kBackwardGate,  // dpre, wact, dots from dout, w2
  kBackwardIn,    // dxr from dpre, w1
  kWeightsIn,     // dw1 from dpre, x
  kWeightsOut     // dw2 from dout, wact
};

// Workgroups for every tile of a product.
inline int64_t product_blocks(Kind kind, const Experts& x) {
  const auto up = [](int64_t n, int64_t per) { return (n + per - 1) / per; };
  const bool of_hidden = kind == kForwardGate || kind == kBackwardGate || kind == kWeightsOut;
  const int64_t n = up(of_hidden ? x.hidden : x.dim, kind == kForwardGate ? x.side / 2 : x.side);
  const int64_t m = kind == kWeightsIn    ? x.experts * up(2 * int64_t{x.hidden}, x.side)
                    : kind == kWeightsOut ? x.experts * up(x.dim, x.side)
                    : x.side == kSmallRows
                        ? x.plan.most_small
                        : int64_t{x.plan.most_tiles} * (kPlanRows / x.side);
  const int64_t round = x.side == kSmallRows ? 1 : 8 * tile_run(x.side);
  return up(n * m, round) * round;
}

}  // namespace gsn
