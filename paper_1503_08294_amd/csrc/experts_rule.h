// The experts' products: which tiles a call takes (host code alone).
#pragma once

#include <stdint.h>

namespace gsn {

// Sides of the products' tiles, and the run of them that goes to one XCD.
constexpr int32_t kTileRows = 256;
constexpr int32_t kMiddleRows = 128;
constexpr int32_t kSmallRows = 64;
constexpr int32_t tile_run(int32_t side) {
  return side == kTileRows ? 32 : side == kMiddleRows ? 16 : 1;
}

// Sides of the products' tiles: of 2-byte elements the larger ones, from 128 pairs an expert on and
// where the first product has enough of them to fill the chip; the largest need rows, and starts
// of rows, at multiples of 16 bytes.  Forward and backward pass in us, with sides of
// 256 and 64 (from 128 tiles of 256 on): 2,000 tokens, 2 of 8 experts, 1,024 x 1,024: 218 and 251;
//   16,384, 2 of 32, 2,048 x 2,048: 2,900 and 5,282; 1,024, 2 of 4, 1,024 x 512 (40 tiles): 141 and
//   94; 495, 3 of 7, 1,984 x 320: 175 and 116; forward of 5,100, 1 of 8, 448 x 992: 55 and 66;
// 128 and 64 (from 256 tiles of 128 on): 16,384, 2 of 32, 2,047 x 2,047: 5,243 and 7,782; 1,500, 2
//   of 8, 999 x 701 (297 tiles): 174 and 190; 1,500, 1 of 8, 511 x 1,023 (240 tiles): 141 and 109;
//   with fewer pairs an expert, 2,048, 2 of 64, 511 x 701: 307 and 281.
// In binary32, where the matrix cores are 16 times slower, small tiles waste less at the edges:
// 128 and 64: 4,096, 2 of 16, 1,024 x 1,024: 1,981 and 1,558.
// (aligned: every matrix, and the step from row to row of x, at multiples of 16 bytes)
inline int32_t tile_side(bool binary32, int64_t pairs, int32_t experts, int32_t dim,
                         int32_t hidden, bool aligned) {
  const auto tiles = [&](int32_t side) {
    return (pairs / side + experts / 2) * ((2 * static_cast<int64_t>(hidden) + side - 1) / side);
  };
  if (binary32 || pairs < int64_t{128} * experts) return kSmallRows;
  if (aligned && dim % 8 == 0 && hidden % 8 == 0 && tiles(kTileRows) >= 128) return kTileRows;
  // (a row shorter than 16 bytes is loaded by the small tiles alone)
  return dim >= 8 && hidden >= 8 && tiles(kMiddleRows) >= 256 ? kMiddleRows : kSmallRows;
}

}  // namespace gsn
