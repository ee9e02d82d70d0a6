// Tiles of the matrix products (mhcl_product.h).
#pragma once

namespace mhcl {

// How a product D[m][n] is tiled: extents in m and n of a block of threads, and that in m of one of its waves (of logits, what a softmax's
// partial maximum and sum stand for).
struct ProductTile {
  int bm, bn, gran;
};
constexpr ProductTile kTileBig{256, 256, 128}, kTileMid{128, 128, 64}, kTileSlim{128, 32, 32};

}  // namespace mhcl
