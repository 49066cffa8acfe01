// Instances of the dense tiles (dense_tile.h) that write dg and du.
#include "dense_tile.h"

namespace si {

hipError_t dense_dh(int type, const DenseArgs& a, int tile, hipStream_t s) {
  if (a.up)
    return type == kTypeBF16 ? dense_launch<kTypeBF16, kCol, kRow, 1, 2>(a, tile, 1, s)
                             : dense_launch<kTypeF16, kCol, kRow, 1, 2>(a, tile, 1, s);
  return type == kTypeBF16 ? dense_launch<kTypeBF16, kCol, kRow, 1, 1>(a, tile, 1, s)
                           : dense_launch<kTypeF16, kCol, kRow, 1, 1>(a, tile, 1, s);
}

}  // namespace si
