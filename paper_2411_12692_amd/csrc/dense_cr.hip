// Instances of the dense tiles (dense_tile.h).
#include "dense_tile.h"

namespace si {

hipError_t dense_cr(int type, const DenseArgs& a, int tile, hipStream_t s) {
  return type == kTypeBF16 ? dense_launch<kTypeBF16, kCol, kRow, 1>(a, tile, 1, s)
                           : dense_launch<kTypeF16, kCol, kRow, 1>(a, tile, 1, s);
}

}  // namespace si
