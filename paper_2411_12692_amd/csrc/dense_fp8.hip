// Instances of the dense tiles (dense_tile.h) for e4m3 values with block scales.
#include "dense_tile.h"

namespace si {

hipError_t dense_fp8(const DenseArgs& a, int mats, int tile, hipStream_t s) {
  return mats == 2 ? dense_launch<kTypeF8, kRow, kRow, 2>(a, tile, 1, s)
                   : dense_launch<kTypeF8, kRow, kRow, 1>(a, tile, 1, s);
}

}  // namespace si
