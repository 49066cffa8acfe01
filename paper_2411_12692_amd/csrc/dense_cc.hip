// Instances of the dense tiles (dense_tile.h).
#include "dense_tile.h"

namespace si {

hipError_t dense_cc(int type, const DenseArgs& a, int tile, int batches, hipStream_t s) {
  return type == kTypeBF16 ? dense_launch<kTypeBF16, kCol, kCol, 1>(a, tile, batches, s)
                           : dense_launch<kTypeF16, kCol, kCol, 1>(a, tile, batches, s);
}

}  // namespace si
