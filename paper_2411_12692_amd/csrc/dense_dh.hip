// Instances of the dense tiles (dense_tile.h) that write dg and du in place of dh: apart
// from the others, whose loop keeps its registers this way (in one kernel the 256 x 256
// tile spilled 25 of them, dx of 4096 tokens 526 -> 1340 us).  4096 tokens, 11008 x 4096,
// bf16: 426 us, of which 540 MB of sums, dg and du take 110 behind the products; with dh
// stored and k_gated_grad 330 + 110.
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
