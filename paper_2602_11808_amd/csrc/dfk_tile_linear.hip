// Linear layers with many rows: the tile kernel with the layer's epilogue.
#include "dfk_tile.h"

namespace dfk {

template <typename E>
static hipError_t launch_linear_of(const TileArgs& a, hipStream_t st) {
    return launch_tile<E, kEpiLinear, 256, 256, 2, 4, 2>(a, (a.M + 255) / 256, st);
}

hipError_t launch_linear_tile(const TileArgs& a, dfk_dtype_t dtype, hipStream_t st) {
    return dtype == DFK_BF16 ? launch_linear_of<BF16>(a, st) : launch_linear_of<FP16>(a, st);
}

}  // namespace dfk
