// Experts with many rows: the tile kernel with the gated epilogue, and with rows that go to their slots.
#include "dfk_tile.h"

namespace dfk {

template <typename E>
static hipError_t launch_experts_of(const TileArgs& a, int epi, hipStream_t st) {
    if (epi == kEpiGated) return launch_tile<E, kEpiGated, 128, 256, 2, 4, 3>(a, a.plan.max_tiles, st);
    return launch_tile<E, kEpiRows, 128, 256, 2, 4, 3>(a, a.plan.max_tiles, st);
}

hipError_t launch_experts_tile(const TileArgs& a, dfk_dtype_t dtype, int epi, hipStream_t st) {
    return dtype == DFK_BF16 ? launch_experts_of<BF16>(a, epi, st) : launch_experts_of<FP16>(a, epi, st);
}

}  // namespace dfk
