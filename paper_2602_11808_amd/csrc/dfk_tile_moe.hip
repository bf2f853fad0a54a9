// Experts with many rows: the tile kernel with the gated epilogue, and with rows that go to their slots.
#include "dfk_tile.h"

namespace dfk {
namespace {

template <typename E, int EPI>
hipError_t launch_of(const TileArgs& a, hipStream_t st) {
    switch (a.plan.tile_rows) {
        case 64: return launch_tile<E, EPI, 64, 128, 2, 2, 3>(a, a.plan.max_tiles, st);
        case 128: return launch_tile<E, EPI, 128, 256, 2, 4, 3>(a, a.plan.max_tiles, st);
        case 256: return launch_tile<E, EPI, 256, 256, 4, 2, 2>(a, a.plan.max_tiles, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_experts_tile(const TileArgs& a, dfk_dtype_t dtype, int epi, hipStream_t st) {
    if (epi == kEpiGated) return dtype == DFK_BF16 ? launch_of<BF16, kEpiGated>(a, st) : launch_of<FP16, kEpiGated>(a, st);
    return dtype == DFK_BF16 ? launch_of<BF16, kEpiRows>(a, st) : launch_of<FP16, kEpiRows>(a, st);
}

}  // namespace dfk
