// Linear layers with many rows: the tile kernel with the layer's epilogue.
#include "dfk_linear_plan.h"
#include "dfk_tile.h"

namespace dfk {
namespace {

// The k splits' partial sums in order, then the epilogue: a thread per four columns.
template <typename E>
__global__ __launch_bounds__(256) void k_linear_sum(TileArgs a) {
    const unsigned w4 = (unsigned)a.pitch >> 2;
    const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (size_t)a.M * w4) return;
    const size_t m = idx / w4;
    const int n = (int)(idx - m * w4) * 4;
    const float* src = a.partial + idx * 4;
    const size_t blk = (size_t)a.M * a.pitch;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = 0; k0 < a.splits; k0 += 8) {
        float4 t[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = k0 + k < a.splits ? *(const float4*)(src + (size_t)(k0 + k) * blk) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) { s.x += t[k].x; s.y += t[k].y; s.z += t[k].z; s.w += t[k].w; }
    }
    const float v[4] = {s.x, s.y, s.z, s.w};
    if (a.out_fp32) linear_store4<E, FP32>(a, m, n, v);
    else linear_store4<E, E>(a, m, n, v);
}

template <typename E>
hipError_t launch_sum(const TileArgs& a, hipStream_t st) {
    return launch_kernel(k_linear_sum<E>, dim3((unsigned)(((size_t)a.M * (a.pitch / 4) + 255) / 256)), dim3(256), 0, st, a);
}

template <typename E, int BM, int BN, int WM, int WN, int NS>
hipError_t launch(const TileArgs& a, hipStream_t st) {
    if (linear_partial_bytes(a.M, a.N, a.splits) > a.partial_bytes) return hipErrorInvalidValue;
    hipError_t e;
    if constexpr (BM == kLinearLinesRows && BN == kLinearLinesRows) e = a.K % kTileStepK != 0 ? launch_tile<E, BM, BN, WM, WN, NS, true>(a, st) : launch_tile<E, BM, BN, WM, WN, NS>(a, st);
    else e = launch_tile<E, BM, BN, WM, WN, NS>(a, st);
    if (e != hipSuccess) return e;
    return a.splits > 1 ? launch_sum<E>(a, st) : hipSuccess;
}

// kLinearTiles.  The two of 64 x 64 and 64 x 128 leave room for a second workgroup on the CU; the others are as deep as LDS allows.
template <typename E>
hipError_t launch_of(const TileArgs& a, int tile, hipStream_t st) {
    switch (tile) {
        case 0: return launch<E, 64, 64, 2, 2, 4>(a, st);
        case 1: return launch<E, 64, 128, 2, 2, 3>(a, st);
        case 2: return launch<E, 64, 256, 2, 4, 3>(a, st);
        case 3: return launch<E, 128, 64, 2, 2, 4>(a, st);
        case 4: return launch<E, 128, 128, 2, 4, 4>(a, st);
        case 5: return launch<E, 256, 128, 4, 2, 3>(a, st);
        case 6: return launch<E, 128, 256, 2, 4, 3>(a, st);
        case 7: return launch<E, 256, 256, 4, 2, 2>(a, st);
        case 8: return launch<E, 256, 224, 4, 2, 2>(a, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_linear_tile(const TileArgs& a, dfk_dtype_t dtype, int tile, hipStream_t st) {
    return dtype == DFK_BF16 ? launch_of<BF16>(a, tile, st) : launch_of<FP16>(a, tile, st);
}

hipError_t launch_linear_sum(const TileArgs& a, dfk_dtype_t dtype, hipStream_t st) { return dtype == DFK_BF16 ? launch_sum<BF16>(a, st) : launch_sum<FP16>(a, st); }

}  // namespace dfk
