// Linear layers with few rows: the weight stream with the layer's epilogue.
#include <algorithm>

#include "dfk_stream.h"

namespace dfk {
namespace {

// WR: rows of a weight tile, 16, or 8 with NT = 1.
template <typename E, int NT, int TT, int XR, int D, int NW, int WR>
__global__ __launch_bounds__(NW * 64) void k_linear_stream(TileArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = (int)blockIdx.x * (WR * NT);
    const unsigned rb = (unsigned)a.K * 2;
    f32x4 acc[NT][TT];
    const char* wb[NT];
    unsigned wr[NT][2], xr[XR / 8];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        wb[n] = (const char*)a.B + (size_t)n0 * rb;
#pragma unroll
        for (int h = 0; h < 2; ++h) wr[n][h] = (unsigned)min(16 * n + 8 * h + (lane >> 3), a.N - 1 - n0) * rb;
    }
#pragma unroll
    for (int h = 0; h < XR / 8; ++h) xr[h] = (unsigned)min(8 * h + (lane >> 3), a.M - 1) * rb;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    stream_dot<E, NW, NT, TT, XR, D, 0, WR>(acc, lds, wave, wb, wr, (const char*)a.A, xr, a.K, wave, NW);
    f32x4* const sums = (f32x4*)lds;
    lds_barrier();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int t = 0; t < TT; ++t) sums[(wave * NT * TT + n * TT + t) * 64 + lane] = acc[n][t];
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < NT * TT * 64; i += NW * 64) {
        f32x4 s = sums[i];
#pragma unroll
        for (int w = 1; w < NW; ++w) s += sums[w * NT * TT * 64 + i];
        const int tile = i >> 6, n = tile / TT, t = tile - n * TT, m = 16 * t + (i & 15), col = n0 + 16 * n + 4 * ((i >> 4) & 3);
        const float v[4] = {s[0], s[1], s[2], s[3]};
        if (m < a.M && (WR == 16 || ((i >> 4) & 3) < 2)) {
            if (a.out_fp32) linear_store4<E, FP32>(a, m, col, v);
            else linear_store4<E, E>(a, m, col, v);
        }
    }
}

template <typename E, int NT, int TT, int XR, int D, int NW, int WR = 16>
hipError_t launch(const TileArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    constexpr size_t end = (size_t)NW * NT * TT * 1024;
    static_assert(end <= (size_t)kLdsLimit && (size_t)NW * stream_ring_bytes<NW, NT, XR, D, WR>(8) <= (size_t)kLdsLimit, "the rings fit LDS");
    const size_t lds = std::max(end, (size_t)NW * stream_ring_bytes<NW, NT, XR, D, WR>(a.K));
    if (hipError_t e = allow_lds(allowed, (const void*)k_linear_stream<E, NT, TT, XR, D, NW, WR>, lds); e != hipSuccess) return e;
    return launch_kernel(k_linear_stream<E, NT, TT, XR, D, NW, WR>, dim3((unsigned)((a.N + WR * NT - 1) / (WR * NT))), dim3(NW * 64), lds, st, a);
}

// Wavefronts and depth of the rings: two workgroups and more fit a CU's LDS (16 rows, 4096 -> 50257, two chunks deep 75 us, four chunks 86).
template <typename E>
hipError_t launch_of(const TileArgs& a, int nt, hipStream_t st) {
    // Eight rows of W where sixteen would be no workgroup for every second CU.  us, 16 / 8 rows: 1 x 8192 -> 2048 9.8 / 8.4, 8 x 16384 -> 1024 16.8 / 12.4, 1 x 4096 -> 1536 5.8 / 5.3,
    // 4 x 4096 -> 3584 7.3 / 7.8, 1 x 8192 -> 4096 12.8 / 13.3.
    if (a.M <= 8) return a.N <= 2048 ? launch<E, 1, 1, 8, 5, 8, 8>(a, st) : launch<E, 1, 1, 8, 3, 8>(a, st);
    if (a.M <= 16) return nt == 1 ? launch<E, 1, 1, 16, 2, 8>(a, st) : launch<E, 2, 1, 16, 2, 8>(a, st);
    if (a.M <= 32) return nt == 1 ? launch<E, 1, 2, 32, 2, 8>(a, st) : nt == 2 ? launch<E, 2, 2, 32, 2, 4>(a, st) : launch<E, 4, 2, 32, 2, 4>(a, st);
    if (a.M <= 48) return nt == 1 ? launch<E, 1, 3, 48, 2, 8>(a, st) : nt == 2 ? launch<E, 2, 3, 48, 2, 4>(a, st) : launch<E, 4, 3, 48, 2, 4>(a, st);
    if (a.M <= 64) return nt == 1 ? launch<E, 1, 4, 64, 2, 4>(a, st) : nt == 2 ? launch<E, 2, 4, 64, 2, 4>(a, st) : launch<E, 4, 4, 64, 2, 4>(a, st);
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_linear_stream(const TileArgs& a, dfk_dtype_t dtype, int nt, hipStream_t st) {
    return dtype == DFK_BF16 ? launch_of<BF16>(a, nt, st) : launch_of<FP16>(a, nt, st);
}

}  // namespace dfk
