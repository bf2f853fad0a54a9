// Matrix products of 16-bit operands for few rows: the weights stream through LDS once.
//
// A workgroup owns 16 NT rows of the weights; its NW wavefronts divide the k range in chunks of 64 (chunk c belongs to wavefront c mod NW, so that
// together they read whole stretches of a row) and hold TT tiles of 16 rows of the activations against them.  Each wavefront has a ring of D chunks of
// its own in LDS, filled by asynchronous global->LDS loads, and waits for nobody but its own loads.  The way through LDS
// is there for the memory pipe: a load instruction of it covers 8 rows x 128 bytes, eight neighbouring lanes a line, where loads straight into
// the operand layout of v_mfma_f32_16x16x32 have neighbouring lanes in different rows, which costs four times the
// address cycles (16 rows, 4096 -> 50257: 112 us, and 69 with one row, whose activations are one address per group).
// In LDS a tile of 16 rows is 2 KB, the eight 16-byte pieces of row i XOR-swizzled by i / 2.
// The wavefronts' sums meet in LDS at the end and are added in order.
#pragma once

#include "dfk_epilogue.h"
#include "dfk_mfma_common.h"

namespace dfk {
namespace {

constexpr int kChunkK = 64;
constexpr int kStreamTile = 2048;

// XR: rows of activations loaded, 8 or 16 TT; WR: rows of a weight tile loaded, 8 or 16 (with 8 a tile's other eight are copies).
template <int NT, int XR, int D, int WR = 16>
struct StreamRing {
    static constexpr int kLoads = NT * WR / 8 + XR / 8;
    static constexpr int kStage = NT * WR * 128 + XR * 128;
    static constexpr int kBytes = D * kStage;      // of a wavefront
};

// Waits until the loads of all but the newest `newer` (at most D - 1, uniform) chunks are there.
template <int LOADS, int D>
__device__ __forceinline__ void stream_wait(int newer) {
    static_assert(LOADS * (D - 1) <= 63, "counts of s_waitcnt");
    if constexpr (D > 1) {
        if (newer < D - 1) return stream_wait<LOADS, D - 1>(newer);
    }
    DFK_WAIT_VM(LOADS * (D - 1));
    asm volatile("" ::: "memory");
}

// acc[nt][tt] += products of chunks first, first + stride, ...  Weight tile nt: rows wr[nt][0] and wr[nt][1] (byte offsets from the scalar base
// wb[nt]) are those of this lane's two loads: tile rows lane / 8 and lane / 8 + 8; likewise the activations' xr.  K: a multiple of 8; pieces past its end are
// read from before it and zeroed.
// (USER: a number of the caller's own.  Two kernels that shared an instantiation were refused by the compiler's host pass.)
template <typename E, int NT, int TT, int XR, int D, int USER, int WR = 16>
__device__ __forceinline__ void stream_dot(f32x4 (&acc)[NT][TT], unsigned char* ring, const char* const (&wb)[NT], const unsigned (&wr)[NT][2], const char* xb,
                                           const unsigned (&xr)[XR / 8], int K, int first, int stride) {
    using R = StreamRing<NT, XR, D, WR>;
    constexpr int kTile = WR * 128;
    const int lane = threadIdx.x & 63, q = lane & 15, g = lane >> 4;
    const int chunks = (K + kChunkK - 1) / kChunkK, mine = chunks > first ? (chunks - first + stride - 1) / stride : 0;
    const unsigned piece = (unsigned)((((lane & 7) ^ (lane >> 4)) & 7) * 16);     // of tile rows 0..7 (row / 2 = lane / 16); rows 8..15: ^ 64
    const unsigned k_last = (unsigned)(K - 8) * 2;
    const auto load = [&](int i) {
        unsigned char* dst = ring + (i % D) * R::kStage;
        const unsigned k = (unsigned)(first + i * stride) * (kChunkK * 2);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < WR / 8; ++h) {
                unsigned o = wr[n][h] + min(k + (piece ^ (64 * h)), k_last);
                asm("" : "+v"(o));             // 32 bits from a scalar base
                if (K % kChunkK == 0) __builtin_amdgcn_global_load_lds(wb[n] + o, DFK_LDS_PTR(dst + n * kTile + h * 1024), 16, 0, kAuxNonTemporal);
                else __builtin_amdgcn_global_load_lds(wb[n] + o, DFK_LDS_PTR(dst + n * kTile + h * 1024), 16, 0, 0);
            }
#pragma unroll
        for (int h = 0; h < XR / 8; ++h) {
            unsigned o = xr[h] + min(k + (piece ^ (64 * (h & 1))), k_last);
            asm("" : "+v"(o));
            __builtin_amdgcn_global_load_lds(xb + o, DFK_LDS_PTR(dst + NT * kTile + h * 1024), 16, 0, 0);
        }
    };
    const int lo16 = q * 128 + ((g ^ (q >> 1)) & 7) * 16, lo8 = (q & 7) * 128 + ((g ^ ((q & 7) >> 1)) & 7) * 16;
    const int lo = WR == 8 ? lo8 : lo16, xlo = XR == 8 ? lo8 : lo16;
    const auto use = [&](int i) {
        const unsigned char* src = ring + (i % D) * R::kStage;
        u32x4 w[2][NT], x[2][TT];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int n = 0; n < NT; ++n) w[j][n] = *(const u32x4*)(src + n * kTile + (lo ^ (64 * j)));
#pragma unroll
            for (int t = 0; t < TT; ++t) x[j][t] = *(const u32x4*)(src + NT * kTile + t * kStreamTile + (xlo ^ (64 * j)));
        }
        if ((first + i * stride + 1) * kChunkK > K) {       // the chunk that ends early
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if ((first + i * stride) * kChunkK + j * 32 + g * 8 >= K) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) w[j][n] = u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < TT; ++t) x[j][t] = u32x4{0, 0, 0, 0};
                }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[n][t] = mfma16<E>(w[j][n], x[j][t], acc[n][t]);
    };
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (d < mine) load(d);
    int i = 0;
#pragma unroll 1
    for (; i + D < mine; ++i) {
        DFK_WAIT_VM(R::kLoads * (D - 1));
        asm volatile("" ::: "memory");
        use(i);
        __builtin_amdgcn_sched_barrier(0);     // (the operands are in registers before their place is filled again)
        load(i + D);
    }
#pragma unroll 1
    for (; i < mine; ++i) {
        stream_wait<R::kLoads, D>(mine - 1 - i);
        use(i);
    }
}

}  // namespace
}  // namespace dfk
