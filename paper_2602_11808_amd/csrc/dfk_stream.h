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
template <int NT, int XR, int WR = 16>
struct StreamRing {          // (a ring's size: stream_ring_bytes)
    static constexpr int kLoads = NT * WR / 8 + XR / 8;
    static constexpr int kStage = NT * WR * 128 + XR * 128;
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
template <typename E, int NT, int TT, int XR, int D, int USER, int WR>
__device__ __forceinline__ void stream_chunks(f32x4 (&acc)[NT][TT], unsigned char* ring, const char* const (&wb)[NT], const unsigned (&wr)[NT][2], const char* xb,
                                           const unsigned (&xr)[XR / 8], int K, int first, int stride) {
    using R = StreamRing<NT, XR, WR>;
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

// The same for rows that start anywhere in a line of 128 bytes (K a multiple of 8 only), a stretch of chunks for each of `stride`.  What is loaded is each row's own lines,
// one more than it has chunks; the 16-byte piece of an operand is found by its row's offset in this chunk's place of the ring or in the next one's.
// (Chunks that straddle two lines ask for most lines twice.)  Pieces outside a row are replaced by its first or last one, and zeroed past its end.
template <typename E, int NT, int TT, int XR, int D, int USER, int WR>
__device__ __forceinline__ void stream_off_lines(f32x4 (&acc)[NT][TT], unsigned char* ring, const char* const (&wb)[NT], const unsigned (&wr)[NT][2], const char* xb,
                                                 const unsigned (&xr)[XR / 8], int K, int first, int stride) {
    static_assert(D >= 2, "a chunk's two places");
    using R = StreamRing<NT, XR, WR>;
    constexpr int kTile = WR * 128, WH = WR / 8, XH = XR / 8;
    const int lane = threadIdx.x & 63, q = lane & 15, g = lane >> 4;
    const int chunks = (K + kChunkK - 1) / kChunkK, c0 = chunks * first / stride, mine = chunks * (first + 1) / stride - c0;
    if (mine == 0) return;
    const int piece = (((lane & 7) ^ (lane >> 4)) & 7) * 16, k_last = (K - 8) * 2;
    // of the rows of this lane's loads: offset in a line; of its operands' rows: place of its pieces, and whether that is in the next line
    int w_at[NT][WH], x_at[XH], w_off[2][NT], x_off[2][TT];
    bool w_next[2][NT], x_next[2][TT];
    const auto place = [&](int o, int row, int j, int& off, bool& next) {
        const int p = 4 * j + g + (o >> 4);
        next = p >= 8;
        off = row * 128 + ((p ^ (row >> 1)) & 7) * 16;
    };
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        int o[WH];
#pragma unroll
        for (int h = 0; h < WH; ++h) {
            o[h] = (int)((uintptr_t)wb[n] + wr[n][h]) & 127;
            w_at[n][h] = (piece ^ (64 * h)) - o[h];
        }
        const int lo = __shfl(o[0], (q & 7) * 8), hi = __shfl(o[WH - 1], (q & 7) * 8);
#pragma unroll
        for (int j = 0; j < 2; ++j) place(WR == 16 && q >= 8 ? hi : lo, WR == 8 ? q & 7 : q, j, w_off[j][n], w_next[j][n]);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        int o[XR == 8 ? 1 : 2];
#pragma unroll
        for (int h = 0; h < (XR == 8 ? 1 : 2); ++h) {
            o[h] = (int)((uintptr_t)xb + xr[2 * t + h]) & 127;
            x_at[2 * t + h] = (piece ^ (64 * h)) - o[h];
        }
        const int lo = __shfl(o[0], (q & 7) * 8), hi = __shfl(o[XR == 8 ? 0 : 1], (q & 7) * 8);
#pragma unroll
        for (int j = 0; j < 2; ++j) place(XR > 8 && q >= 8 ? hi : lo, XR == 8 ? q & 7 : q, j, x_off[j][t], x_next[j][t]);
    }
    const auto load = [&](int i) {                  // line c0 + i of every row
        unsigned char* dst = ring + (i % D) * R::kStage;
        const int k = (c0 + i) * (kChunkK * 2);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < WH; ++h) {
                unsigned o = wr[n][h] + (unsigned)min(max(k + w_at[n][h], 0), k_last);
                asm("" : "+v"(o));
                __builtin_amdgcn_global_load_lds(wb[n] + o, DFK_LDS_PTR(dst + n * kTile + h * 1024), 16, 0, 0);
            }
#pragma unroll
        for (int h = 0; h < XH; ++h) {
            unsigned o = xr[h] + (unsigned)min(max(k + x_at[h], 0), k_last);
            asm("" : "+v"(o));
            __builtin_amdgcn_global_load_lds(xb + o, DFK_LDS_PTR(dst + NT * kTile + h * 1024), 16, 0, 0);
        }
    };
    const auto use = [&](int i) {
        const int now = (i % D) * R::kStage, step = ((i + 1) % D) * R::kStage - now;
        const unsigned char* src = ring + now;
        u32x4 w[2][NT], x[2][TT];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int n = 0; n < NT; ++n) w[j][n] = *(const u32x4*)(src + n * kTile + w_off[j][n] + (w_next[j][n] ? step : 0));
#pragma unroll
            for (int t = 0; t < TT; ++t) x[j][t] = *(const u32x4*)(src + NT * kTile + t * kStreamTile + x_off[j][t] + (x_next[j][t] ? step : 0));
        }
        if ((c0 + i + 1) * kChunkK > K) {           // the chunk that ends early
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if ((c0 + i) * kChunkK + j * 32 + g * 8 >= K) {
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
        if (d <= mine) load(d);
    int i = 0;
#pragma unroll 1
    for (; i + D <= mine; ++i) {                    // (lines 0 .. mine)
        DFK_WAIT_VM(R::kLoads * (D - 2));
        asm volatile("" ::: "memory");
        use(i);
        __builtin_amdgcn_sched_barrier(0);
        load(i + D);
    }
#pragma unroll 1
    for (; i < mine; ++i) {
        stream_wait<R::kLoads, D - 1>(mine - 1 - i);
        use(i);
    }
}

// Rows off the lines by their lines: where a wavefront has enough chunks, one line more being their price.  us with straddling chunks / by lines: layers of 64 x 2888 -> 7688 (11 chunks
// a wavefront) 20.0 / 16.1, 16 x 2888 -> 7688 (6) 12.4 / 11.5, 64 x 1000 -> 3000 (4) 5.5 / 5.9; 8 x 4104 -> 7688 (8) 15.9 / 14.5, 1 x 2888 -> 4096 (6) 6.6 / 6.9.
template <int XR>
__host__ __device__ constexpr bool by_lines(int K, int stride) {
    return K % kChunkK != 0 && (K + kChunkK - 1) / kChunkK >= (XR == 8 ? 8 : 5) * stride;
}
// Depth of their rings: a line more has to be there before a chunk can be used.  (NW: wavefronts, whose rings have to fit LDS.)
constexpr int lines_depth(int D, int stage, int NW) { return D < 3 && (D + 1) * stage * NW <= kLdsLimit ? D + 1 : D; }

// Bytes of a wavefront's ring.  (Of three and more places a ring is as large either way, so that there `stride` may be any; else it is NW.)
template <int NW, int NT, int XR, int D, int WR = 16>
__host__ __device__ constexpr int stream_ring_bytes(int K) {
    constexpr int stage = StreamRing<NT, XR, WR>::kStage;
    return (by_lines<XR>(K, NW) ? lines_depth(D, stage, NW) : D) * stage;
}

// The rings lie one after the other at `rings`, wavefront `wave`'s of stream_ring_bytes(K).
template <typename E, int NW, int NT, int TT, int XR, int D, int USER, int WR = 16>
__device__ __forceinline__ void stream_dot(f32x4 (&acc)[NT][TT], unsigned char* rings, int wave, const char* const (&wb)[NT], const unsigned (&wr)[NT][2], const char* xb,
                                           const unsigned (&xr)[XR / 8], int K, int first, int stride) {
    unsigned char* const ring = rings + wave * stream_ring_bytes<NW, NT, XR, D, WR>(K);
    constexpr int DL = lines_depth(D, StreamRing<NT, XR, WR>::kStage, NW);
    if constexpr (DL >= 2) {
        if (by_lines<XR>(K, stride)) return stream_off_lines<E, NT, TT, XR, DL, USER, WR>(acc, ring, wb, wr, xb, xr, K, first, stride);
    }
    stream_chunks<E, NT, TT, XR, D, USER, WR>(acc, ring, wb, wr, xb, xr, K, first, stride);
}

}  // namespace
}  // namespace dfk
