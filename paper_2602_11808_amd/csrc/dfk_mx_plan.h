// Which kernel and tile a product with MXFP4 weights runs on.  Free of device code, so that a host program can check it.
#pragma once

#include "dfk_linear_plan.h"

namespace dfk {

// MXFP8 activations: whether their large and small elements are multiplied apart (dfk_mx_device.h), which loses nothing and takes twice as many instructions.  Up to 64 rows the
// weights' bytes are what counts; beyond, it is for fp32 results only, as the error, 1.3e-5 of the result on the root-mean-square for normally distributed ones, is 1/130 of what
// rounding to bf16 leaves and 1/15 of half's.
constexpr int kMxExactRows = 64;
inline bool mx_exact_sums(int M, int out_fp32) { return M <= kMxExactRows || out_fp32; }

// The tile kernel (dfk_mx_tile.hip), steps of KS k: bytes of LDS of a step's operands and of two steps' scales (`words`: as they are, else a word for each).
constexpr int mx_tile_stage(bool x8, int KS, int BM, int BN) { return BM * (x8 ? KS : KS / 2) + BN * (KS / 2); }
constexpr int mx_tile_scales(int KS, int BM, int BN, bool words) { return (BM + BN) * (KS / 32) * (words ? 2 : 8); }

// Its tiles; [format of the activations]: workgroups that a CU holds (0: not offered), and microseconds of a step of 256 k and of a round's filling and stores.  The
// gated half's tiles have bn / 2 columns, and none of 64 x 64.  Rows that are no multiple of 256 k have the first one (linear layers only) and the one of 128 x 128, in steps of 128 k.
struct MxTile { int bm, bn, per_cu[2]; double step[2], fill[2]; };
constexpr MxTile kMxTiles[] = {
    {64, 64, {2, 2}, {0.39, 0.43}, {0.5, 0.8}},   {64, 128, {2, 2}, {0.52, 0.60}, {0.9, 1.2}},   {128, 128, {1, 1}, {0.63, 0.82}, {1.6, 1.6}},
    {128, 256, {1, 1}, {0.89, 1.40}, {2.8, 3.0}}, {256, 256, {1, 1}, {1.43, 2.00}, {5.5, 5.7}}, {128, 128, {2, 0}, {0.62, 0.0}, {2.2, 0.0}}};      // (the last one: four wavefronts)
constexpr int kMxTileCount = (int)(sizeof(kMxTiles) / sizeof(kMxTiles[0]));
constexpr int kMxTileSmall = 0, kMxTile128 = 2, kMxTile256 = 4;

struct MxPlan { int tile, splits; };

// Microseconds, as a sum of what a launch is made of; the constants are fitted to 10000 shapes (17 to 4096 rows, 32 to 50000 columns, K 512 to 14336, every tile and split: 7 % off on the
// root-mean-square, and its choices 1.2 % slower than the best measured ones on the average):
//   start and end; per round of workgroups the filling of its pipeline and its stores; per step its multiplications and loads, longer where workgroups share a CU; all of it no less than the
//   weights take from memory beside the activations, which every column tile reads again; stores of the results; with k splits the partial sums' way to memory and back.
// Elements multiplied apart (mx_exact_sums) take 1.8 times as long, half lines (K no multiple of 256) 1.3 times.
inline double mx_tile_cost(const MxTile& t, int M, int N, int K, bool x8, bool gated, bool exact, int splits) {
    const double mt = (M + t.bm - 1) / t.bm, cols = gated ? t.bn / 2 : t.bn, nt = (double)(long long)((N + cols - 1) / cols);
    const int per = K % 256 ? 1 : t.per_cu[x8];
    const double wgs = mt * nt * splits, slots = kLinearCus * per, steps = ((K + 255) / 256 + splits - 1) / splits;
    const double rounds = (double)(long long)((wgs + slots - 1) / slots);
    const double crowd = wgs <= kLinearCus ? 1.0 : wgs >= slots ? per : wgs < 1.5 * kLinearCus ? 1.5 : wgs / kLinearCus;
    double step = t.step[x8] * (exact ? 1.8 : 1.0) * (K % 256 ? 1.3 : 1.0);
    const double weights = 0.4 * t.bn / 256.0 / (mt < 4 ? mt : 4);
    if (weights > step) step = weights;
    double us = rounds * (t.fill[x8] + (gated ? 0.5 : 0.0) + steps * crowd * step);
    const double mem = K * (0.53 * N * (gated ? 2 : 1) + (x8 ? 0.65 * 1.03 : 0.15 * 0.53) * nt * M) / (x8 ? 5.9e6 : 4.7e6);
    if (mem > us) us = mem;
    us += 3.2 + 0.45e-6 * M * N;
    if (splits > 1) us += 0.24e-6 * 8.0 * splits * M * N + 2.5;
    return us;
}

inline MxPlan mx_tile_plan(int M, int N, int K, bool x8, bool gated, bool exact) {
    MxPlan p{kMxTile128, 1};
    double best = 1e30;
    for (int i = 0; i < kMxTileCount; ++i) {
        const MxTile& t = kMxTiles[i];
        if (t.per_cu[x8] == 0 || (gated && i == kMxTileSmall) || (x8 && exact && i == kMxTile256) || (K % 256 && i != kMxTileSmall && i != kMxTile128)) continue;
        for (int s = 1; s <= (gated ? 1 : kLinearMaxSplits); s *= 2) {
            // splits fill up one round of workgroups, of at least two steps each
            if (s > 1 && ((long long)((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn) * s > kLinearCus * t.per_cu[x8] || K / 256 < 2 * s)) break;
            const double c = mx_tile_cost(t, M, N, K, x8, gated, exact, s);
            if (c < best) { best = c; p = MxPlan{i, s}; }
        }
    }
    return p;
}

// The weight stream (dfk_mx_stream.hip): NT tiles of 16 weight rows a wavefront, TT tiles of activations, NW wavefronts, rings of D chunks of 256 k.
constexpr int kMxStreamDepth = 4, kMxStreamDepthGated = 3;
constexpr int kMxStreamHalf = 80 * 1024 - 128;       // of LDS: two workgroups a CU
constexpr int mx_stream_stage(int NT, bool words) { return NT * 2048 + (words ? 256 * ((NT + 1) / 2) : 512 * NT); }
constexpr int mx_x_pitch(bool x8, int K) { return ((x8 ? K : K / 2) + 1023) / 1024 * 1024 + 16; }
inline size_t mx_stream_lds(bool x8, int NT, int TT, int NW, int D, bool words, int M, int K) {
    return (size_t)NW * D * mx_stream_stage(NT, words) + (size_t)NW * NT * TT * 1024 + (size_t)M * mx_x_pitch(x8, K) + ((size_t)M * (K / 32) + 1039) / 1024 * 1024;
}
// Whether the activations fit beside the rings.
inline bool mx_stream_fits(int M, int K, bool x8, bool gated) {
    const int TT = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    return M <= 64 && mx_stream_lds(x8, gated ? 2 : 1, TT, 8, gated ? kMxStreamDepthGated : kMxStreamDepth, K % 128 == 0, M, K) <= 160 * 1024 - 256;
}

}  // namespace dfk
