// Which kernel and tile a product with MXFP4 weights runs on.  Free of device code, so that a host program can check it.
#pragma once

#include <cmath>

#include "dfk_linear_plan.h"

namespace dfk {

// MXFP8 activations: whether their large and small elements are multiplied apart (dfk_mx_device.h), which loses nothing and takes twice as many instructions.  Beyond 64 rows that is for fp32
// results only: 4096 x 14336 -> 4096 172 us, apart 353; 256 x 14336 -> 4096 26 and 43; 128 x 4096 -> 4096 12 and 15.  What it leaves otherwise, on the root-mean-square and relative to the
// results', is 4.6e-6 for normally distributed activations, 1.4e-5 with 0.4 % of the columns 16 times as large, 1.7e-5 for SiLU(gate) x up, 7e-5 with 1 % of the columns 300 times as large: 1/360 to
// 1/24 of what rounding to bf16 leaves, 1/45 to a third of half's.  Up to 32 rows the weights' bytes are what counts.  From 33 to 64, where most calls run on tiles, it costs up to a fifth, and is
// kept all the same: rows of a decode batch are as exact as a single one (64 and 65 rows: gated 4096 -> 14336 26.2 and 21.7 us, 8192 -> 28672 73.4 and 73.3, 8192 -> 7168 27.0 and 34.0; 14336 -> 4096
// 19.3 and 18.7, 4096 -> 4096 11.6 and 11.1, 2880 -> 7680 16.9 and 18.5).
constexpr int kMxExactRows = 64;
inline bool mx_exact_sums(int M, int out_fp32) { return M <= kMxExactRows || out_fp32; }

// The tile kernel (dfk_mx_tile.hip), steps of KS k: bytes of LDS of a step's operands and of two steps' scales (`words`: as they are, else a word for each).
constexpr int mx_tile_stage(bool x8, int KS, int BM, int BN) { return BM * (x8 ? KS : KS / 2) + BN * (KS / 2); }
constexpr int mx_tile_scales(int KS, int BM, int BN, bool words) { return (BM + BN) * (KS / 32) * (words ? 2 : 8); }

// LDS of a group of wavefronts: NS steps' operands, three pairs of steps' scales, and where rows do not end with a step 1 KB for what is written to no purpose.
constexpr int kMxNoneBytes = 1024;
constexpr int mx_tile_lds(bool x8, int KS, int BM, int BN, int NS, bool words) { return NS * mx_tile_stage(x8, KS, BM, BN) + 3 * mx_tile_scales(KS, BM, BN, words) + (words ? 0 : kMxNoneBytes); }

// Its tiles: rows, columns (of the gated half: twice as many weight rows), groups of wavefronts with a share of the steps each, and for either format of the activations workgroups that a CU holds
// (0: not offered), microseconds of a step of 256 k and of a round's filling and stores, and the terabytes per second that the tile draws from memory; then how many times as long a step
// is with elements multiplied apart.  K no multiple of 256: the first tile and that of 128 x 128, in steps of 128 k.
struct MxTile { int bm, bn, groups, per_cu[2]; double step[2], fill[2], rate[2], exact; };
constexpr MxTile kMxTiles[] = {
    {64, 64, 1, {2, 2}, {0.397, 0.473}, {1.26, 1.52}, {7.09, 6.83}, 1.51},
    {64, 128, 1, {2, 2}, {0.621, 0.658}, {1.84, 2.29}, {5.98, 5.26}, 1.66},
    {128, 128, 1, {1, 1}, {0.623, 0.797}, {2.15, 2.62}, {9.01, 13.1}, 2.08},
    {128, 256, 1, {1, 1}, {1.076, 1.495}, {2.94, 3.99}, {6.46, 6.82}, 1.8},
    {256, 256, 1, {1, 1}, {1.388, 2.069}, {5.79, 8.3}, {6.26, 6.5}, 0.0},
    {128, 128, 1, {2, 0}, {0.741, 0.0}, {2.43, 0.0}, {7.52, 1.0}, 0.0},      // four wavefronts
    {32, 128, 1, {2, 2}, {0.481, 0.595}, {1.54, 1.46}, {6.85, 4.84}, 1.28},
    {64, 64, 2, {1, 1}, {0.665, 0.8}, {2.11, 2.74}, {6.33, 5.68}, 1.32}};
constexpr int kMxTileCount = (int)(sizeof(kMxTiles) / sizeof(kMxTiles[0]));
constexpr int kMxTileSmall = 0, kMxTile128 = 2, kMxTile256 = 4;

// Which of them there are (`steps256`: K a multiple of 256).  With elements multiplied apart there is none of 256 x 256, and for the gated half, where that is done up to 64 rows, none of 128 rows in
// steps of 256, which never is the cheapest (of 60 million shapes).
constexpr bool mx_tile_offered(int tile, bool x8, bool gated, bool exact, bool steps256) {
    if (kMxTiles[tile].per_cu[x8] == 0 || (!steps256 && tile != kMxTileSmall && tile != kMxTile128)) return false;
    return !(exact && (tile == kMxTile256 || (gated && steps256 && kMxTiles[tile].bm == 128)));
}

// The weight stream (dfk_mx_stream.hip): NT tiles of 16 weight rows a wavefront, WK x WU wavefronts, rings of DEPTH chunks of 256 LINES k; for either format of the activations microseconds
// of a chunk, of a chunk for each tile of 16 rows of the activations, the terabytes per second that it draws from memory, and how much longer a chunk takes where two workgroups share a
// CU.  The gated half has the last two.
struct MxStream { int nt, lines, wk, wu, depth; double chunk[2], by_tile[2], rate[2], second[2]; };
constexpr MxStream kMxStreams[] = {
    {1, 1, 4, 2, 3, {0.29, 0.212}, {0.079, 0.305}, {10.41, 11.74}, {0.66, 0.51}},  {1, 1, 8, 1, 2, {0.351, 0.314}, {0.006, 0.113}, {9.38, 10.2}, {0.45, 0.39}},
    {1, 2, 8, 1, 1, {0.54, 0.327}, {0.0, 0.328}, {7.98, 8.93}, {0.23, 0.34}},      {2, 1, 4, 2, 2, {0.523, 0.049}, {0.196, 0.733}, {10.39, 12.0}, {0.17, 0.95}},
    {2, 2, 4, 1, 1, {0.711, 0.461}, {0.136, 0.522}, {8.12, 9.46}, {0.0, 0.06}},
    {2, 1, 4, 2, 1, {0.737, 0.355}, {0.043, 0.404}, {8.27, 9.23}, {0.21, 0.29}},   {2, 2, 4, 2, 1, {1.138, 0.79}, {0.039, 0.689}, {9.38, 12.0}, {1.0, 1.0}}};
constexpr int kMxStreamRows = 64, kMxStreamGated = 5, kMxStreamCount = (int)(sizeof(kMxStreams) / sizeof(kMxStreams[0]));
constexpr size_t kMxLds = 160 * 1024 - 256;
constexpr int mx_stream_tiles(int M) { return M <= 16 ? 1 : M <= 32 ? 2 : 4; }       // of 16 rows of the activations
constexpr int mx_stream_stage(int NT, int LN, bool words) { return NT * LN * 2048 + (words ? 256 * ((NT * LN + 1) / 2) : 512 * NT * LN); }
constexpr int mx_x_pitch(bool x8, int K) { return ((x8 ? K : K / 2) + 1023) / 1024 * 1024 + 16; }
constexpr size_t mx_stream_fixed(int NT, int LN, int TT, int NW, int D, bool words) { return (size_t)NW * (D * mx_stream_stage(NT, LN, words) + NT * TT * 1024); }
constexpr size_t mx_stream_lds(const MxStream& f, bool x8, int M, int K) {
    return mx_stream_fixed(f.nt, f.lines, mx_stream_tiles(M), f.wk * f.wu, f.depth, K % 128 == 0) + (size_t)M * mx_x_pitch(x8, K) + ((size_t)M * (K / 32) + 1039) / 1024 * 1024;
}
// Which of them there are for so many tiles of rows (`words`: K a multiple of 128): those whose LDS holds as many rows of the shortest K, but for two that never are the
// cheapest (of 60 million shapes).
constexpr bool mx_stream_offered(int form, bool x8, int tiles, bool words) {
    const int rows = tiles == 1 ? 1 : tiles == 2 ? 17 : 33;
    if (mx_stream_lds(kMxStreams[form], x8, rows, words ? 128 : 32) > kMxLds) return false;
    return !(tiles == 4 && ((form == 2 && x8 && !words) || (form == 4 && !x8 && words)));
}
inline int mx_stream_per_cu(size_t lds) { return lds <= 80 * 1024 - 128 ? 2 : 1; }

// Microseconds of a call, as a sum of what its launch is made of.  Constants are fitted to measured shapes, every form, tile and split in turn, weights from memory: the streams' to the times of 30800
// shapes; the tiles', to the choices among them, 8000 shapes of 17 to 1000 rows and 3600 of up to 4096.  The choices are 1 to 3 % slower than the best measured ones on the average (tiles of 65 to
// 512 rows in MXFP4 2, where a fit to the times had left 5).
//
// Tiles: start and end; per round of workgroups the filling of its pipeline and its stores, and per step its multiplications and loads, longer where workgroups share a CU and most so where a round
// is not full; the weights' way from memory beside the activations, which every column tile reads again: a norm of the two between their sum and the larger one; stores of the results; with k
// splits the partial sums' way to memory and back.  Half lines (K no multiple of 256) are taken to be
// 1.3 times as long: the shapes measured have K a multiple of 256, all of them.
inline double mx_tile_cost(const MxTile& t, int M, int N, int K, bool x8, bool gated, bool exact, int splits) {
    const double mt = (M + t.bm - 1) / t.bm, cols = gated ? t.bn / 2 : t.bn, nt = std::ceil(N / cols);
    const int per = K % 256 ? 1 : t.per_cu[x8], parts = splits * t.groups;
    const double wgs = mt * nt * splits, slots = kLinearCus * per, share = wgs / slots, steps = ((K + 255) / 256 + parts - 1) / parts, power = x8 ? 4.92 : 2.17;
    const double rounds = share <= 1 ? 1.0 : x8 ? 0.882 * std::ceil(share) + 0.118 * share : std::ceil(share);
    const double both = x8 ? 0.45 : 0.23, some = both * (wgs / kLinearCus - 1), least = x8 ? 0.53 : 0.57;
    const double crowd = per == 1 || wgs <= kLinearCus ? 1.0 : share >= 1 ? 1 + both : 1 + (some > least ? some : least);
    const double step = t.step[x8] * (exact ? t.exact : 1.0) * (K % 256 ? 1.3 : 1.0);
    const double work = rounds * (t.fill[x8] + (gated ? 0.62 : 0.0) + steps * crowd * step);
    const double mem = K * (0.531 * N * (gated ? 2 : 1) + (x8 ? 0.46 * 1.03 : 0.34 * 0.53) * nt * M) / (t.rate[x8] * 1e6);
    const double us = 2.7 + std::pow(std::pow(work, power) + std::pow(mem, power), 1 / power) + (x8 ? 0.55e-6 : 0.66e-6) * M * N;
    return splits > 1 ? us + 0.25e-6 * 8.0 * splits * M * N + 2.3 : us;
}

// Streams: start and end; the activations' way into LDS; per round of units (of which the last, partial one counts for less) and chunk
// the multiplications and waits, and the weights' way from memory, which hide each other in part: a norm of the two between their sum and the larger one.
inline double mx_stream_cost(const MxStream& f, int M, int N, int K, bool x8, bool gated, size_t lds) {
    const int per = mx_stream_per_cu(lds), tt = mx_stream_tiles(M), cols = 16 * f.wu * (gated ? 1 : f.nt), units = (N + cols - 1) / cols, k = 256 * f.lines;
    const double slots = kLinearCus * per, share = units / slots, chunks = ((K + k - 1) / k + f.wk - 1) / f.wk, power = x8 ? 1.15 : 1.29;
    const double rounds = share <= 1 ? 1.0 : 0.8 * std::ceil(share) + 0.2 * share, second = per == 1 || units <= kLinearCus ? 0.0 : share >= 1 ? 1.0 : 2 * share - 1;
    const double work = rounds * (1 + second * f.second[x8]) * ((x8 ? 0.328 : 0.262) * tt + chunks * (f.chunk[x8] + f.by_tile[x8] * tt));
    const double mem = 0.531e-6 * K * N * (gated ? 2 : 1) / f.rate[x8];
    return (x8 ? 2.8 : 2.67) + std::pow(std::pow(work, power) + std::pow(mem, power), 1 / power) + (x8 ? 18.1e-6 * 1.03 : 16.1e-6 * 0.53) * M * K;
}

struct MxPlan { int form, tile, splits; };      // form of the stream, or -1: tile

inline MxPlan mx_plan(int M, int N, int K, bool x8, bool gated, bool out_fp32) {
    const bool exact = x8 && mx_exact_sums(M, out_fp32);
    MxPlan p{-1, kMxTile128, 1};
    double best = 1e30;
    if (M <= kMxStreamRows)
        for (int f = gated ? kMxStreamGated : 0; f < (gated ? kMxStreamCount : kMxStreamGated); ++f) {
            const size_t lds = mx_stream_lds(kMxStreams[f], x8, M, K);
            if (lds > kMxLds || !mx_stream_offered(f, x8, mx_stream_tiles(M), K % 128 == 0)) continue;
            const double c = mx_stream_cost(kMxStreams[f], M, N, K, x8, gated, lds);
            if (c < best) { best = c; p = MxPlan{f, 0, 1}; }
        }
    for (int i = 0; i < kMxTileCount; ++i) {
        const MxTile& t = kMxTiles[i];
        if (!mx_tile_offered(i, x8, gated, exact, K % 256 == 0)) continue;
        for (int s = 1; s <= (gated ? 1 : kLinearMaxSplits); s *= 2) {
            // splits fill up one round of workgroups, of at least two steps each
            if (s > 1 && ((long long)((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn) * s > kLinearCus * t.per_cu[x8] || K / 256 < 2 * s)) break;
            const double c = mx_tile_cost(t, M, N, K, x8, gated, exact, s);
            if (c < best) { best = c; p = MxPlan{-1, i, s}; }
        }
    }
    return p;
}

}  // namespace dfk
