// Which kernel and tile a linear layer of 16-bit operands runs on.  Free of device code, so that a host program can check it.
#pragma once

#include <stddef.h>

namespace dfk {

// A choice: the weight stream (weight tiles of 16 rows per workgroup), or a tile with its k splits.
struct LinearPlan {
    bool stream;
    int nt;          // stream: weight tiles per workgroup
    int tile;        // index into kLinearTiles
    int splits;
};

struct LinearTile { int bm, bn, per_cu; };   // rows, columns, workgroups that a CU holds
constexpr LinearTile kLinearTiles[] = {{64, 64, 2}, {64, 128, 2}, {64, 256, 1}, {128, 64, 1}, {128, 128, 1}, {256, 128, 1}, {128, 256, 1}, {256, 256, 1}, {256, 224, 1}};
// The last one is there for rounds that come out even: us without / with it, 4096 -> N: 4096 rows, N = 14336 430 / 399, 7168 210 / 200, 3584 100 / 98; 2048 rows, 14336 214 / 204,
// 7168 104 / 100; 3000 x 4096 95 / 92; 2000 x 5001 99 / 93; 1200 x 7680 96 / 88; 1024 x 14336 109 / 103; 512 x 28672 120 / 113.
constexpr int kLinearTileCount = (int)(sizeof(kLinearTiles) / sizeof(kLinearTiles[0]));
constexpr int kLinearCus = 256, kLinearMaxSplits = 8;
constexpr int kLinearLinesRows = 128;        // the tile of 128 x 128 takes rows off the cache lines by their own lines (dfk_tile.h)

inline long long linear_tiles(const LinearTile& t, int M, int N) { return (long long)((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn); }

// Microseconds, as a sum of what a launch is made of; the constants are fitted to 1900 measured launches (9 to 4096 rows, 64 to 60000 columns, K 64 to 60000;
// 15 % off on the root-mean-square, and its choices 2 % slower than the best measured ones on the average):
//   start and end; per round of workgroups the filling of its pipeline and its stores; per step of 64 k the largest of its multiplications (1.56 us at
//   256 x 256), its loads out of L2 (0.99 us for 512 rows) and, with few row tiles, its weights out of memory (0.66 us for 256 rows);
//   all of it no less than the weights take at 6.1 TB/s beside the activations, which every column tile reads again;
//   with k splits the partial sums' way to memory and back (the further launch is made up for by the shorter rounds' ends).
// Rows off the cache lines cost 1.3 of the loads out of L2 where steps straddle two lines (a little less where the smallest tiles have a CU each), 1.1 and a microsecond a round by
// lines (44 more shapes, 65 to 4000 rows: 5 % faster on the average than without the tile by lines and these factors, at worst 2 % slower).
inline double linear_tile_cost(const LinearTile& t, int M, int N, int K, int splits) {
    const double mt = (M + t.bm - 1) / t.bm, nt = (N + t.bn - 1) / t.bn;
    const double wgs = mt * nt * splits, slots = kLinearCus * t.per_cu;
    const double steps = ((K + 63) / 64 + splits - 1) / splits;
    const double rounds = (double)(long long)((wgs + slots - 1) / slots);
    // Workgroups that share a CU; a few CUs with two are what the others wait for (600 x 4096 -> 4096, where the average chose 320 workgroups of 64 x 128: 48 us, 128 x 128 38).
    const double crowd = wgs <= kLinearCus ? 1.0 : wgs >= slots ? t.per_cu : wgs < 1.5 * kLinearCus ? 1.5 : wgs / kLinearCus;
    const bool off = K % 64 != 0, lines = off && t.bm == kLinearLinesRows && t.bn == kLinearLinesRows;
    const double mul = 1.56 * t.bm * t.bn / 65536.0, loads = (!off ? 1.0 : lines ? 1.1 : t.bn == 64 && t.bm == 64 && wgs <= kLinearCus ? 1.25 : 1.3) * 0.99 * (t.bm + t.bn) / 512.0, weights = 0.66 * t.bn / 256.0 / (mt < 4 ? mt : 4);
    double step = mul > loads ? mul : loads;
    if (weights > step) step = weights;
    double us = rounds * ((lines ? 5.9 : 4.9) + steps * crowd * step);
    const double mem = 2.0 * K * (1.03 * N + 0.30 * nt * M) / 6.3e6;
    if (mem > us) us = mem;
    us += 3.6;
    if (splits > 1) us += 0.27e-6 * 8.0 * splits * M * N - 1.4;
    return us;
}

// The weight stream with nt weight tiles of 16 rows against xr rows of activations per workgroup: what both bring into a CU, or the weights out of memory
// beside the activations out of L2.
inline double linear_stream_cost(int nt, int xr, int M, int N, int K) {
    const double wgs = (N + 16 * nt - 1) / (16 * nt), per_cu = (double)(long long)((wgs + kLinearCus - 1) / kLinearCus);
    const double cu = per_cu * ((K + 63) / 64) * 1.2 * (16 * nt + xr) / 512.0;
    const double mem = 2.0 * K * (0.97 * N + 0.35 * wgs * xr) / 6.3e6;
    return 3.0 + (cu > mem ? cu : mem);
}

inline LinearPlan linear_plan(int M, int N, int K) {
    LinearPlan p{true, 1, 0, 1};
    // Up to 8 rows the activations are half a tile of LDS traffic beside each tile of weights and the stream is at the rate of
    // memory: 4096 -> 50257 63 us, where the best tile takes 66.
    if (M <= 8) return p;
    double best = 1e30;
    // Layers of 100 MB and more: tiles, which read the activations once per 64 to 256 columns (16 x 4096 -> 50257: stream 75, tile 66 us;
    // 48 x 8192 -> 28672 94 and 72).
    if (M <= 64 && (double)N * K < 5e7) {
        for (int nt = 1; nt <= 4; nt *= 2) {
            if (nt == 4 && M <= 16) continue;
            const double c = linear_stream_cost(nt, (M + 15) / 16 * 16, M, N, K);
            if (c < best) { best = c; p.nt = nt; }
        }
    }
    for (int i = 0; i < kLinearTileCount; ++i)
        for (int s = 1; s <= kLinearMaxSplits; s *= 2) {
            // splits fill up one round of workgroups, of at least four steps each
            if (s > 1 && (linear_tiles(kLinearTiles[i], M, N) * s > kLinearCus || (K + 63) / 64 < 4 * s)) break;
            const double c = linear_tile_cost(kLinearTiles[i], M, N, K, s);
            if (c < best) { best = c; p = LinearPlan{false, 0, i, s}; }
        }
    return p;
}

// Partial sums of the k splits: fp32 [splits][M][pitch], pitch = N rounded up to a multiple of 4.
inline size_t linear_partial_bytes(int M, int N, int splits) { return splits > 1 ? (size_t)splits * M * ((N + 3) / 4 * 4) * 4 : 0; }
// No less than that for any choice up to M rows: at most kLinearMaxSplits, and at most kLinearCus tiles of 256 x 256.
inline size_t linear_partial_bound(int M, int N) {
    const size_t by_rows = linear_partial_bytes(M, N, kLinearMaxSplits), by_tiles = (size_t)kLinearCus * 256 * 256 * 4;
    return by_rows < by_tiles ? by_rows : by_tiles;
}

}  // namespace dfk
