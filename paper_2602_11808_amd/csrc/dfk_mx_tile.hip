// Products with MXFP4 weights on the scaled matrix instructions, many rows: the tile kernel of the linear layers and of the MLP's gated half.
//
// out[m, n] = sum_k A[m, k] B[n, k].  A workgroup owns BM rows of A and BN rows of B (gated: BN / 2 columns, 32 rows of the gate's weights and the same 32 of the up projection's
// in turn, so that a wavefront has both sums of a column); wavefront (wm, wn) TN x TM products of 32 x 32.
//
// Data movement: asynchronous global->LDS loads NS steps deep, a step being KS = 256 k: one cache line of a row in MXFP4, two in MXFP8, and eight scales; or 128 k, half of that, where 256 rows in MXFP8
// would have too few steps in LDS (4096 x 14336 -> 4096 in MXFP8: tiles of 256 x 256 179 us, of 128 x 256 with 256 k 203; in MXFP4, where half lines are all that it brings, 127 and 114).
// In LDS a row's line is 128 bytes, its eight 16-byte pieces XOR-swizzled by row / 2 (64 bytes, four, by row / 4), so that an operand read of 16 rows covers all banks once.
// Slice t of the SL = KS / 64 of a step multiplies its blocks t and SL + t, so that a lane's scales of a step are the bytes of one word, from which the instruction takes byte t.  While a
// slice multiplies, the operands of the next one are read.  One barrier per step, ahead of its last slice: by then every wavefront has that slice's operands in registers and has waited,
// by count, for its own loads of the following step.
//
// Scales: words of four where a row has a whole number of them (K a multiple of 128), else each byte by a load of its own, which arrives as a word.  Those of two steps are loaded
// together, as each row's are a line of their own for the caches.
//
// Pieces past the end of a row are copies of the last one, and zeroed in A; rows past the end are copies of the last one and are not stored.
#include "dfk_mx_device.h"
#include "dfk_mx_plan.h"
#include "dfk_tile.h"

namespace dfk {
namespace {

constexpr int mx_epilogue_tiles(int TM, int TN, int NW) {
    int pm = TM;
    while (pm > 1 && (size_t)NW * pm * 32 * (TN * 32 + 4) * 4 > (size_t)kLdsLimit) pm /= 2;
    return pm;
}
// Columns col .. col + 31 of row r of the gated half, of which lane (., b) has 8 i + 4 b .. + 3 in a[4 i ..]: as MX, lane b takes columns 16 b .. 16 b + 15 after an exchange with the other.
template <int MX>
__device__ __forceinline__ void mx_store_block(const MxArgs& a, const float (&v)[16], size_t r, int col, int b, bool live) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = mx_top(top, v[i]);
    const unsigned s = mx_scale_of<MX>(max(top, (unsigned)__shfl_xor((int)top, 32)));
    const size_t blk = r * (size_t)(a.t.N / kMxBlock) + col / kMxBlock;
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float f[4] = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
        w[i] = mx_elements<MX>(f, s);
    }
    if constexpr (MX == DFK_MXFP4) {
        const unsigned lo = w[0] | (w[1] << 16), hi = w[2] | (w[3] << 16);     // groups 0, 1 and 2, 3
        const unsigned got = (unsigned)__shfl_xor((int)(b ? lo : hi), 32), e = b ? got : lo, o = b ? hi : got;   // of the even and of the odd four columns
        uint2 out;
        out.x = (e & 0xFFFFu) | (o << 16);
        out.y = (e >> 16) | (o & 0xFFFF0000u);
        if (live) *(uint2*)(a.q + blk * 16 + 8 * b) = out;
    } else {
        const unsigned g0 = (unsigned)__shfl_xor((int)(b ? w[0] : w[2]), 32), g1 = (unsigned)__shfl_xor((int)(b ? w[1] : w[3]), 32);
        const u32x4 out = b ? u32x4{g0, w[2], g1, w[3]} : u32x4{w[0], g0, w[1], g1};
        if (live) *(u32x4*)(a.q + blk * 32 + 16 * b) = out;
    }
    if (live && b == 0) a.qs[blk] = (unsigned char)s;
}

template <bool X8, int KS, int BM, int BN, int WM, int WN, int KG, int NS, bool GATED, bool WHOLE, bool EXACT>
__global__ __launch_bounds__(WM * WN * KG * 64) void k_mx_tile(MxArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char all_lds[];
    constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, XL = X8 ? 2 : 1, SL = KS / 64, BLOCKS = KS / 32;
    constexpr int A_STEP = X8 ? KS : KS / 2, B_ROW = KS / 2, A_ROW = A_STEP < 128 ? A_STEP : 128, A_LINES = A_STEP / A_ROW;      // bytes of a row's step, and of a row in LDS
    constexpr int B_OFF = BM * A_STEP, STAGE = mx_tile_stage(X8, KS, BM, BN), S_OFF = NS * STAGE;
    constexpr int S_PAIR = mx_tile_scales(KS, BM, BN, WHOLE), S_ROW = BLOCKS * (WHOLE ? 2 : 8), NONE = S_OFF + 3 * S_PAIR;
    constexpr int A_PER = 1024 / A_ROW, B_PER = 1024 / B_ROW;       // rows of a load instruction
    constexpr int LA = BM / A_PER / NW, LB = BN / B_PER / NW, LOADS = LA * A_LINES + LB;       // of a wavefront and step
    constexpr int S_PER = 256 / S_ROW, S_ALL = (BM + BN) / S_PER, LS = (S_ALL + NW - 1) / NW, LH = (LS + 1) / 2;      // scales: of two steps, and half of that
    static_assert(BM % (A_PER * NW) == 0 && BN % (B_PER * NW) == 0 && BM % (32 * WM) == 0 && BN % (32 * WN) == 0 && NW % 2 == 0, "whole loads and tiles");
    static_assert(!GATED || TN % 2 == 0 || (TN == 1 && WN % 2 == 0), "gate and up of a column in one wavefront, or in neighbours");
    static_assert(NS >= 2 && NS <= 4, "the waits below");
    static_assert(WHOLE || A_LINES == 1, "the tail below");
    constexpr int COLS = GATED ? BN / 2 : BN;
    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, b = lane >> 5;
    const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6) / NW, wave = __builtin_amdgcn_readfirstlane(tid >> 6) - kg * NW;
    const int wm = wave / WN, wn = wave % WN;
    unsigned char* const lds = all_lds + kg * mx_tile_lds(X8, KS, BM, BN, NS, WHOLE);

    const TileArgs& t = a.t;
    const int n_tiles = (t.N + COLS - 1) / COLS;
    int mt, nt;
    if (!tile_of((t.M + BM - 1) / BM, n_tiles * t.splits, mt, nt)) return;
    const int k_split = nt / n_tiles;
    nt -= k_split * n_tiles;
    const size_t row0 = (size_t)mt * BM;
    const int rows = min(BM, t.M - (int)row0), n0 = nt * COLS;
    int s_lo = 0, steps = (t.K + KS - 1) / KS;
    if (t.splits > 1) {
        int s1;
        share_of((unsigned)steps, (unsigned)t.splits, (unsigned)k_split, s_lo, s1);
        steps = s1 - s_lo;
    }
    // KG groups of wavefronts with a share of the steps each (the last ones one less, or none: steps that are not theirs multiply zeros)
    const int loops = (steps + KG - 1) / KG;
    int own = steps;
    if constexpr (KG > 1) {
        int g0, g1;
        const int end = s_lo + steps;
        share_of((unsigned)steps, KG, (unsigned)(KG - 1 - kg), g0, g1);
        own = g1 - g0;
        s_lo = min(s_lo + g0, end - 1);
        steps = max(own, 1);
    }
    const int left = min(t.K / kMxBlock - (s_lo + steps - 1) * BLOCKS, BLOCKS);      // blocks of the last step
    const int whole = left == BLOCKS ? steps : steps - 1;
    const int rot = t.M <= 4 * BM && whole > 0 ? (int)((unsigned)nt % (unsigned)whole) : 0;     // (dfk_tile.h)
    const auto place = [&](int s) __attribute__((always_inline)) {           // of step s in the row (past the last one: the last one)
        const int c = min(s, steps - 1), r = c + rot;
        return c < whole ? (r >= whole ? r - whole : r) : c;
    };

    // ---- loads: an instruction covers 1 KB, whole rows of a step; lane l brings the piece whose place is l.  Wavefront w has instructions w, w + NW, ...
    const unsigned arb = (unsigned)t.K / (X8 ? 1 : 2), brb = (unsigned)t.K / 2, srb = (unsigned)t.K / kMxBlock;
    const auto piece = [&](int row_bytes) { return row_bytes == 128 ? (unsigned)((((lane & 7) ^ (lane >> 4)) & 7) * 16) ^ ((wave & 1) ? 64u : 0u) : (unsigned)(((lane & 3) ^ ((lane >> 4) & 3)) * 16); };
    const unsigned piece_a = piece(A_ROW), piece_b = piece(B_ROW);
    const char* const base_a = (const char*)t.A + row0 * arb + (size_t)s_lo * A_STEP;
    const char* const base_b = (const char*)t.B + (size_t)n0 * brb + (size_t)s_lo * B_ROW;
    const char* const base_u = GATED ? (const char*)t.B2 + (size_t)n0 * brb + (size_t)s_lo * B_ROW : nullptr;
    const int n_last = t.N - n0 - 1;
    // row of B of a place in the tile (gated: of the gate's or the up projection's weights)
    const auto b_row = [&](int i) { return min(GATED ? (i >> 6) * 32 + (i & 31) : i, n_last); };
    unsigned off_a[LA], off_b[LB], off_s[LS];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        off_a[i] = (unsigned)min(A_PER * (wave + NW * i) + lane / (64 / A_PER), rows - 1) * arb + piece_a;
        asm("" : "+v"(off_a[i]));             // (one register: out of the multiplication it would keep two)
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        off_b[i] = (unsigned)b_row(B_PER * (wave + NW * i) + lane / (64 / B_PER)) * brb + piece_b;
        asm("" : "+v"(off_b[i]));
    }
    // scales: an instruction covers S_PER rows, A's first: the words (bytes) of two steps of each
    const int s_in = lane % (64 / S_PER), s_row = lane / (64 / S_PER);
    const bool s_odd = s_in >= 32 / S_PER;     // this lane's are of the second step of two
    const unsigned s_byte = WHOLE ? 4 * (s_in % (BLOCKS / 4)) : s_in % BLOCKS;
    const unsigned char* s_base[LS];
#pragma unroll
    for (int i = 0; i < LS; ++i) {
        const int first = (wave + NW * i) % S_ALL * S_PER;     // (a few twice where they do not come out even)
        if (first < BM) {
            s_base[i] = a.As + row0 * srb;
            off_s[i] = (unsigned)min(first + s_row, rows - 1) * srb + s_byte;
        } else {
            const int i0 = first - BM;
            s_base[i] = (GATED && (i0 & 32) ? a.B2s : a.Bs) + (size_t)n0 * srb;
            off_s[i] = (unsigned)b_row(i0 + s_row) * srb + s_byte;
        }
        s_base[i] += s_lo * BLOCKS;
        asm("" : "+v"(off_s[i]));
    }
    // in the last, partial step a piece (a scale) past the end is replaced by the last one there is
    const auto past = [](unsigned at, unsigned size, unsigned end) { return at + size > end ? at + size - end : 0u; };
    const unsigned tail_a = past(piece_a, 16, left * (16u * XL)), tail_b = past(piece_b, 16, left * 16u), tail_s = WHOLE ? 0u : past(s_byte, 1, left);
    // The step loop is one block without branches: the compiler moves multiplications across a branch to the block that uses their results.  So every step requests as many loads:
    // what it does not need is a line that is there already.
    // Loads of part Q of the SL of step s into buffer `buf` (with NS = 2 all of them are the first part).
    const auto load_part = [&](auto q_, int s, int buf) __attribute__((always_inline)) {
        constexpr int Q = decltype(q_)::value, FROM = NS == 2 ? (Q ? LOADS : 0) : Q * LOADS / SL, TO = NS == 2 ? LOADS : (Q + 1) * LOADS / SL;
        const size_t st = place(s);
        const unsigned live = s < steps ? ~0u : 0u, end = s == steps - 1 ? ~0u : 0u;
        const char* const pa = base_a + st * A_STEP;
        const char* const pb = base_b + st * B_ROW;
        const char* const pu = base_u + st * B_ROW;
        unsigned char* const dst = lds + buf * STAGE + wave * 1024;
#pragma unroll
        for (int i = FROM; i < TO; ++i) {
            if (i < LA * A_LINES) {
                const int j = i / A_LINES, l = i % A_LINES;
                unsigned o = (off_a[j] + 128u * l - (WHOLE ? 0u : tail_a & end)) & live;
                asm("" : "+v"(o));            // 32 bits from a scalar base, not a 64-bit sum of its own
                __builtin_amdgcn_global_load_lds(pa + o, DFK_LDS_PTR(dst + l * (BM * A_ROW) + NW * j * 1024), 16, 0, 0);
            } else {
                const int j = i - LA * A_LINES;
                unsigned o = (off_b[j] - (WHOLE ? 0u : tail_b & end)) & live;
                asm("" : "+v"(o));
                const char* const p = GATED && ((B_PER * (wave + NW * j)) & 32) ? pu : pb;
                __builtin_amdgcn_global_load_lds(p + o, DFK_LDS_PTR(dst + B_OFF + NW * j * 1024), 16, 0, 0);
            }
        }
    };
    // Half of the scales of steps s and s + 1, for an even s, the other half for an odd one; `pair`: where they go.
    const auto load_scales = [&](int s, int pair) __attribute__((always_inline)) {
        const bool odd = s & 1;
        const int s0 = s & ~1, e0 = place(s0) * BLOCKS, e1 = place(s0 + 1) * BLOCKS;
        unsigned at = s_odd ? e1 : e0;
        if (!WHOLE) at -= s0 + (s_odd ? 1 : 0) >= steps - 1 ? tail_s : 0u;
#pragma unroll
        for (int i = 0; i < LH; ++i) {
            const int j = LH + i < LS ? LH + i : i;      // (one too few: the first half's again)
            unsigned o = (odd ? off_s[j] : off_s[i]) + at;
            asm("" : "+v"(o));
            const unsigned char* const p = odd ? s_base[j] : s_base[i];
            unsigned char* const dst = lds + S_OFF + pair * S_PAIR + (wave + NW * (odd ? j : i)) % S_ALL * 256;
            if constexpr (WHOLE) __builtin_amdgcn_global_load_lds(p + o, DFK_LDS_PTR(dst), 4, 0, 0);
            else __builtin_amdgcn_global_load_lds(p + o, DFK_LDS_PTR(dst), 1, 0, 0);
        }
    };
    constexpr std::integral_constant<int, 0> i0{};
    constexpr std::integral_constant<int, 1> i1{};
    constexpr std::integral_constant<int, 2> i2{};
    constexpr std::integral_constant<int, 3> i3{};
    // (in the order of the step loop, whose waits count)
    load_scales(0, 0);
    load_scales(1, 0);
    if (NS == 2) {
        load_scales(2, 1);
        load_scales(3, 1);
    }
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        load_part(i0, s, s);
        if (NS > 2 && s == NS - 3) load_scales(2, 1);
        if (NS > 2 && s == NS - 2) load_scales(3, 1);
        if (s + 1 < NS) {
            load_part(i1, s, s);
            if constexpr (SL == 4) {
                load_part(i2, s, s);
                load_part(i3, s, s);
            }
        }
    }

    f32x16 acc[TN][TM];
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.f;

    // operands: rows r32 of 32-row tiles; MXFP4 block SL b + t, MXFP8 halves b of blocks t and SL + t
    const int as_o = S_OFF + (wm * TM * 32 + r32) * S_ROW + b * (S_ROW / 4), bs_o = S_OFF + (BM + wn * TN * 32 + r32) * S_ROW + b * (S_ROW / 4);
    const auto place_in = [&](int piece, int row_bytes) { return r32 * row_bytes + (row_bytes == 128 ? ((piece ^ (r32 >> 1)) & 7) * 16 : ((piece ^ (r32 >> 2)) & 3) * 16); };
    int ax[SL][XL], aw[SL];
#pragma unroll
    for (int k = 0; k < SL; ++k) {
        aw[k] = B_OFF + wn * TN * 32 * B_ROW + place_in(SL * b + k, B_ROW);
#pragma unroll
        for (int l = 0; l < XL; ++l) {
            const int at = 2 * (l * SL + k) + b;      // MXFP8: 16-byte piece of the step
            ax[k][l] = wm * TM * 32 * A_ROW + (X8 ? (at >> 3) * (BM * A_ROW) + place_in(at & 7, A_ROW) : place_in(SL * b + k, A_ROW));
        }
    }
    u32x4 x[2][TM][XL], w[2][TN];
    unsigned xs[2][TM], ws[2][TN];             // scales of this step and the next one
    const auto scale_at = [&](int at) __attribute__((always_inline)) -> unsigned {
        if constexpr (WHOLE && SL == 4) return *(const unsigned*)(lds + at);
        if constexpr (WHOLE) return *(const unsigned short*)(lds + at);
        const uint2 v = *(const uint2*)(lds + at);
        return v.x | (v.y << 8);
    };
    static_assert(WHOLE || SL == 2, "two scales");
    // Multiplications of slice T beside the reads of the next one of buffer `rb` (with those of a step's first slice its scales, at `so`) and a part of the loads of step `ls` into `lb`: the
    // three in turn, so that none of the units waits for another's block to end.
    const auto slice = [&](auto t_, int rbuf, int so, int ls, int lb, unsigned mask) __attribute__((always_inline)) {
        constexpr int T = decltype(t_)::value, R = (T + 1) % SL, SET = T & 1, OTHER = SET ^ 1;
        const unsigned char* const p = lds + rbuf * STAGE;
        constexpr int READS = TM * XL + TN, G = TN > 1 ? TN - 1 : 1;      // none beside the last multiplications: what the next slice waits for first is then there
        load_part(std::integral_constant<int, R>{}, ls, lb);
        DFK_WAIT_LGKM0();                      // (the compiler would wait behind the first read of this slice, for that one too)
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            if (n < G) {
#pragma unroll
                for (int i = n * READS / G; i < (n + 1) * READS / G; ++i) {
                    if (i < TM * XL) {
                        const int m = i / XL, l = i % XL;
                        x[OTHER][m][l] = *(const u32x4*)(p + ax[R][l] + m * (32 * A_ROW));
                        if (R == 0 && l == 0) xs[1][m] = scale_at(so + as_o + m * 32 * S_ROW);
                    } else {
                        const int k = i - TM * XL;
                        w[OTHER][k] = *(const u32x4*)(p + aw[R] + k * (32 * B_ROW));
                        if (R == 0) ws[1][k] = scale_at(so + bs_o + k * 32 * S_ROW);
                    }
                }
            }
            __builtin_amdgcn_s_setprio(1);     // of the two wavefronts of a SIMD, the one that multiplies goes first
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                if constexpr (KG > 1) {
                    if (n == 0) {
#pragma unroll
                        for (int k = 0; k < XL; ++k) x[SET][m][k] &= mask;
                    }
                }
                if constexpr (X8 && EXACT) {
                    u32x4 h[2], l[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            h[k][i] = mx_fp8_large(x[SET][m][k][i]);
                            l[k][i] = x[SET][m][k][i] ^ h[k][i];
                        }
                    acc[n][m] = mx_mfma32<X8, T>(w[SET][n], h[0], h[1], acc[n][m], ws[0][n], xs[0][m]);
                    acc[n][m] = mx_mfma32<X8, T>(w[SET][n], l[0], l[1], acc[n][m], ws[0][n], xs[0][m]);
                } else {
                    acc[n][m] = mx_mfma32<X8, T>(w[SET][n], x[SET][m][0], x[SET][m][XL - 1], acc[n][m], ws[0][n], xs[0][m]);
                }
            }
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // The last step's blocks past the end of A become zeros, so that what stands in B's place is not added (its elements are finite, and its scales those of the same rows' last blocks).  Each
    // wavefront sees to the pieces that its own loads brought.
    const auto cut = [&](int buf, bool now) __attribute__((always_inline)) {
        if constexpr (!WHOLE) {
#pragma unroll
            for (int j = 0; j < LA; ++j) {
                const int at = now && (int)(piece_a >> 4) >= XL * left ? buf * STAGE + (wave + NW * j) * 1024 : NONE;
                lds_write_b128_raw(lds_addr(lds) + at + lane * 16, f32x4{0.f, 0.f, 0.f, 0.f});
            }
        }
    };
    tile_wait_const<LOADS * (NS - 2) + (NS == 2 ? LOADS : LOADS / SL)>();
    cut(0, steps == 1);
    lds_barrier();
#pragma unroll
    for (int m = 0; m < TM; ++m) {
#pragma unroll
        for (int l = 0; l < XL; ++l) x[0][m][l] = *(const u32x4*)(lds + ax[0][l] + m * (32 * A_ROW));
        xs[0][m] = scale_at(as_o + m * 32 * S_ROW);
    }
#pragma unroll
    for (int n = 0; n < TN; ++n) {
        w[0][n] = *(const u32x4*)(lds + aw[0] + n * (32 * B_ROW));
        ws[0][n] = scale_at(bs_o + n * 32 * S_ROW);
    }
    // Step s: the last parts of step s - 1 + NS go into the buffer before this one, the first part of step s + NS into this one, behind the barrier.  (The last step reads what it does not use.)
    // Scales: of three pairs of steps, one that is read, the next one and one on its way, which has until its first step begins.
    int buf = 0, prev = NS - 1, pair = 0;
#pragma unroll 1
    for (int s = 0; s < loops; ++s) {
        const unsigned mask = s < own ? ~0u : 0u;
        const int next = buf + 1 == NS ? 0 : buf + 1, pair1 = pair + 1 == 3 ? 0 : pair + 1, pair2 = pair1 + 1 == 3 ? 0 : pair1 + 1;
        load_scales(s + 4, pair2);
        slice(i0, buf, 0, s + NS - 1, prev, mask);
        if constexpr (SL == 4) {
            slice(i1, buf, 0, s + NS - 1, prev, mask);
            slice(i2, buf, 0, s + NS - 1, prev, mask);
        }
        // The loads of step s + 1 have landed: newer ones are those of steps s + 2 to s + NS - 1 and the scales that were requested beside them.  (The scales of step s + 1 were requested three steps
        // ago or more.)
        tile_wait_const<NS == 2 ? LH : (LOADS + LH) * (NS - 2)>();
        cut(next, s + 2 == steps);
        lds_barrier();                         // (waits for this wavefront's LDS accesses first)
        slice(std::integral_constant<int, SL - 1>{}, next, s & 1 ? pair1 * S_PAIR : pair * S_PAIR + S_ROW / 2, s + NS, buf, mask);
#pragma unroll
        for (int m = 0; m < TM; ++m) xs[0][m] = xs[1][m];
#pragma unroll
        for (int n = 0; n < TN; ++n) ws[0][n] = ws[1][n];
        prev = buf;
        buf = next;
        if (s & 1) pair = pair1;
    }
    tile_wait_const<0>();                      // (the repeated loads)

    if constexpr (KG > 1) {                    // the groups' sums, in order
        static_assert(KG == 2, "one sum");
        lds_barrier();
        f32x4* const box = (f32x4*)all_lds + wave * (TN * TM * 4 * 64);
        if (kg) {
#pragma unroll
            for (int j = 0; j < TN * TM * 4; ++j) {
                const f32x16& c = acc[j / 4 / TM][j / 4 % TM];
                box[j * 64 + lane] = f32x4{c[4 * (j % 4)], c[4 * (j % 4) + 1], c[4 * (j % 4) + 2], c[4 * (j % 4) + 3]};
            }
        }
        lds_barrier();
        if (kg) return;
#pragma unroll
        for (int j = 0; j < TN * TM * 4; ++j) {
            const f32x4 v = box[j * 64 + lane];
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[j / 4 / TM][j / 4 % TM][4 * (j % 4) + k] += v[k];
        }
    }
    if constexpr (GATED) {
        const auto finish = [&](const f32x16& gate, const f32x16& up, int m, int col) __attribute__((always_inline)) {
            const int r = (wm * TM + m) * 32 + r32;
            const bool live = r < rows && col < t.N;
            float v[16];
            if (a.out_mx >= 0) {
                silu_mul_all<true>(gate, up, v);
                if (a.out_mx == DFK_MXFP4) mx_store_block<DFK_MXFP4>(a, v, row0 + r, col, b, live);
                else mx_store_block<DFK_MXFP8>(a, v, row0 + r, col, b, live);
            } else {
                silu_mul_all<false>(gate, up, v);
                if (live) {
                    const size_t at = (row0 + r) * (size_t)t.N + col + 4 * b;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (a.dtype == DFK_BF16) BF16::store4(t.out, at + 8 * i, v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                        else FP16::store4(t.out, at + 8 * i, v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                    }
                }
            }
        };
        if constexpr (TN == 1) {               // the up projection's sums come from the next wavefront
            lds_barrier();
            f32x4* const box = (f32x4*)lds + (wm * (WN / 2) + wn / 2) * (TM * 4 * 64);
            if (wn & 1) {
#pragma unroll
                for (int m = 0; m < TM; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) box[(m * 4 + i) * 64 + lane] = f32x4{acc[0][m][4 * i], acc[0][m][4 * i + 1], acc[0][m][4 * i + 2], acc[0][m][4 * i + 3]};
            }
            lds_barrier();
            if (wn & 1) return;
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                f32x16 up;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 u = box[(m * 4 + i) * 64 + lane];
#pragma unroll
                    for (int k = 0; k < 4; ++k) up[4 * i + k] = u[k];
                }
                finish(acc[0][m], up, m, n0 + wn * 16);
            }
        } else {
#pragma unroll
            for (int n = 0; n < TN; n += 2)
#pragma unroll
                for (int m = 0; m < TM; ++m) finish(acc[n][m], acc[n + 1 < TN ? n + 1 : n][m], m, n0 + (wn * TN + n) * 16);
        }
    } else {
        // ---- epilogue: through LDS, as in dfk_tile.h
        constexpr int PM = mx_epilogue_tiles(TM, TN, NW), PITCH = TN * 32 + 4, CV = TN * 8;
        lds_barrier();
        float* const mine = (float*)lds + wave * (PM * 32 * PITCH);
#pragma unroll
        for (int m0 = 0; m0 < TM; m0 += PM) {
#pragma unroll
            for (int m = m0; m < m0 + PM; ++m)
#pragma unroll
                for (int n = 0; n < TN; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *(f32x4*)(mine + ((m - m0) * 32 + r32) * PITCH + n * 32 + 8 * i + 4 * b) = f32x4{acc[n][m][4 * i], acc[n][m][4 * i + 1], acc[n][m][4 * i + 2], acc[n][m][4 * i + 3]};
            if (t.splits == 1 && t.vec4 && t.act == DFK_ACT_NONE) {
                // four vectors at a time, so that their way through LDS (and the residual's from memory) is waited for once
                const auto plain = [&](auto e_, auto out_) __attribute__((always_inline)) {
                    using E = decltype(e_);
                    using OUT = decltype(out_);
#pragma unroll 1
                    for (int i0 = lane; i0 < PM * 32 * CV; i0 += 256) {
                        float v[4][4];
                        size_t at[4];
                        bool live[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int i = i0 + 64 * u, lr = i / CV, c = i - lr * CV, r = (wm * TM + m0) * 32 + lr, col = n0 + wn * TN * 32 + 4 * c;
                            const f32x4 s = *(const f32x4*)(mine + lr * PITCH + 4 * c);
                            live[u] = r < rows && col < t.N;
                            at[u] = (row0 + r) * (size_t)t.N + col;
                            float bias[4] = {0.f, 0.f, 0.f, 0.f};
                            if (t.bias && live[u]) E::load4(t.bias, col, bias);
#pragma unroll
                            for (int k = 0; k < 4; ++k) v[u][k] = s[k] + bias[k];
                        }
                        if (t.resid) {
                            float x[4][4];
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                if (live[u]) OUT::load4(t.resid, at[u], x[u]);
#pragma unroll
                            for (int u = 0; u < 4; ++u)
#pragma unroll
                                for (int k = 0; k < 4; ++k) v[u][k] += x[u][k];
                        }
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (live[u]) OUT::store4(t.out, at[u], v[u][0], v[u][1], v[u][2], v[u][3]);
                    }
                };
                if (a.dtype == DFK_BF16) {
                    if (t.out_fp32) plain(BF16{}, FP32{});
                    else plain(BF16{}, BF16{});
                } else {
                    if (t.out_fp32) plain(FP16{}, FP32{});
                    else plain(FP16{}, FP16{});
                }
                continue;
            }
#pragma unroll 1
            for (int i = lane; i < PM * 32 * CV; i += 64) {
                const int lr = i / CV, c = i - lr * CV, r = (wm * TM + m0) * 32 + lr, col = n0 + wn * TN * 32 + 4 * c;
                const f32x4 s = *(const f32x4*)(mine + lr * PITCH + 4 * c);
                const float v[4] = {s[0], s[1], s[2], s[3]};
                if (r >= rows) break;          // (rows rise with i)
                if (t.splits > 1) {
                    if (col < t.N) FP32::store4(t.partial, ((size_t)k_split * t.M + row0 + r) * t.pitch + col, v[0], v[1], v[2], v[3]);
                } else if (a.dtype == DFK_BF16) {
                    if (t.out_fp32) linear_store4<BF16, FP32>(t, row0 + r, col, v);
                    else linear_store4<BF16, BF16>(t, row0 + r, col, v);
                } else {
                    if (t.out_fp32) linear_store4<FP16, FP32>(t, row0 + r, col, v);
                    else linear_store4<FP16, FP16>(t, row0 + r, col, v);
                }
            }
        }
    }
}

template <bool X8, int KS, int BM, int BN, int WM, int WN, int KG, int NS, bool GATED, bool WHOLE, bool EXACT>
hipError_t launch(const MxArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr size_t stages = (size_t)KG * mx_tile_lds(X8, KS, BM, BN, NS, WHOLE), sums = KG > 1 ? (size_t)WM * WN * TN * TM * 4096 : 0;
    constexpr size_t end = GATED ? (TN == 1 ? (size_t)WM * (WN / 2) * TM * 4096 : 0) : (size_t)WM * WN * mx_epilogue_tiles(TM, TN, WM * WN) * 32 * (TN * 32 + 4) * 4;
    constexpr size_t most = end > sums ? end : sums, lds = most > stages ? most : stages;
    static_assert(lds <= (size_t)kLdsLimit, "buffers fit LDS");
    if ((WHOLE && a.t.K % KS) || (GATED && a.t.splits != 1) || linear_partial_bytes(a.t.M, a.t.N, a.t.splits) > a.t.partial_bytes) return hipErrorInvalidValue;
    const auto kernel = k_mx_tile<X8, KS, BM, BN, WM, WN, KG, NS, GATED, WHOLE, EXACT>;
    if (hipError_t e = allow_lds(allowed, (const void*)kernel, lds); e != hipSuccess) return e;
    const int cols = GATED ? BN / 2 : BN;
    const long long tiles = (long long)((a.t.M + BM - 1) / BM) * ((a.t.N + cols - 1) / cols) * a.t.splits;
    if ((tiles + 7) / 8 * 8 * (WM * WN * KG * 64) >= 1ll << 32) return hipErrorInvalidValue;
    return launch_kernel(kernel, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(WM * WN * KG * 64), lds, st, a);
}

// kMxTiles, mx_tile_offered
template <int TILE, bool GATED, bool X8, bool EXACT>
hipError_t of_256(const MxArgs& a, hipStream_t st) {
    if constexpr (!mx_tile_offered(TILE, X8, GATED, EXACT, true)) return hipErrorInvalidValue;
    else if constexpr (TILE == kMxTileSmall) return launch<X8, 256, 64, 64, 2, 2, 1, X8 ? 3 : 4, GATED, true, EXACT>(a, st);
    else if constexpr (TILE == 1) return launch<X8, 256, 64, 128, 2, 2, 1, 2, GATED, true, EXACT>(a, st);
    else if constexpr (TILE == kMxTile128) return launch<X8, 256, 128, 128, GATED ? 4 : 2, GATED ? 2 : 4, 1, 3, GATED, true, EXACT>(a, st);
    else if constexpr (TILE == 3) return launch<X8, 256, 128, 256, 2, 4, 1, 2, GATED, true, EXACT>(a, st);
    else if constexpr (TILE == kMxTile256) return launch<X8, X8 ? 128 : 256, 256, 256, 4, 2, 1, X8 ? 3 : 2, GATED, true, EXACT>(a, st);
    else if constexpr (TILE == 5) return launch<X8, 256, 128, 128, 2, 2, 1, 2, GATED, true, EXACT>(a, st);
    else if constexpr (TILE == 6) return launch<X8, 256, 32, 128, 1, 4, 1, 3, GATED, true, EXACT>(a, st);
    else return launch<X8, 256, 64, 64, 2, 2, 2, X8 ? 3 : 4, GATED, true, EXACT>(a, st);
}
template <bool GATED, bool X8, bool EXACT>
hipError_t of_256(const MxArgs& a, int tile, hipStream_t st) {
    static_assert(kMxTileCount == 8, "the cases");
    switch (tile) {
        case 0: return of_256<0, GATED, X8, EXACT>(a, st);
        case 1: return of_256<1, GATED, X8, EXACT>(a, st);
        case 2: return of_256<2, GATED, X8, EXACT>(a, st);
        case 3: return of_256<3, GATED, X8, EXACT>(a, st);
        case 4: return of_256<4, GATED, X8, EXACT>(a, st);
        case 5: return of_256<5, GATED, X8, EXACT>(a, st);
        case 6: return of_256<6, GATED, X8, EXACT>(a, st);
        case 7: return of_256<7, GATED, X8, EXACT>(a, st);
    }
    return hipErrorInvalidValue;
}
template <bool GATED, bool X8, bool EXACT, bool WHOLE>
hipError_t of_128(const MxArgs& a, int tile, hipStream_t st) {
    if (tile == kMxTileSmall) return launch<X8, 128, 64, 64, 2, 2, 1, 4, GATED, WHOLE, EXACT>(a, st);
    return tile == kMxTile128 ? launch<X8, 128, 128, 128, 2, 2, 1, 3, GATED, WHOLE, EXACT>(a, st) : hipErrorInvalidValue;
}
template <bool GATED, bool X8, bool EXACT>
hipError_t by_width(const MxArgs& a, int tile, hipStream_t st) {
    if (a.t.K % 256 == 0) return of_256<GATED, X8, EXACT>(a, tile, st);
    return a.t.K % 128 == 0 ? of_128<GATED, X8, EXACT, true>(a, tile, st) : of_128<GATED, X8, EXACT, false>(a, tile, st);
}
template <bool GATED>
hipError_t by_format(const MxArgs& a, int x_mx, int tile, hipStream_t st) {
    if (x_mx == DFK_MXFP4) return by_width<GATED, false, false>(a, tile, st);
    return mx_exact_sums(a.t.M, !GATED && a.t.out_fp32) ? by_width<GATED, true, true>(a, tile, st) : by_width<GATED, true, false>(a, tile, st);
}

}  // namespace

hipError_t launch_mx_linear_tile(const MxArgs& a, int x_mx, int tile, hipStream_t st) {
    const hipError_t e = by_format<false>(a, x_mx, tile, st);
    return e != hipSuccess || a.t.splits == 1 ? e : launch_linear_sum(a.t, (dfk_dtype_t)a.dtype, st);
}

hipError_t launch_mx_gateup_tile(const MxArgs& a, int x_mx, int tile, hipStream_t st) { return by_format<true>(a, x_mx, tile, st); }

}  // namespace dfk
