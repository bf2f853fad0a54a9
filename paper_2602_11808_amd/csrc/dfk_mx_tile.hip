// Products with MXFP4 weights on the scaled matrix instructions, many rows: the tile kernel of the linear layers and of the MLP's gated half.
//
// out[m, n] = sum_k A[m, k] B[n, k].  A workgroup owns BM rows of A and BN rows of B (gated: BN / 2 columns, 32 rows of the gate's weights and the same 32 of the up projection's
// in turn, so that a wavefront has both sums of a column); wavefront (wm, wn) TN x TM products of 32 x 32.
//
// Data movement: as in dfk_tile.h, asynchronous global->LDS loads NS steps deep, a step being 256 k: one cache line of a row in MXFP4, two in MXFP8, and eight scales.
// In LDS a row's line is 128 bytes, its eight 16-byte pieces XOR-swizzled by row / 2.  Slice t (0..3) of a step multiplies blocks t and 4 + t of it, so that a lane's four scales
// of a step are the bytes of one word, from which the instruction takes byte t.  While a slice multiplies, the operands of the next one are read.  One barrier per step, ahead of its
// last slice: by then every wavefront has that slice's operands in registers and has waited, by count, for its own loads of the following step.
//
// Scales: words of four where a row has a whole number of them (K a multiple of 128), else each byte by a load of its own, which arrives as a word.  Those of two steps are loaded together, 16
// bytes of a row at a time: each is a line of its own for the caches.
//
// Pieces past the end of a row are copies of the last one, and zeroed in A; rows past the end are copies of the last one and are not stored.
#include "dfk_mx_device.h"
#include "dfk_mx_plan.h"
#include "dfk_tile.h"

namespace dfk {
namespace {

constexpr int kMxStepK = 256;
constexpr int kMxNoneBytes = 1024;          // of LDS, for what is written to no purpose
enum { kMxWhole = 0, kMxWords = 1, kMxBytes = 2 };      // rows of whole steps, of whole words of scales, of any number of blocks

constexpr int mx_epilogue_tiles(int TM, int TN, int NW) {
    int pm = TM;
    while (pm > 1 && (size_t)NW * pm * 32 * (TN * 32 + 4) * 4 > (size_t)kLdsLimit) pm /= 2;
    return pm;
}
constexpr int mx_stage_bytes(bool x8, int BM, int BN) { return BM * (x8 ? 256 : 128) + BN * 128; }
constexpr int mx_scale_bytes(int BM, int BN, bool words) { return (BM + BN) * (words ? 16 : 64); }      // of two steps

// Columns col .. col + 31 of row r of the gated half, of which lane (., b) has 8 i + 4 b .. + 3 in a[4 i ..]: as MX, lane b takes columns 16 b .. 16 b + 15 after an exchange with the other.
__device__ __forceinline__ void mx_store_block(const MxArgs& a, const float (&v)[16], size_t r, int col, int b, bool live) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = mx_top(top, v[i]);
    top = mx_top(top, __shfl_xor(top, 32));
    int up;
    const unsigned s = mx_scale_of(top, a.out_mx, up);
    const bool none = s == 255u;
    const size_t blk = r * (size_t)(a.t.N / kMxBlock) + col / kMxBlock;
    unsigned w[4];
    if (a.out_mx == DFK_MXFP4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f[4] = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
            w[i] = mx_fp4x4(f, up, none);
        }
        const unsigned lo = w[0] | (w[1] << 16), hi = w[2] | (w[3] << 16);     // groups 0, 1 and 2, 3
        const unsigned got = (unsigned)__shfl_xor((int)(b ? lo : hi), 32), e = b ? got : lo, o = b ? hi : got;   // of the even and of the odd four columns
        uint2 out;
        out.x = (e & 0xFFFFu) | (o << 16);
        out.y = (e >> 16) | (o & 0xFFFF0000u);
        if (live) *(uint2*)(a.q + blk * 16 + 8 * b) = out;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f[4] = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
            w[i] = mx_fp8x4(f, up, none);
        }
        const unsigned g0 = (unsigned)__shfl_xor((int)(b ? w[0] : w[2]), 32), g1 = (unsigned)__shfl_xor((int)(b ? w[1] : w[3]), 32);
        const u32x4 out = b ? u32x4{g0, w[2], g1, w[3]} : u32x4{w[0], g0, w[1], g1};
        if (live) *(u32x4*)(a.q + blk * 32 + 16 * b) = out;
    }
    if (live && b == 0) a.qs[blk] = (unsigned char)s;
}

template <bool X8, int BM, int BN, int WM, int WN, int NS, bool GATED, int KIND, bool EXACT>
__global__ __launch_bounds__(WM * WN * 64) void k_mx_tile(MxArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr bool WORDS = KIND < kMxBytes, TAIL = KIND != kMxWhole;
    constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, XL = X8 ? 2 : 1;
    constexpr int B_OFF = BM * 128 * XL, STAGE = mx_stage_bytes(X8, BM, BN), S_OFF = NS * STAGE, S_PAIR = mx_scale_bytes(BM, BN, WORDS), S_ROW = WORDS ? 16 : 64, NONE = S_OFF + 2 * S_PAIR;
    constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, S_PER = WORDS ? 16 : 4, S_ALL = (BM + BN) / S_PER, LS = (S_ALL + NW - 1) / NW;
    constexpr int LOADS = LA * XL + LB;        // of a wavefront and step; LS more in every other step
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM % (32 * WM) == 0 && BN % (32 * WN) == 0 && NW % 2 == 0, "whole loads and tiles");
    static_assert(!GATED || TN % 2 == 0, "gate and up of a column in one wavefront");
    static_assert(NS == 2 || NS == 3, "the waits below");
    constexpr int COLS = GATED ? BN / 2 : BN;
    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, b = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    const TileArgs& t = a.t;
    const int n_tiles = (t.N + COLS - 1) / COLS;
    int mt, nt;
    if (!tile_of((t.M + BM - 1) / BM, n_tiles * t.splits, mt, nt)) return;
    const int k_split = nt / n_tiles;
    nt -= k_split * n_tiles;
    const size_t row0 = (size_t)mt * BM;
    const int rows = min(BM, t.M - (int)row0), n0 = nt * COLS;
    int s_lo = 0, steps = (t.K + kMxStepK - 1) / kMxStepK;
    if (t.splits > 1) {
        int s1;
        share_of((unsigned)steps, (unsigned)t.splits, (unsigned)k_split, s_lo, s1);
        steps = s1 - s_lo;
    }
    const int blocks = min(t.K / kMxBlock - s_lo * 8, steps * 8);     // of 32 k, this workgroup's

    // ---- loads: instruction j covers rows 8 j .. 8 j + 7 of a line, lane l row l / 8 and the piece whose place is l % 8; wavefront w has instructions w, w + NW, ...
    const unsigned arb = (unsigned)t.K / (X8 ? 1 : 2), brb = (unsigned)t.K / 2, srb = (unsigned)t.K / kMxBlock;
    const int prow = lane >> 3;
    const unsigned kb = (unsigned)((((lane & 7) ^ (prow >> 1)) & 7) * 16) ^ ((wave & 1) ? 64u : 0u);
    const char* const base_a = (const char*)t.A + row0 * arb + (size_t)s_lo * (128 * XL);
    const char* const base_b = (const char*)t.B + (size_t)n0 * brb + (size_t)s_lo * 128;
    const char* const base_u = GATED ? (const char*)t.B2 + (size_t)n0 * brb + (size_t)s_lo * 128 : nullptr;
    const int n_last = t.N - n0 - 1;
    // row of B of a place in the tile, and whether it is one of the up projection's
    const auto b_row = [&](int i) __attribute__((always_inline)) { return min(GATED ? (i >> 6) * 32 + (i & 31) : i, n_last); };
    unsigned off_a[LA], off_b[LB], off_s[LS];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        off_a[i] = (unsigned)min(8 * (wave + NW * i) + prow, rows - 1) * arb + kb;
        asm("" : "+v"(off_a[i]));             // (one register: out of the multiplication it would keep two)
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        off_b[i] = (unsigned)b_row(8 * (wave + NW * i) + prow) * brb + kb;
        asm("" : "+v"(off_b[i]));
    }
    // scales: instruction e covers S_PER rows, A's first, four words (sixteen bytes) of each
    const int s_in = lane % (64 / S_PER), s_row = lane / (64 / S_PER);
    const bool s_odd = s_in >= 32 / S_PER;     // this lane's are of the second step of two
    const unsigned s_byte = WORDS ? 4 * (s_in & 1) : s_in & 7;
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
        s_base[i] += s_lo * 8;
        asm("" : "+v"(off_s[i]));
    }
    const int whole = blocks / 8, left = blocks - (steps - 1) * 8;     // whole steps, and blocks of the last one
    const int rot = t.M <= 4 * BM && whole > 0 ? (int)((unsigned)nt % (unsigned)whole) : 0;     // (dfk_tile.h)
    // in the last, partial step a piece (a scale) past the end is replaced by the last one there is
    const auto past = [](unsigned at, unsigned size, unsigned end) { return at + size > end ? at + size - end : 0u; };
    const unsigned tail_b = past(kb, 16, left * 16u), tail_s = past(s_byte, WORDS ? 4 : 1, left);
    unsigned tail_a[XL];
#pragma unroll
    for (int l = 0; l < XL; ++l) tail_a[l] = past(kb + 128u * l, 16, left * (16u * XL));
    const auto place = [&](int s) __attribute__((always_inline)) {           // of step s in the row (past the last one: the last one)
        const int c = min(s, steps - 1), r = c + rot;
        return c < whole ? (r >= whole ? r - whole : r) : c;
    };
    // The step loop is one block without branches: the compiler moves multiplications across a branch to the block that uses their results.  So every step requests as many loads:
    // what it does not need is a line that is there already, and scales go to a place that nobody reads.
    // Loads of quarter Q of step s into buffer `buf`.
    const auto load_quarter = [&](auto q_, int s, int buf) __attribute__((always_inline)) {
        constexpr int Q = decltype(q_)::value;
        const size_t st = place(s);
        const unsigned live = s < steps ? ~0u : 0u, end = s == steps - 1 ? ~0u : 0u;
        const char* const pa = base_a + st * (128 * XL);
        const char* const pb = base_b + st * 128;
        const char* const pu = base_u + st * 128;
        unsigned char* const dst = lds + buf * STAGE + wave * 1024;
#pragma unroll
        for (int i = Q * LOADS / 4; i < (Q + 1) * LOADS / 4; ++i) {
            if (i < LA * XL) {
                const int j = i / XL, l = i % XL;
                unsigned o = (off_a[j] + 128u * l - (TAIL ? tail_a[l] & end : 0u)) & live;      // (never below its row's start: the line is part of what a tail is taken from)
                asm("" : "+v"(o));            // 32 bits from a scalar base, not a 64-bit sum of its own
                __builtin_amdgcn_global_load_lds(pa + o, DFK_LDS_PTR(dst + l * (BM * 128) + NW * j * 1024), 16, 0, 0);
            } else {
                const int j = i - LA * XL;
                unsigned o = (off_b[j] - (TAIL ? tail_b & end : 0u)) & live;
                asm("" : "+v"(o));
                const char* const p = GATED && ((8 * (wave + NW * j)) & 32) ? pu : pb;
                __builtin_amdgcn_global_load_lds(p + o, DFK_LDS_PTR(dst + B_OFF + NW * j * 1024), 16, 0, 0);
            }
        }
    };
    // scales of steps s and s + 1, for an even s
    const auto load_scales = [&](int s) __attribute__((always_inline)) {
        const int s0 = s & ~1, e0 = place(s0) * 8, e1 = place(s0 + 1) * 8;
        unsigned at = s_odd ? e1 : e0;
        if (TAIL) at -= s0 + (s_odd ? 1 : 0) >= steps - 1 ? tail_s : 0u;
        const unsigned live = s & 1 ? 0u : ~0u;
#pragma unroll
        for (int i = 0; i < LS; ++i) {
            unsigned o = (off_s[i] + at) & live;
            asm("" : "+v"(o));
            unsigned char* const dst = lds + (s & 1 ? NONE : S_OFF + ((s >> 1) & 1) * S_PAIR + (wave + NW * i) % S_ALL * 256);
            if constexpr (WORDS) __builtin_amdgcn_global_load_lds(s_base[i] + o, DFK_LDS_PTR(dst), 4, 0, 0);
            else __builtin_amdgcn_global_load_lds(s_base[i] + o, DFK_LDS_PTR(dst), 1, 0, 0);
        }
    };
    constexpr std::integral_constant<int, 0> i0{};
    constexpr std::integral_constant<int, 1> i1{};
    constexpr std::integral_constant<int, 2> i2{};
    constexpr std::integral_constant<int, 3> i3{};
    load_scales(0);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        load_quarter(i0, s, s);
        if (s + 1 < NS) {
            load_quarter(i1, s, s);
            load_quarter(i2, s, s);
            load_quarter(i3, s, s);
        }
    }

    f32x16 acc[TN][TM];
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.f;

    // operands: rows r32 of 32-row tiles; MXFP4 piece 4 b + t, MXFP8 piece 2 t + b of both lines
    const int sw = (r32 >> 1) & 7;
    const int ao = wm * TM * 4096 + r32 * 128, bo = B_OFF + wn * TN * 4096 + r32 * 128;
    const int as_o = S_OFF + (wm * TM * 32 + r32) * S_ROW + b * (S_ROW / 4), bs_o = S_OFF + (BM + wn * TN * 32 + r32) * S_ROW + b * (S_ROW / 4);
    u32x4 x[2][TM][XL], w[2][TN];
    unsigned xs[2][TM], ws[2][TN];             // scales of this step and the next one
    const auto scale_at = [&](int at) __attribute__((always_inline)) -> unsigned {
        if constexpr (WORDS) return *(const unsigned*)(lds + at);
        const u32x4 v = *(const u32x4*)(lds + at);
        return v.x | (v.y << 8) | (v.z << 16) | (v.w << 24);
    };
    int ax[4], aw[4];                          // a slice's pieces
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        ax[k] = ao + ((X8 ? 2 * k + b : 4 * b + k) ^ sw) * 16;
        aw[k] = bo + ((4 * b + k) ^ sw) * 16;
    }
    // Multiplications of slice T beside the reads of slice R of buffer `rb` (with those of a step's first slice its scales, at `so`) and the loads of quarter R of step `ls` into `lb`: the
    // three in turn, so that none of the units waits for another's block to end.
    const auto slice = [&](auto t_, int rbuf, int so, int ls, int lb) __attribute__((always_inline)) {
        constexpr int T = decltype(t_)::value, SET = T & 1, R = (T + 1) & 3;
        const unsigned char* const px = lds + rbuf * STAGE + ax[R];
        const unsigned char* const pw = lds + rbuf * STAGE + aw[R];
        load_quarter(std::integral_constant<int, R>{}, ls, lb);
#pragma unroll
        for (int n = 0; n < TN; ++n) {
#pragma unroll
            for (int m = n * TM / TN; m < (n + 1) * TM / TN; ++m) {
#pragma unroll
                for (int l = 0; l < XL; ++l) x[SET ^ 1][m][l] = *(const u32x4*)(px + l * (BM * 128) + m * 4096);
                if (R == 0) xs[1][m] = scale_at(so + as_o + m * 32 * S_ROW);
            }
            w[SET ^ 1][n] = *(const u32x4*)(pw + n * 4096);
            if (R == 0) ws[1][n] = scale_at(so + bs_o + n * 32 * S_ROW);
            __builtin_amdgcn_s_setprio(1);     // of the two wavefronts of a SIMD, the one that multiplies goes first
#pragma unroll
            for (int m = 0; m < TM; ++m) {
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
        if constexpr (TAIL) {
#pragma unroll
            for (int j = 0; j < LA; ++j)
#pragma unroll
                for (int l = 0; l < XL; ++l) {
                    const int at = now && (int)(kb >> 4) + 8 * l >= XL * left ? buf * STAGE + l * (BM * 128) + (wave + NW * j) * 1024 : NONE;
                    lds_write_b128_raw(lds_addr(lds) + at + lane * 16, f32x4{0.f, 0.f, 0.f, 0.f});
                }
        }
    };
    tile_wait_const<LOADS * (NS - 2) + LOADS / 4>();
    cut(0, steps == 1);
    lds_barrier();
#pragma unroll
    for (int m = 0; m < TM; ++m) {
#pragma unroll
        for (int l = 0; l < XL; ++l) x[0][m][l] = *(const u32x4*)(lds + ax[0] + l * (BM * 128) + m * 4096);
        xs[0][m] = scale_at(as_o + m * 32 * S_ROW);
    }
#pragma unroll
    for (int n = 0; n < TN; ++n) {
        w[0][n] = *(const u32x4*)(lds + aw[0] + n * 4096);
        ws[0][n] = scale_at(bs_o + n * 32 * S_ROW);
    }
    // Step s: quarters 1 to 3 of step s - 1 + NS go into the buffer before this one, quarter 0 of step s + NS into this one, behind the barrier.  (The last step reads what it does not use.)
    int buf = 0, prev = NS - 1;
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
        const int next = buf + 1 == NS ? 0 : buf + 1;
        load_scales(s + 2);
        slice(i0, buf, 0, s + NS - 1, prev);
        slice(i1, buf, 0, s + NS - 1, prev);
        slice(i2, buf, 0, s + NS - 1, prev);
        // the loads of step s + 1 have landed, and its scales: newer ones are, with NS = 3, those of step s + 2, and the scales that this step requested, which count as its last ones
        tile_wait_const<NS == 2 ? 0 : LOADS>();
        cut(next, s + 2 == steps);
        lds_barrier();                         // (waits for this wavefront's LDS accesses first)
        slice(i3, next, ((s + 1) >> 1 & 1) * S_PAIR + ((s + 1) & 1) * (S_ROW / 2), s + NS, buf);
#pragma unroll
        for (int m = 0; m < TM; ++m) xs[0][m] = xs[1][m];
#pragma unroll
        for (int n = 0; n < TN; ++n) ws[0][n] = ws[1][n];
        prev = buf;
        buf = next;
    }
    tile_wait_const<0>();                      // (the repeated loads)

    if constexpr (GATED) {
#pragma unroll
        for (int n = 0; n < TN; n += 2) {
            const int col = n0 + (wn * TN + n) * 16;
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const int r = (wm * TM + m) * 32 + r32;
                const bool live = r < rows && col < t.N;
                float v[16];
                if (a.out_mx >= 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = silu_mul(acc[n][m][i], acc[n + 1][m][i]);
                    mx_store_block(a, v, row0 + r, col, b, live);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = silu_mul_fast(acc[n][m][i], acc[n + 1][m][i]);
                    if (live) {
                        const size_t at = (row0 + r) * (size_t)t.N + col + 4 * b;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (a.dtype == DFK_BF16) BF16::store4(t.out, at + 8 * i, v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                            else FP16::store4(t.out, at + 8 * i, v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                        }
                    }
                }
            }
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

template <bool X8, int BM, int BN, int WM, int WN, int NS, bool GATED, int KIND, bool EXACT>
hipError_t launch(const MxArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr size_t stages = (size_t)NS * mx_stage_bytes(X8, BM, BN) + 2 * mx_scale_bytes(BM, BN, KIND < kMxBytes) + kMxNoneBytes, end = GATED ? 0 : (size_t)WM * WN * mx_epilogue_tiles(TM, TN, WM * WN) * 32 * (TN * 32 + 4) * 4;
    constexpr size_t lds = end > stages ? end : stages;
    static_assert(lds <= (size_t)kLdsLimit, "buffers fit LDS");
    if (linear_partial_bytes(a.t.M, a.t.N, a.t.splits) > a.t.partial_bytes) return hipErrorInvalidValue;
    const auto kernel = k_mx_tile<X8, BM, BN, WM, WN, NS, GATED, KIND, EXACT>;
    if (hipError_t e = allow_lds(allowed, (const void*)kernel, lds); e != hipSuccess) return e;
    const int cols = GATED ? BN / 2 : BN;
    const long long tiles = (long long)((a.t.M + BM - 1) / BM) * ((a.t.N + cols - 1) / cols) * a.t.splits;
    return launch_kernel(kernel, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(WM * WN * 64), lds, st, a);
}

template <bool X8, int KIND, bool EXACT>
hipError_t linear_of(const MxArgs& a, int tile, hipStream_t st) {
    switch (tile) {
        case 0: return launch<X8, 64, 64, 2, 2, 3, false, KIND, EXACT>(a, st);
        case 1: if constexpr (KIND == kMxWhole) return launch<X8, 64, 128, 2, 2, X8 ? 2 : 3, false, KIND, EXACT>(a, st); break;
        case 2: if constexpr (KIND == kMxWhole) return launch<X8, 64, 256, 2, 4, 3, false, KIND, EXACT>(a, st); break;
        case 3: return launch<X8, 128, 128, 2, 4, KIND == kMxBytes && X8 ? 2 : 3, false, KIND, EXACT>(a, st);
        case 4: if constexpr (KIND == kMxWhole) return launch<X8, 128, 256, 2, 4, X8 ? 2 : 3, false, KIND, EXACT>(a, st); break;
        case 5: if constexpr (KIND == kMxWhole && !X8) return launch<X8, 256, 128, 4, 2, 3, false, KIND, EXACT>(a, st); break;
        case 6: if constexpr (KIND == kMxWhole && !X8) return launch<X8, 256, 256, 4, 2, 2, false, KIND, EXACT>(a, st); break;
    }
    return hipErrorInvalidValue;
}
template <bool X8, int KIND, bool EXACT>
hipError_t gateup_of(const MxArgs& a, int tile, hipStream_t st) {
    switch (tile) {
        case 1: return launch<X8, 64, 128, 2, 2, X8 ? 2 : 3, true, KIND, EXACT>(a, st);
        case 2: if constexpr (KIND == kMxWhole) return launch<X8, 64, 256, 2, 4, 3, true, KIND, EXACT>(a, st); break;
        case 3: return launch<X8, 128, 128, 4, 2, KIND == kMxBytes && X8 ? 2 : 3, true, KIND, EXACT>(a, st);
        case 4: if constexpr (KIND == kMxWhole) return launch<X8, 128, 256, 2, 4, X8 ? 2 : 3, true, KIND, EXACT>(a, st); break;
        case 6: if constexpr (KIND == kMxWhole && !X8) return launch<X8, 256, 256, 4, 2, 2, true, KIND, EXACT>(a, st); break;
    }
    return hipErrorInvalidValue;
}
template <bool GATED, bool X8, bool EXACT>
hipError_t by_kind(const MxArgs& a, int tile, hipStream_t st) {
    const auto of = [&](auto kind_) {
        constexpr int KIND = decltype(kind_)::value;
        if constexpr (GATED) return gateup_of<X8, KIND, EXACT>(a, tile, st);
        else return linear_of<X8, KIND, EXACT>(a, tile, st);
    };
    if (a.t.K % kMxStepK == 0) return of(std::integral_constant<int, kMxWhole>{});
    if (a.t.K % 128 == 0) return of(std::integral_constant<int, kMxWords>{});
    return of(std::integral_constant<int, kMxBytes>{});
}
template <bool GATED>
hipError_t by_format(const MxArgs& a, int x_mx, int tile, hipStream_t st) {
    if (x_mx == DFK_MXFP4) return by_kind<GATED, false, false>(a, tile, st);
    return mx_exact_sums(a.t.M, !GATED && a.t.out_fp32) ? by_kind<GATED, true, true>(a, tile, st) : by_kind<GATED, true, false>(a, tile, st);
}

}  // namespace

extern "C" { int g_mx_tile = -1, g_mx_splits = 1; }
hipError_t launch_mx_linear_tile(const MxArgs& a0, int x_mx, int tile, hipStream_t st) {
    MxArgs a = a0;
    if (g_mx_tile >= 0) { tile = g_mx_tile; a.t.splits = g_mx_splits; }
    else tile = 3;
    if (a.t.K % 256) tile = 3;
    const hipError_t e = by_format<false>(a, x_mx, tile, st);
    if (e != hipSuccess || a.t.splits == 1) return e;
    return launch_linear_sum(a.t, (dfk_dtype_t)a.dtype, st);
}

hipError_t launch_mx_gateup_tile(const MxArgs& a, int x_mx, int tile, hipStream_t st) {
    tile = g_mx_tile >= 0 ? g_mx_tile : 3;
    if (a.t.K % 256) tile = 3;
    return by_format<true>(a, x_mx, tile, st);
}

}  // namespace dfk
