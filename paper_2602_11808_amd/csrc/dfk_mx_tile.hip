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
// Scales: words of four where a row has a whole number of them (K a multiple of 128), else each byte by a load of its own, which arrives as a word.
//
// Pieces past the end of a row are copies of the last one and zeroed in both factors; rows past the end are copies of the last one and are not stored.
#include "dfk_mx_device.h"
#include "dfk_mx_plan.h"
#include "dfk_tile.h"

namespace dfk {
namespace {

constexpr int kMxStepK = 256;

constexpr int mx_epilogue_tiles(int TM, int TN, int NW) {
    int pm = TM;
    while (pm > 1 && (size_t)NW * pm * 32 * (TN * 32 + 4) * 4 > (size_t)kLdsLimit) pm /= 2;
    return pm;
}
constexpr int mx_stage_bytes(bool x8, int BM, int BN, bool words) { return BM * (x8 ? 256 : 128) + BN * 128 + (BM + BN) * (words ? 8 : 32); }

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

template <bool X8, int BM, int BN, int WM, int WN, int NS, bool GATED, bool WORDS, bool EXACT>
__global__ __launch_bounds__(WM * WN * 64) void k_mx_tile(MxArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, XL = X8 ? 2 : 1;
    constexpr int B_OFF = BM * 128 * XL, S_OFF = B_OFF + BN * 128, STAGE = mx_stage_bytes(X8, BM, BN, WORDS), S_ROW = WORDS ? 8 : 32;
    constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, S_ALL = (BM + BN) / (WORDS ? 32 : 8), LS = (S_ALL + NW - 1) / NW;
    constexpr int LOADS = LA * XL + LB + LS;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM % (32 * WM) == 0 && BN % (32 * WN) == 0 && NW % 2 == 0, "whole loads and tiles");
    static_assert(!GATED || TN % 2 == 0, "gate and up of a column in one wavefront");
    static_assert(NS >= 2 && NS <= 4, "the waits below");
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
    const bool once = t.M <= BM && t.K % kMxStepK == 0;

    // ---- loads: instruction j covers rows 8 j .. 8 j + 7 of a line, lane l row l / 8 and the piece whose place is l % 8; wavefront w has instructions w, w + NW, ...
    const unsigned arb = (unsigned)t.K / (X8 ? 1 : 2), brb = (unsigned)t.K / 2, srb = (unsigned)t.K / kMxBlock;
    const int prow = lane >> 3;
    const unsigned kb = (unsigned)((((lane & 7) ^ (prow >> 1)) & 7) * 16) ^ ((wave & 1) ? 64u : 0u);
    const char* const base_a = (const char*)t.A + row0 * arb + (size_t)s_lo * (128 * XL);
    const char* const base_b = (const char*)t.B + (size_t)n0 * brb + (size_t)s_lo * 128;
    const char* const base_u = GATED ? (const char*)t.B2 + (size_t)n0 * brb + (size_t)s_lo * 128 : nullptr;
    const int n_last = t.N - n0 - 1;
    // row of B of a place in the tile, and whether it is one of the up projection's
    const auto b_row = [&](int i) { return min(GATED ? (i >> 6) * 32 + (i & 31) : i, n_last); };
    unsigned off_a[LA], off_b[LB], off_s[LS];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        off_a[i] = (unsigned)min(8 * (wave + NW * i) + prow, rows - 1) * arb;
        asm("" : "+v"(off_a[i]));
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        off_b[i] = (unsigned)b_row(8 * (wave + NW * i) + prow) * brb;
        asm("" : "+v"(off_b[i]));
    }
    // scales: instruction e covers S_PER rows, A's first
    constexpr int S_PER = WORDS ? 32 : 8;
    const int s_in = WORDS ? lane & 1 : lane & 7, s_row = WORDS ? lane >> 1 : lane >> 3;
    const unsigned char* s_base[LS];
    int s_at[LS];                              // (uniform) place in LDS
#pragma unroll
    for (int i = 0; i < LS; ++i) {
        const int e = (wave + NW * i) % S_ALL;    // (a few twice where they do not come out even)
        const int first = e * S_PER;
        s_at[i] = S_OFF + e * 256;
        if (first < BM) {
            s_base[i] = a.As + row0 * srb;
            off_s[i] = (unsigned)min(first + s_row, rows - 1) * srb;
        } else {
            const int i0 = first - BM;
            s_base[i] = (GATED && (i0 & 32) ? a.B2s : a.Bs) + (size_t)n0 * srb;
            off_s[i] = (unsigned)b_row(i0 + s_row) * srb;
        }
        s_base[i] += s_lo * 8;
        asm("" : "+v"(off_s[i]));
    }
    const int whole = blocks / 8;
    const int rot = t.M <= 4 * BM && whole > 0 ? (int)((unsigned)nt % (unsigned)whole) : 0;     // (dfk_tile.h)
    const unsigned a_last = (unsigned)blocks * (16 * XL) - 16, b_last = (unsigned)blocks * 16 - 16;
    const unsigned s_last = (unsigned)blocks - (WORDS ? 4 : 1);
    // load i of step `s` (past the last one it is the last one again: every step requests as many) into buffer `buf`
    const auto load_step = [&](int s, int i, int buf) {
        const int c = min(s, steps - 1);
        int st = c < whole ? c + rot : c;
        if (c < whole && st >= whole) st -= whole;
        unsigned char* const dst = lds + buf * STAGE;
        if (i < LA * XL) {
            const int j = i / XL, l = i % XL;
            unsigned o = off_a[j] + min((unsigned)st * (128u * XL) + 128u * l + kb, a_last);
            asm("" : "+v"(o));
            __builtin_amdgcn_global_load_lds(base_a + o, DFK_LDS_PTR(dst + l * (BM * 128) + (wave + NW * j) * 1024), 16, 0, 0);
        } else if (i < LA * XL + LB) {
            const int j = i - LA * XL;
            unsigned o = off_b[j] + min((unsigned)st * 128u + kb, b_last);
            asm("" : "+v"(o));
            const char* p = GATED && ((8 * (wave + NW * j)) & 32) ? base_u : base_b;
            if (once) __builtin_amdgcn_global_load_lds(p + o, DFK_LDS_PTR(dst + B_OFF + (wave + NW * j) * 1024), 16, 0, kAuxNonTemporal);
            else __builtin_amdgcn_global_load_lds(p + o, DFK_LDS_PTR(dst + B_OFF + (wave + NW * j) * 1024), 16, 0, 0);
        } else {
            const int j = i - LA * XL - LB;
            if constexpr (WORDS) {
                unsigned o = off_s[j] + min((unsigned)st * 8u + 4u * s_in, s_last);
                asm("" : "+v"(o));
                __builtin_amdgcn_global_load_lds(s_base[j] + o, DFK_LDS_PTR(dst + s_at[j]), 4, 0, 0);
            } else {
                unsigned o = off_s[j] + min((unsigned)st * 8u + s_in, s_last);
                asm("" : "+v"(o));
                __builtin_amdgcn_global_load_lds(s_base[j] + o, DFK_LDS_PTR(dst + s_at[j]), 1, 0, 0);
            }
        }
    };
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_step(s, i, s);

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
    const int as_o = S_OFF + (wm * TM * 32 + r32) * S_ROW + b * (S_ROW / 2), bs_o = S_OFF + (BM + wn * TN * 32 + r32) * S_ROW + b * (S_ROW / 2);
    u32x4 x[2][TM][XL], w[2][TN];
    unsigned xs[TM], ws[TN];
    const auto read = [&](auto t_, auto set_, int buf) {
        constexpr int T = decltype(t_)::value, SET = decltype(set_)::value;
        const unsigned char* p = lds + buf * STAGE;
        const int pa = ((X8 ? 2 * T + b : 4 * b + T) ^ sw) * 16, pb = ((4 * b + T) ^ sw) * 16;
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int l = 0; l < XL; ++l) x[SET][m][l] = *(const u32x4*)(p + l * (BM * 128) + ao + m * 4096 + pa);
#pragma unroll
        for (int n = 0; n < TN; ++n) w[SET][n] = *(const u32x4*)(p + bo + n * 4096 + pb);
    };
    const auto scale_at = [&](int at) -> unsigned {
        if constexpr (WORDS) return *(const unsigned*)(lds + at);
        const u32x4 v = *(const u32x4*)(lds + at);
        return v.x | (v.y << 8) | (v.z << 16) | (v.w << 24);
    };
    const auto read_scales = [&](unsigned (&xn)[TM], unsigned (&wn_)[TN], int buf) {
#pragma unroll
        for (int m = 0; m < TM; ++m) xn[m] = scale_at(buf * STAGE + as_o + m * 32 * S_ROW);
#pragma unroll
        for (int n = 0; n < TN; ++n) wn_[n] = scale_at(buf * STAGE + bs_o + n * 32 * S_ROW);
    };
    const auto multiply = [&](auto t_, auto set_) {
        constexpr int T = decltype(t_)::value, SET = decltype(set_)::value;
#pragma unroll
        for (int n = 0; n < TN; ++n)
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
                    acc[n][m] = mx_mfma32<X8, T>(w[SET][n], h[0], h[1], acc[n][m], ws[n], xs[m]);
                    acc[n][m] = mx_mfma32<X8, T>(w[SET][n], l[0], l[1], acc[n][m], ws[n], xs[m]);
                } else {
                    acc[n][m] = mx_mfma32<X8, T>(w[SET][n], x[SET][m][0], x[SET][m][XL - 1], acc[n][m], ws[n], xs[m]);
                }
            }
    };
    constexpr std::integral_constant<int, 0> i0{};
    constexpr std::integral_constant<int, 1> i1{};
    constexpr std::integral_constant<int, 2> i2{};
    constexpr std::integral_constant<int, 3> i3{};
    tile_wait_const<LOADS * (NS - 1)>();
    lds_barrier();
    read(i0, i0, 0);
    read_scales(xs, ws, 0);
    int buf = 0;
#pragma unroll 1
    for (int s = 0; s + 1 < steps; ++s) {
        const int next = buf + 1 == NS ? 0 : buf + 1;
        read(i1, i1, buf);
        multiply(i0, i0);
        read(i2, i0, buf);
        multiply(i1, i1);
        read(i3, i1, buf);
        multiply(i2, i0);
        tile_wait_const<LOADS * (NS - 2)>();
        lds_barrier();
        unsigned xn[TM], wn_[TN];
        read(i0, i0, next);
        read_scales(xn, wn_, next);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_step(s + NS, i, buf);
        multiply(i3, i1);
#pragma unroll
        for (int m = 0; m < TM; ++m) xs[m] = xn[m];
#pragma unroll
        for (int n = 0; n < TN; ++n) ws[n] = wn_[n];
        buf = next;
    }
    // the last step, whose blocks past the end are zeroed
    const int left = blocks - (steps - 1) * 8;
    const auto cut = [&](auto t_, auto set_) {
        constexpr int T = decltype(t_)::value, SET = decltype(set_)::value;
        if (left == 8) return;
        const u32x4 none = {0, 0, 0, 0};
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int l = 0; l < XL; ++l)
                if ((X8 ? 4 * l : 4 * b) + T >= left) x[SET][m][l] = none;
#pragma unroll
        for (int n = 0; n < TN; ++n)
            if (4 * b + T >= left) w[SET][n] = none;
    };
    cut(i0, i0);
    multiply(i0, i0);
    read(i1, i1, buf);
    cut(i1, i1);
    multiply(i1, i1);
    read(i2, i0, buf);
    cut(i2, i0);
    multiply(i2, i0);
    read(i3, i1, buf);
    cut(i3, i1);
    multiply(i3, i1);
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

template <bool X8, int BM, int BN, int WM, int WN, int NS, bool GATED, bool WORDS, bool EXACT>
hipError_t launch(const MxArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr size_t stages = (size_t)NS * mx_stage_bytes(X8, BM, BN, WORDS), end = GATED ? 0 : (size_t)WM * WN * mx_epilogue_tiles(TM, TN, WM * WN) * 32 * (TN * 32 + 4) * 4;
    constexpr size_t lds = end > stages ? end : stages;
    static_assert(lds <= (size_t)kLdsLimit, "buffers fit LDS");
    if (linear_partial_bytes(a.t.M, a.t.N, a.t.splits) > a.t.partial_bytes) return hipErrorInvalidValue;
    const auto kernel = k_mx_tile<X8, BM, BN, WM, WN, NS, GATED, WORDS, EXACT>;
    if (hipError_t e = allow_lds(allowed, (const void*)kernel, lds); e != hipSuccess) return e;
    const int cols = GATED ? BN / 2 : BN;
    const long long tiles = (long long)((a.t.M + BM - 1) / BM) * ((a.t.N + cols - 1) / cols) * a.t.splits;
    return launch_kernel(kernel, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(WM * WN * 64), lds, st, a);
}

}  // namespace

hipError_t launch_mx_linear_tile(const MxArgs& a, int x_mx, int tile, hipStream_t st) {
    const bool words = a.t.K % 128 == 0;
    (void)tile;
    if (x_mx == DFK_MXFP4) return words ? launch<false, 128, 128, 2, 4, 3, false, true, false>(a, st) : launch<false, 128, 128, 2, 4, 3, false, false, false>(a, st);
    if (mx_exact_sums(a.t.M, a.t.out_fp32)) return words ? launch<true, 128, 128, 2, 4, 2, false, true, true>(a, st) : launch<true, 128, 128, 2, 4, 2, false, false, true>(a, st);
    return words ? launch<true, 128, 128, 2, 4, 2, false, true, false>(a, st) : launch<true, 128, 128, 2, 4, 2, false, false, false>(a, st);
}

hipError_t launch_mx_gateup_tile(const MxArgs& a, int x_mx, int tile, hipStream_t st) {
    const bool words = a.t.K % 128 == 0;
    (void)tile;
    if (x_mx == DFK_MXFP4) return words ? launch<false, 128, 128, 4, 2, 3, true, true, false>(a, st) : launch<false, 128, 128, 4, 2, 3, true, false, false>(a, st);
    if (mx_exact_sums(a.t.M, 0)) return words ? launch<true, 128, 128, 4, 2, 2, true, true, true>(a, st) : launch<true, 128, 128, 4, 2, 2, true, false, true>(a, st);
    return words ? launch<true, 128, 128, 4, 2, 2, true, true, false>(a, st) : launch<true, 128, 128, 4, 2, 2, true, false, false>(a, st);
}

}  // namespace dfk
