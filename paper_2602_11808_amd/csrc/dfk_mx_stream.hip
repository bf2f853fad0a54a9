// Products with MXFP4 weights on the scaled matrix instructions, few rows: the weights stream through LDS once, past activations that stay there.
//
// A workgroup goes from unit to unit of 16 NT WU weight rows (gated: the 16 WU columns whose gate and up rows they are).  Wavefront (wk, wu) multiplies tiles of 16 rows of part wu in
// chunks wk, wk + WK, ... of 256 LN k, against all rows of the activations.  It has a ring of D chunks of its own in LDS, filled by asynchronous loads that run on through the ends of units,
// and waits for nobody but its own loads until a unit's sums meet in LDS, where they are added in order.
// A chunk is a cache line (LN = 2: two) of each weight row and eight scales for each: loads, swizzle and scales as in dfk_mx_tile.hip.  Product j (0, 1) of a line takes blocks 2 g + j
// (g: lane / 16), so that a lane's two scales are one halfword.
//
// What bounds it: the weights' bytes.  4096 -> 50257, MXFP4, 112.6 MB: 19.9 us, which is 3.6 us for an empty stream of units (start, first loads' latency, end) and then 6.9 TB/s, what plain
// reads of memory reach.  Two lines a row where rows are long, since neighbouring lines asked for together come faster: 1 x 8192 -> 28672 25.5 -> 24.9 us in MXFP8 and 25.1 -> 24.0 in
// MXFP4 with eight wavefronts (rings of two such chunks 23.6 and 22.4, but more on shorter rows), and 22.3 and 21.0 with whole kilobytes of a row an instruction, which would not feed the matrix instructions' rows.  Without the loads of scales (6 % of the bytes) it takes 6 to
// 9 % less, without multiplications 3 % less; cached loads instead of non-temporal ones take 4 to 10 % more.  With MXFP8 activations of 16 rows the products, each done twice, no longer hide:
// forms with two tiles a wavefront, which split the activations once for both, 16 x 4096 -> 50257 26.7 -> 23.7 us.
#include "dfk_epilogue.h"
#include "dfk_mx_device.h"
#include "dfk_mx_plan.h"

namespace dfk {
namespace {

// v_mfma_scale_f32_16x16x128_f8f6f4, MXFP4 weights (16 rows) first.  Lane (q, g) holds of the weights row q, block g; of MXFP4 activations the same; of MXFP8 ones elements 16 (g & 1)
// .. + 15 of blocks g / 2 and 2 + g / 2.  Result: row q of the activations, columns 4 g .. 4 g + 3.
template <bool X8, int SEL>
__device__ __forceinline__ f32x4 mx_mfma16(const u32x4& w, const u32x4& x0, const u32x4& x1, const f32x4& c, unsigned ws, unsigned xs) {
    const i32x8 a = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
    typedef float v4 __attribute__((ext_vector_type(4)));
    union { f32x4 f; v4 v; } u;
    u.f = c;
    if constexpr (X8) {
        const i32x8 b = {(int)x0.x, (int)x0.y, (int)x0.z, (int)x0.w, (int)x1.x, (int)x1.y, (int)x1.z, (int)x1.w};
        u.v = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, u.v, 4, 0, SEL, (int)ws, SEL, (int)xs);
    } else {
        const i32x8 b = {(int)x0.x, (int)x0.y, (int)x0.z, (int)x0.w, 0, 0, 0, 0};
        u.v = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, u.v, 4, 4, SEL, (int)ws, SEL, (int)xs);
    }
    return u.f;
}

__device__ __forceinline__ void lds_write_b8_raw(unsigned addr, unsigned v) { asm volatile("ds_write_b8 %0, %1" : : "v"(addr), "v"(v) : "memory"); }

// Waits until the loads of all but the newest `newer` (at most D - 1, uniform) chunks are there.
template <int LOADS, int D>
__device__ __forceinline__ void mx_stream_wait(int newer) {
    static_assert(LOADS * (D - 1) <= 63, "counts of s_waitcnt");
    if constexpr (D > 1) {
        if (newer < D - 1) return mx_stream_wait<LOADS, D - 1>(newer);
    }
    DFK_WAIT_VM(LOADS * (D - 1));
    asm volatile("" ::: "memory");
}

template <bool X8, int NT, int LN, int TT, int WK, int WU, int D, bool GATED, bool WORDS>
__global__ __launch_bounds__(WK * WU * 64) void k_mx_stream(MxArgs a, int x_pitch) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr int NW = WK * WU, XL = X8 ? 2 : 1;
    constexpr int STAGE = mx_stream_stage(NT, LN, WORDS), TILE = LN * 2048, S_OFF = NT * TILE, LS = WORDS ? (NT * LN + 1) / 2 : 2 * NT * LN, LOADS = 2 * NT * LN + LS;
    constexpr int ROWS = 8 / LN, PCS = 8 * LN;        // rows of a load instruction, pieces of a row
    constexpr int RED = NW * D * STAGE, X_OFF = RED + NW * NT * TT * 1024;
    constexpr int COLS = 16 * WU * (GATED ? 1 : NT);
    static_assert(!GATED || (NT == 2 && WU == 2), "a unit of the gated half is an MX block of its result");
    const TileArgs& t = a.t;
    const int tid = threadIdx.x, lane = tid & 63, q = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = wave % WK, wu = wave / WK;
    const int M = t.M, blocks = t.K / kMxBlock, chunks = (blocks + PCS - 1) / PCS;
    const int units = (t.N + COLS - 1) / COLS, step = (int)gridDim.x;
    const unsigned xb = (unsigned)t.K / (X8 ? 1 : 2), rb = (unsigned)t.K / 2, srb = (unsigned)blocks;
    const int xs_off = X_OFF + M * x_pitch;

    // ---- activations: 1 KB of a row an instruction, the rows 16 bytes off each other's banks; their scales as they lie in memory, but where rows of scales start in the same banks their
    // 16-byte pieces change places by row (32 x 4096 -> 14336 in MXFP4 10.8 -> 10.2 us)
    const int xs_shift = srb % 256 == 0 ? 0 : srb % 128 == 0 ? 1 : srb % 64 == 0 ? 2 : 4;
    const unsigned xs_all = (unsigned)M * srb, xs_whole = xs_all & ~15u;
    unsigned tail = 0;
    if (tid < (int)(xs_all - xs_whole)) tail = a.As[xs_whole + tid];
    {
        const int per = (x_pitch - 16) >> 10;
        for (int e = wave; e < M * per; e += NW) {
            const int r = e / per, p = e - r * per;
            const char* src = (const char*)t.A + (size_t)r * xb;
            unsigned o = min((unsigned)p * 1024u + lane * 16u, xb - 16u);
            asm("" : "+v"(o));
            __builtin_amdgcn_global_load_lds(src + o, DFK_LDS_PTR(lds + X_OFF + r * x_pitch + p * 1024), 16, 0, 0);
        }
        for (unsigned e = wave * 1024u; e < xs_whole; e += NW * 1024u) {
            unsigned o = e + lane * 16u;
            if (o < xs_whole) {
                if (xs_shift < 4) {
                    const unsigned r = o / srb, in = o - r * srb;
                    o = r * srb + (in ^ (((r & 15) >> xs_shift) * 16u));
                }
                __builtin_amdgcn_global_load_lds(a.As + o, DFK_LDS_PTR(lds + xs_off + e), 16, 0, 0);
            }
        }
    }

    // ---- the weight stream.  In LDS a tile's row is its 8 LN pieces, XOR-swizzled so that an operand read of 16 rows covers all banks as often as it has to
    const auto swizzle = [](int r) { return LN == 1 ? (r >> 1) & 7 : r & 15; };
    unsigned char* const ring = lds + wave * (D * STAGE);
    unsigned w_off[2 * LN], w_pc[2 * LN];       // row of this lane's loads in a tile, and piece
#pragma unroll
    for (int h = 0; h < 2 * LN; ++h) {
        const int r = ROWS * h + lane / PCS;
        w_off[h] = (unsigned)r * rb;
        w_pc[h] = (unsigned)((lane % PCS) ^ swizzle(r)) * 16u;
    }
    const int unit0 = (int)blockIdx.x;
    const int mine = chunks > wk ? (chunks - wk + WK - 1) / WK : 0;
    const int my_units = (units - unit0 + step - 1) / step, total = mine * my_units;
    int l_unit = unit0, l_chunk = wk, l_slot = 0;
    const auto load = [&]() {
        unsigned char* const dst = ring + l_slot * STAGE;
        const int row0 = l_unit * COLS + wu * (GATED ? 16 : 16 * NT);      // first row of the wavefront's first tile
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int first = min(GATED ? row0 : row0 + 16 * n, t.N - 1);
            const char* const base = (const char*)(GATED && n == 1 ? t.B2 : t.B) + (size_t)first * rb;
            const unsigned last = (unsigned)min(t.N - 1 - first, 15) * rb;      // (of a tile's 16: within 32 bits)
#pragma unroll
            for (int h = 0; h < 2 * LN; ++h) {
                unsigned o = min(w_off[h], last) + min((unsigned)l_chunk * (128u * LN) + w_pc[h], rb - 16u);
                asm("" : "+v"(o));
                __builtin_amdgcn_global_load_lds(base + o, DFK_LDS_PTR(dst + n * TILE + h * 1024), 16, 0, kAuxNonTemporal);
            }
        }
#pragma unroll
        for (int e = 0; e < LS; ++e) {
            constexpr int E = WORDS ? 2 * LN : PCS, PER = 64 / E;        // lanes of a row, rows of an instruction
            const int at = e * PER + lane / E, n = NT == 1 ? 0 : at >> 4, r = at & 15;
            const unsigned char* const s = GATED && n == 1 ? a.B2s : a.Bs;
            const int row = min(GATED ? row0 + r : row0 + 16 * n + r, t.N - 1);
            const unsigned char* const p = s + (size_t)row * srb;
            if constexpr (WORDS) __builtin_amdgcn_global_load_lds(p + min((unsigned)l_chunk * PCS + 4u * (lane % E), srb - 4u), DFK_LDS_PTR(dst + S_OFF + e * 256), 4, 0, 0);
            else __builtin_amdgcn_global_load_lds(p + min((unsigned)l_chunk * PCS + (lane % E), srb - 1u), DFK_LDS_PTR(dst + S_OFF + e * 256), 1, 0, 0);
        }
        l_slot = l_slot + 1 == D ? 0 : l_slot + 1;
        l_chunk += WK;
        if (l_chunk >= chunks) {
            l_chunk = wk;
            l_unit += step;
        }
    };
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (d < total) load();
    if (tid < (int)(xs_all - xs_whole)) lds_write_b8_raw(lds_addr(lds) + xs_off + xs_whole + tid, tail);
    if (total >= D) DFK_WAIT_VM(LOADS * D < 63 ? LOADS * D : 63);
    else DFK_WAIT_VM(0);
    asm volatile("" ::: "memory");
    lds_barrier();

    int x_row[TT], xs_swap[TT];
#pragma unroll
    for (int m = 0; m < TT; ++m) {
        x_row[m] = min(16 * m + q, M - 1);
        xs_swap[m] = ((x_row[m] & 15) >> xs_shift) * 16;
    }
    int slot = 0, done = 0;
    for (int unit = unit0; unit < units; unit += step) {
        f32x4 acc[NT][TT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < TT; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int c = wk; c < chunks; c += WK) {
            mx_stream_wait<LOADS, D>(total - 1 - done);
            const unsigned char* const src = ring + slot * STAGE;
#pragma unroll
            for (int half = 0; half < LN; ++half) {
                const int line = c * LN + half;
                u32x4 w[2][NT];
                unsigned ws[NT], xs[TT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) w[j][n] = *(const u32x4*)(src + n * TILE + q * (128 * LN) + ((8 * half + 2 * g + j) ^ swizzle(q)) * 16);
                    if constexpr (WORDS) {
                        ws[n] = *(const unsigned short*)(src + S_OFF + (n * 16 + q) * PCS + 8 * half + 2 * g);
                    } else {
                        const uint2 v = *(const uint2*)(src + S_OFF + (n * 16 + q) * (4 * PCS) + 32 * half + 8 * g);
                        ws[n] = v.x | (v.y << 8);
                    }
                }
                u32x4 x[2][TT][XL];
#pragma unroll
                for (int m = 0; m < TT; ++m) {
                    const unsigned char* const p = lds + X_OFF + x_row[m] * x_pitch + line * (128 * XL);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if constexpr (X8) {
                            x[j][m][0] = *(const u32x4*)(p + 32 * (2 * (g >> 1) + j) + 16 * (g & 1));
                            x[j][m][1] = *(const u32x4*)(p + 128 + 32 * (2 * (g >> 1) + j) + 16 * (g & 1));
                        } else {
                            x[j][m][0] = *(const u32x4*)(p + (2 * g + j) * 16);
                        }
                    }
                    const unsigned char* const s = lds + xs_off + x_row[m] * srb + ((line * 8 + 2 * g) ^ xs_swap[m]);
                    if constexpr (WORDS) xs[m] = *(const unsigned short*)s;
                    else xs[m] = (unsigned)s[0] | ((unsigned)s[1] << 8);
                }
                if ((line + 1) * 8 > blocks) {        // the line that ends early: blocks past the end are zeros with scales that are not NaN
                    const u32x4 none = {0, 0, 0, 0};
                    const int left = blocks - line * 8;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (2 * g + j >= left) {
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                w[j][n] = none;
                                ws[n] &= ~(0xFFu << (8 * j));
                            }
#pragma unroll
                            for (int m = 0; m < TT; ++m) xs[m] &= ~(0xFFu << (8 * j));
                        }
#pragma unroll
                        for (int m = 0; m < TT; ++m)
#pragma unroll
                            for (int l = 0; l < XL; ++l)
                                if ((X8 ? 4 * l + 2 * (g >> 1) : 2 * g) + j >= left) x[j][m][l] = none;
                    }
                }
                const auto multiply = [&](auto j_) {
                    constexpr int J = decltype(j_)::value;
#pragma unroll
                    for (int m = 0; m < TT; ++m) {
                        if constexpr (X8) {
                            u32x4 h[2], l[2];
#pragma unroll
                            for (int k = 0; k < 2; ++k)
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    h[k][i] = mx_fp8_large(x[J][m][k][i]);
                                    l[k][i] = x[J][m][k][i] ^ h[k][i];
                                }
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                acc[n][m] = mx_mfma16<true, J>(w[J][n], h[0], h[1], acc[n][m], ws[n], xs[m]);
                                acc[n][m] = mx_mfma16<true, J>(w[J][n], l[0], l[1], acc[n][m], ws[n], xs[m]);
                            }
                        } else {
#pragma unroll
                            for (int n = 0; n < NT; ++n) acc[n][m] = mx_mfma16<false, J>(w[J][n], x[J][m][0], x[J][m][0], acc[n][m], ws[n], xs[m]);
                        }
                    }
                };
                multiply(std::integral_constant<int, 0>{});
                multiply(std::integral_constant<int, 1>{});
            }
            __builtin_amdgcn_sched_barrier(0);     // (the operands are in registers before their place is filled again)
            slot = slot + 1 == D ? 0 : slot + 1;
            ++done;
            if (done + D - 1 < total) load();
        }

        // ---- the unit's sums: [wavefront][tile][lane] in LDS, added over wk in order
        if (unit != unit0) lds_barrier();      // (the last unit's have been read)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < TT; ++m) lds_write_b128_raw(lds_addr(lds) + RED + ((wave * NT + n) * TT + m) * 1024 + lane * 16, acc[n][m]);
        lds_barrier();
        const auto sum = [&](int part, int n, int r, int gg) {
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < WK; ++k) s += *(const f32x4*)(lds + RED + (((part * WK + k) * NT + n) * TT + (r >> 4)) * 1024 + (gg * 16 + (r & 15)) * 16);
            return s;
        };
        if constexpr (GATED) {
            for (int idx = tid; idx < M * 8; idx += NW * 64) {
                const int r = idx >> 3, v = idx & 7;
                const f32x4 sg = sum(v >> 2, 0, r, v & 3), su = sum(v >> 2, 1, r, v & 3);
                const size_t at = (size_t)r * t.N + unit * 32 + 4 * v;
                float f[4];
                if (a.out_mx < 0) {
                    silu_mul_all<false>(sg, su, f);
                    if (a.dtype == DFK_BF16) BF16::store4(t.out, at, f[0], f[1], f[2], f[3]);
                    else FP16::store4(t.out, at, f[0], f[1], f[2], f[3]);
                } else {
                    silu_mul_all<true>(sg, su, f);
                    unsigned top = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = mx_top(top, f[i]);
#pragma unroll
                    for (int o = 1; o < 8; o *= 2) top = max(top, (unsigned)__shfl_xor((int)top, o));
                    const unsigned s = a.out_mx == DFK_MXFP4 ? mx_scale_of<DFK_MXFP4>(top) : mx_scale_of<DFK_MXFP8>(top);
                    if (a.out_mx == DFK_MXFP4) ((unsigned short*)a.q)[at >> 2] = (unsigned short)mx_elements<DFK_MXFP4>(f, s);
                    else ((unsigned*)a.q)[at >> 2] = mx_elements<DFK_MXFP8>(f, s);
                    if (v == 0) a.qs[at >> 5] = (unsigned char)s;
                }
            }
        } else {
            constexpr int CV = COLS / 4;
            for (int idx = tid; idx < M * CV; idx += NW * 64) {
                const int r = idx / CV, v = idx - r * CV, tile = v >> 2;
                const f32x4 s = sum(tile / NT, tile % NT, r, v & 3);
                const float f[4] = {s[0], s[1], s[2], s[3]};
                const int col = unit * COLS + 4 * v;
                if (a.dtype == DFK_BF16) {
                    if (t.out_fp32) linear_store4<BF16, FP32>(t, r, col, f);
                    else linear_store4<BF16, BF16>(t, r, col, f);
                } else {
                    if (t.out_fp32) linear_store4<FP16, FP32>(t, r, col, f);
                    else linear_store4<FP16, FP16>(t, r, col, f);
                }
            }
        }
    }
}

template <bool X8, int NT, int LN, int TT, int WK, int WU, int D, bool GATED, bool WORDS>
hipError_t launch(const MxArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    const size_t lds = mx_stream_lds(MxStream{NT, LN, WK, WU, D, {}, {}}, X8, a.t.M, a.t.K);
    if (lds > kMxLds || a.t.M > 16 * TT || WORDS != (a.t.K % 128 == 0)) return hipErrorInvalidValue;
    const auto kernel = k_mx_stream<X8, NT, LN, TT, WK, WU, D, GATED, WORDS>;
    if (hipError_t e = allow_lds(allowed, (const void*)kernel, lds); e != hipSuccess) return e;
    constexpr int COLS = 16 * WU * (GATED ? 1 : NT);
    const int units = (a.t.N + COLS - 1) / COLS, slots = kLinearCus * mx_stream_per_cu(lds);
    return launch_kernel(kernel, dim3((unsigned)(units < slots ? units : slots)), dim3(WK * WU * 64), lds, st, a, mx_x_pitch(X8, a.t.K));
}

// kMxStreams, mx_stream_offered
template <int FORM, bool X8, int TT, bool WORDS>
hipError_t of_form(const MxArgs& a, hipStream_t st) {
    constexpr MxStream f = kMxStreams[FORM];
    if constexpr (!mx_stream_offered(FORM, X8, TT, WORDS)) return hipErrorInvalidValue;
    else return launch<X8, f.nt, f.lines, TT, f.wk, f.wu, f.depth, (FORM >= kMxStreamGated), WORDS>(a, st);
}
template <bool X8, int TT, bool WORDS>
hipError_t linear_of(const MxArgs& a, int form, hipStream_t st) {
    static_assert(kMxStreamGated == 5, "the cases");
    switch (form) {
        case 0: return of_form<0, X8, TT, WORDS>(a, st);
        case 1: return of_form<1, X8, TT, WORDS>(a, st);
        case 2: return of_form<2, X8, TT, WORDS>(a, st);
        case 3: return of_form<3, X8, TT, WORDS>(a, st);
        case 4: return of_form<4, X8, TT, WORDS>(a, st);
    }
    return hipErrorInvalidValue;
}
template <bool X8, int TT, bool WORDS>
hipError_t gateup_of(const MxArgs& a, int form, hipStream_t st) {
    static_assert(kMxStreamCount == 7, "the cases");
    switch (form) {
        case 5: return of_form<5, X8, TT, WORDS>(a, st);
        case 6: return of_form<6, X8, TT, WORDS>(a, st);
    }
    return hipErrorInvalidValue;
}
template <bool GATED, bool X8, bool WORDS>
hipError_t by_rows(const MxArgs& a, int form, hipStream_t st) {
    const auto of = [&](auto tt_) {
        constexpr int TT = decltype(tt_)::value;
        if constexpr (GATED) return gateup_of<X8, TT, WORDS>(a, form, st);
        else return linear_of<X8, TT, WORDS>(a, form, st);
    };
    switch (mx_stream_tiles(a.t.M)) {
        case 1: return of(std::integral_constant<int, 1>{});
        case 2: return of(std::integral_constant<int, 2>{});
        case 4: return of(std::integral_constant<int, 4>{});
    }
    return hipErrorInvalidValue;
}
template <bool GATED>
hipError_t by_format(const MxArgs& a, int x_mx, int form, hipStream_t st) {
    const bool words = a.t.K % 128 == 0;
    if (x_mx == DFK_MXFP8) return words ? by_rows<GATED, true, true>(a, form, st) : by_rows<GATED, true, false>(a, form, st);
    return words ? by_rows<GATED, false, true>(a, form, st) : by_rows<GATED, false, false>(a, form, st);
}

}  // namespace

hipError_t launch_mx_linear_stream(const MxArgs& a, int x_mx, int form, hipStream_t st) { return by_format<false>(a, x_mx, form, st); }
hipError_t launch_mx_gateup_stream(const MxArgs& a, int x_mx, int form, hipStream_t st) { return by_format<true>(a, x_mx, form, st); }

}  // namespace dfk
