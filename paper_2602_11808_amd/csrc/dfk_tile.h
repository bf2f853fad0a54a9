// Matrix products of 16-bit operands on the matrix cores for many rows: the tile kernel of the linear layers (the experts' has a copy of its step loop, with
// waits of its own).
//
// out[m, n] = sum_k A[m, k] B[n, k].  A workgroup of eight wavefronts (WM x WN) owns BM rows of A and BN rows of B; wavefront (wm, wn) a
// BM/WM x BN/WN share of the products, TN x TM tiles of v_mfma_f32_16x16x32 with B's rows as the first operand: lane (q, g) of
// a result holds row q of A and four adjacent columns.
//
// Data movement: asynchronous global->LDS loads of 64 k a step (one cache line per row), NS steps deep.  In LDS a tile of 16 rows is
// 2 KB, the eight 16-byte pieces of row i XOR-swizzled by i / 2, so that an operand read of 16 rows covers all banks once.
// A step is two halves of 32 k; beside the multiplications of one half a wavefront reads the operands of the next.  There is one
// barrier per step, between its halves: before it every wavefront has its operands of the second half in registers and has waited, by count, for its own loads
// of the following step; behind it that step is whole in LDS, and this step's buffer is free for the loads of step s + NS.
//
// The last step of a K that is no multiple of 64 loads clamped pieces and zeroes the operands past the end in both factors.  LINES, for such K: a step brings in each row's own
// next line (one more than it has steps) instead of 64 k that straddle two, and an operand's 16-byte piece is found by its row's offset in this step's buffer or the next one's, which has
// to be there a step sooner.  128 x 128 tiles, us, straddling / by lines: 80 x 2872 -> 7680 41 / 30, 600 x 2040 -> 30000 142 / 117, 4000 x 2872 -> 7680 281 / 226.
// Rows past the end are copies of the last one and are not stored.
#pragma once

#include <type_traits>

#include "dfk_epilogue.h"
#include "dfk_mfma_common.h"

namespace dfk {
namespace {

constexpr int kTileStepK = 64;
constexpr int kTile16 = 2048;        // 16 rows x 128 bytes

template <int N>
__device__ __forceinline__ void tile_wait_const() {
    DFK_WAIT_VM(N < 63 ? N : 63);
    asm volatile("" ::: "memory");
}

// The tile of a workgroup: the launch's workgroups b, b + 8, ... sit on one XCD and get neighbouring tiles, in groups of kGroupM row tiles
// that run through the columns together, so that the tiles that an XCD works on at a time share rows of both operands in its L2 (us with 1 / 2 / 4 / 8 row tiles: layers of
// 4096 x 4096 -> 14336 394 / 388 / 382 / 381, 4096 x 14336 -> 4096 380 / 378 / 366 / 363, 128 x 4096 -> 50257 84 / 85 / 85 / 86; experts, 4096 tokens, 2 of 8 of 4096 x 4096 977 / 880 /
// 812 / 818, 300, 4 of 32 of 4096 x 1024 170 / 171 / 173 / 182).
constexpr int kGroupM = 4;
__device__ __forceinline__ void tile_at(unsigned idx, int m_tiles, int n_tiles, int& mt, int& nt) {
    const unsigned gsize = kGroupM * (unsigned)n_tiles, grp = idx / gsize, r = idx - grp * gsize;
    const unsigned first = grp * kGroupM, gm = min((unsigned)kGroupM, (unsigned)m_tiles - first);
    nt = (int)(r / gm);
    mt = (int)(first + (r - (unsigned)nt * gm));
}
__device__ __forceinline__ bool tile_of(int m_tiles, int n_tiles, int& mt, int& nt) {
    const unsigned total = (unsigned)m_tiles * (unsigned)n_tiles, per = (total + 7) / 8;
    const unsigned b = blockIdx.x >> 3, idx = (blockIdx.x & 7) * per + b;
    if (b >= per || idx >= total) return false;
    tile_at(idx, m_tiles, n_tiles, mt, nt);
    return true;
}

// Row tiles that go through LDS together at the end, a power of two that divides TM.
constexpr int tile_epilogue_tiles(int TM, int TN, int NW) {
    int pm = TM;
    while (pm > 1 && (size_t)NW * pm * 16 * (TN * 16 + 4) * 4 > (size_t)kLdsLimit) pm /= 2;
    return pm;
}

template <typename E, int BM, int BN, int WM, int WN, int NS, bool LINES>
__global__ __launch_bounds__(WM * WN * 64) void k_tile(TileArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr int NW = WM * WN;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int STAGE = (BM + BN) * 128, B_OFF = BM * 128;
    constexpr int LA = BM / 8 / NW, LB = (BN / 8 + NW - 1) / NW, LOADS = LA + LB;    // load instructions (8 rows each) of a wavefront and step
    constexpr bool EVEN = BN % (8 * NW) == 0;      // else the later wavefronts have one less
    static_assert(BM % (8 * NW) == 0 && (EVEN || NS == 2) && BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "whole loads and tiles");
    static_assert(NS >= 2 && NS <= 4 && (!LINES || NS >= 3), "the waits below");
    constexpr int NEWER = LOADS * (NS - (LINES ? 3 : 2));      // loads that may be under way when the next step's have to be there
    static_assert(NW % 2 == 0, "a wavefront's loads are all of one half of their tiles");
    const int tid = threadIdx.x, lane = tid & 63, q = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    const int n_tiles = (a.N + BN - 1) / BN;
    int mt, nt;
    if (!tile_of((a.M + BM - 1) / BM, n_tiles * a.splits, mt, nt)) return;
    const int k_split = nt / n_tiles;
    nt -= k_split * n_tiles;
    const size_t row0 = (size_t)mt * BM;
    const int rows = min(BM, a.M - (int)row0), n0 = nt * BN;
    int k_lo = 0, steps = (a.K + kTileStepK - 1) / kTileStepK;
    if (a.splits > 1) {
        int s1;
        share_of((unsigned)steps, (unsigned)a.splits, (unsigned)k_split, k_lo, s1);
        steps = s1 - k_lo;
        k_lo *= kTileStepK;
    }
    const int k_end = min(a.K, k_lo + steps * kTileStepK);     // (a split that ends early ends at a whole step)

    // Rows of B that one workgroup alone reads leave the caches to others; not where they are off the lines, whose ends two steps share.
    const bool once = a.M <= BM && (LINES || a.K % kTileStepK == 0);
    // ---- loads: instruction i of this wavefront covers rows 8 (wave + NW i) .. + 7, lane l row l / 8 and the piece whose place is l % 8
    const unsigned rb = (unsigned)a.K * 2;
    const int prow = lane >> 3;
    const unsigned kb = (unsigned)((((lane & 7) ^ (prow >> 1)) & 7) * 16) ^ ((wave & 1) ? 64u : 0u);
    const char* base_a = (const char*)a.A + row0 * rb + (size_t)k_lo * 2;
    const char* base_b = (const char*)a.B + (size_t)n0 * rb + (size_t)k_lo * 2;
    unsigned off_a[LA], off_b[LB];
    int at_a[LINES ? LA : 1], at_b[LINES ? LB : 1];            // LINES: place of a load's piece in its row, less what the row is off its line
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int r = min(8 * (wave + NW * i) + prow, rows - 1);
        off_a[i] = (unsigned)r * rb + (LINES ? 0u : kb);
        if constexpr (LINES) at_a[i] = (int)kb - ((int)((uintptr_t)base_a + off_a[i]) & 127);
        asm("" : "+v"(off_a[i]));             // (one register: out of the multiplication it would keep two)
    }
    const int n_last = a.N - n0 - 1;
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        off_b[i] = (unsigned)min(8 * (wave + NW * i) + prow, n_last) * rb + (LINES ? 0u : kb);
        if constexpr (LINES) at_b[i] = (int)kb - ((int)((uintptr_t)base_b + off_b[i]) & 127);
        asm("" : "+v"(off_b[i]));
    }
    // in the last, partial step a piece past the end is replaced by the last one there is
    const unsigned k_left = (unsigned)(k_end - k_lo - (steps - 1) * kTileStepK) * 2;
    const unsigned tail_off = kb + 16 > k_left ? kb + 16 - k_left : 0u;
    const auto load = [&](int i, unsigned o, const char* pa, const char* pb, unsigned char* dst) {
        asm("" : "+v"(o));                    // 32 bits from a scalar base, not a 64-bit sum of its own
        const int j = NW * (i < LA ? i : i - LA);
        if (!EVEN && i == LOADS - 1 && wave + j >= BN / 8) return;
        const char* p = i < LA ? pa : pb;
        if (i >= LA && once) __builtin_amdgcn_global_load_lds(p + o, DFK_LDS_PTR(dst + B_OFF + j * 1024), 16, 0, kAuxNonTemporal);
        else __builtin_amdgcn_global_load_lds(p + o, DFK_LDS_PTR(dst + (i < LA ? 0 : B_OFF) + j * 1024), 16, 0, 0);
    };

    // The sums begin with the bias: read at the end, between stores, each of its loads was a trip to memory (4096 x 4096 -> 14336 with GELU 447 -> 440 us, 200 x 1024 -> 4097
    // 15.1 -> 13.4).
    f32x4 acc[TN][TM];
#pragma unroll
    for (int n = 0; n < TN; ++n) {
        float b[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.bias && a.splits == 1) {
            const int col = n0 + (wn * TN + n) * 16 + 4 * g;
            if (a.vec4) {
                if (col < a.N) E::load4(a.bias, col, b);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (col + i < a.N) b[i] = E::load1(a.bias, col + i);
            }
        }
#pragma unroll
        for (int m = 0; m < TM; ++m) acc[n][m] = f32x4{b[0], b[1], b[2], b[3]};
    }

    // A step past the last one is the last one again: every step requests one, and the waits count the same number throughout.
    const int whole = (k_end - k_lo) / kTileStepK;
    // Workgroups start at different steps: in lock-step they would all ask for the same few columns, whose lines lie in few memory channels where
    // rows are a power of two apart (64 x 4096 -> 14336: 29.3 -> 26.6 us, 128 x 4096 -> 50257: 105 -> 93).  Neighbours of many row
    // tiles, which share B, keep in step.
    const int rot = !LINES && a.M <= 4 * BM && whole > 0 ? (int)((unsigned)nt % (unsigned)whole) : 0;
    const auto load_step = [&](int step, int i, int buf) {
        if constexpr (LINES) {                // lines 0 .. steps of a row; pieces outside it are its first or last one
            const unsigned o = (i < LA ? off_a[i] : off_b[i - LA]) +
                               (unsigned)min(max(min(step, steps) * (kTileStepK * 2) + (i < LA ? at_a[i] : at_b[i - LA]), 0), (k_end - k_lo) * 2 - 16);
            load(i, o, base_a, base_b, lds + buf * STAGE + wave * 1024);
        } else {
            const int t = min(step, steps - 1);
            int tr = t < whole ? t + rot : t;
            if (t < whole && tr >= whole) tr -= whole;
            const size_t k = (size_t)tr * (kTileStepK * 2);
            load(i, (i < LA ? off_a[i] : off_b[i - LA]) - (t == steps - 1 ? tail_off : 0u), base_a + k, base_b + k, lds + buf * STAGE + wave * 1024);
        }
    };
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_step(s, i, s);

    // operand of lane (q, g) in a tile: row q, piece 4 half + g
    const int lo = q * 128 + ((g ^ (q >> 1)) & 7) * 16;
    const int ao = wm * TM * kTile16 + lo, bo = B_OFF + wn * TN * kTile16 + lo;
    u32x4 x[2][TM], w[2][TN];
    // LINES: places of the operands' pieces, of half 0 and 1, and whether in the next step's buffer (sixteen rows are a multiple of 128 bytes: all tiles are alike)
    int a_off[2] = {0, 0}, b_off[2] = {0, 0};
    bool a_next[2] = {false, false}, b_next[2] = {false, false};
    if constexpr (LINES) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int pa = 4 * j + g + (int)(((uintptr_t)base_a + (unsigned)q * rb) & 127) / 16, pb = 4 * j + g + (int)(((uintptr_t)base_b + (unsigned)q * rb) & 127) / 16;
            a_off[j] = wm * TM * kTile16 + q * 128 + ((pa ^ (q >> 1)) & 7) * 16;
            b_off[j] = B_OFF + wn * TN * kTile16 + q * 128 + ((pb ^ (q >> 1)) & 7) * 16;
            a_next[j] = pa >= 8;
            b_next[j] = pb >= 8;
        }
    }
    tile_wait_const<(EVEN ? LOADS : LOADS - 1) * (NS - (LINES ? 2 : 1))>();     // (of the step's loads at least)
    lds_barrier();
    // Multiplications of one half (operands `cur`) beside the reads of the next (half H of buffer `buf`, with READ) and the loads of step `ls`
    // into `lbuf` (with LOAD): the three in turn, so that none of the units waits for another's block to end.
    const auto half = [&](auto cur_, auto read_, int buf, auto load_, int ls, int lbuf) {
        constexpr int cur = decltype(cur_)::value, nxt = cur ^ 1, H = nxt;
        constexpr bool READ = decltype(read_)::value, LOAD = decltype(load_)::value;
        const int on = buf + 1 == NS ? -(NS - 1) * STAGE : STAGE;
        const unsigned char* as = lds + buf * STAGE + (LINES ? a_off[H] + (a_next[H] ? on : 0) : ao ^ (64 * H));
        const unsigned char* bs = lds + buf * STAGE + (LINES ? b_off[H] + (b_next[H] ? on : 0) : bo ^ (64 * H));
#pragma unroll
        for (int n = 0; n < TN; ++n) {
            if (READ) {
#pragma unroll
                for (int m = n * TM / TN; m < (n + 1) * TM / TN; ++m) x[nxt][m] = *(const u32x4*)(as + m * kTile16);
                w[nxt][n] = *(const u32x4*)(bs + n * kTile16);
            }
            if (LOAD) {
#pragma unroll
                for (int i = n * LOADS / TN; i < (n + 1) * LOADS / TN; ++i) load_step(ls, i, lbuf);
            }
            __builtin_amdgcn_s_setprio(1);     // of the two wavefronts of a SIMD, the one that multiplies goes first
#pragma unroll
            for (int m = 0; m < TM; ++m) acc[n][m] = mfma16<E>(w[cur][n], x[cur][m], acc[n][m]);
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr auto c0 = std::integral_constant<int, 0>{};
    constexpr auto c1 = std::integral_constant<int, 1>{};
    constexpr auto yes = std::true_type{};
    constexpr auto no = std::false_type{};
#pragma unroll
    for (int m = 0; m < TM; ++m) x[0][m] = *(const u32x4*)(lds + (LINES ? a_off[0] + (a_next[0] ? STAGE : 0) : ao) + m * kTile16);
#pragma unroll
    for (int n = 0; n < TN; ++n) w[0][n] = *(const u32x4*)(lds + (LINES ? b_off[0] + (b_next[0] ? STAGE : 0) : bo) + n * kTile16);
    int buf = 0;
    // A wavefront whose rows are all past the end only loads: of the two wavefronts of its SIMD the other one then goes twice as fast (rows wm and
    // wm + WM / 2 are on one SIMD).
    if (wm * TM * 16 >= rows) {
#pragma unroll 1
        for (int s = 0; s + 1 < steps; ++s) {
            const int next = buf + 1 == NS ? 0 : buf + 1;
            tile_wait_const<NEWER>();
            lds_barrier();
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load_step(s + NS, i, buf);
            buf = next;
        }
    } else {
#pragma unroll 1
        for (int s = 0; s + 1 < steps; ++s) {
            const int next = buf + 1 == NS ? 0 : buf + 1;
            half(c0, yes, buf, no, 0, 0);          // multiplies half 0, reads half 1
            tile_wait_const<NEWER>();   // this wavefront's loads of step s + 1 have landed
            lds_barrier();                         // (waits for this wavefront's LDS reads first)
            half(c1, yes, next, yes, s + NS, buf); // multiplies half 1, reads half 0 of the next step
            buf = next;
        }
        // the last step, whose operands past the end are zeroed
        const auto cut = [&](auto cur_) {
            constexpr int cur = decltype(cur_)::value;
            if ((unsigned)(4 * cur + g) * 16 >= k_left) {
#pragma unroll
                for (int m = 0; m < TM; ++m) x[cur][m] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int n = 0; n < TN; ++n) w[cur][n] = u32x4{0, 0, 0, 0};
            }
        };
        cut(c0);
        half(c0, yes, buf, no, 0, 0);
        cut(c1);
        half(c1, no, 0, no, 0, 0);
    }
    tile_wait_const<0>();                      // (the repeated loads)

    // ---- epilogue: through LDS, a few row tiles at a time and each wavefront by itself.  Stores cover whole lines of a row, and the activation is one loop's
    // code instead of TN x TM copies of it.
    constexpr int PM = tile_epilogue_tiles(TM, TN, NW), PITCH = TN * 16 + 4, CV = TN * 4;      // CV: vectors of four columns in a row
    lds_barrier();                             // nobody reads operands any more
    float* const mine = (float*)lds + wave * (PM * 16 * PITCH);
#pragma unroll
    for (int m0 = 0; m0 < TM; m0 += PM) {
#pragma unroll
        for (int m = m0; m < m0 + PM; ++m)
#pragma unroll
            for (int n = 0; n < TN; ++n) *(f32x4*)(mine + ((m - m0) * 16 + q) * PITCH + n * 16 + 4 * g) = acc[n][m];
#pragma unroll 1
        for (int i = lane; i < PM * 16 * CV; i += 64) {
            const int lr = i / CV, c = i - lr * CV, r = (wm * TM + m0) * 16 + lr, col = n0 + wn * TN * 16 + 4 * c;
            const f32x4 s = *(const f32x4*)(mine + lr * PITCH + 4 * c);
            const float v[4] = {s[0], s[1], s[2], s[3]};
            if (r >= rows) break;              // (rows rise with i)
            if (a.splits > 1) {
                if (col < a.N) FP32::store4(a.partial, ((size_t)k_split * a.M + row0 + r) * a.pitch + col, v[0], v[1], v[2], v[3]);
            } else if (a.out_fp32) {
                linear_store4<E, FP32, false>(a, row0 + r, col, v);
            } else {
                linear_store4<E, E, false>(a, row0 + r, col, v);
            }
        }
    }
}

template <typename E, int BM, int BN, int WM, int WN, int NS, bool LINES = false>
hipError_t launch_tile(const TileArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr size_t stages = (size_t)NS * (BM + BN) * 128, end = (size_t)WM * WN * tile_epilogue_tiles(TM, TN, WM * WN) * 16 * (TN * 16 + 4) * 4;
    constexpr size_t lds = end > stages ? end : stages;
    static_assert(lds <= (size_t)kLdsLimit, "buffers fit LDS");
    if (hipError_t e = allow_lds(allowed, (const void*)k_tile<E, BM, BN, WM, WN, NS, LINES>, lds); e != hipSuccess) return e;
    const long long tiles = (long long)((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN) * a.splits;
    return launch_kernel(k_tile<E, BM, BN, WM, WN, NS, LINES>, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(WM * WN * 64), lds, st, a);
}

}  // namespace
}  // namespace dfk
