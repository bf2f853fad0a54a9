// Experts with many rows: gate/up and down products on the matrix cores.
//
// The steps are k_tile's (dfk_tile.h): 64 k through LDS, NS deep, one barrier each.  What differs is what surrounds them.  A workgroup goes from tile to
// tile, and its results leave straight from the registers: of k_tile's way (a workgroup for each tile, which begins with four trips to memory,
// one after the other, for its tile, its rows, their slots and the first step, and ends with stores through LDS that nothing runs beside) the down product of 4096 tokens,
// 8 of 64 experts of 2048 x 1024, took 240 us and takes 204, the gated one 336 and 323.
//   The down product also loads the first steps of the next tile beside the last ones of this (204 us; 225 without).  The gated one does not: its 32 steps
// hide little, and dividing the slots by top_k amid a step cost more than it gave (333 us with, 322 without).
//   What bounds them: the gated one multiplies at 0.63 of the rate of an 8192^3 product, the other at 0.50 (313 and 198 us), counting the rows that there are; last tiles are partial, a
// step's loads have one step's time to arrive, from memory where weights pass once (0.54 and 0.27 GB), and the down product writes 0.13 GB of P.  The 256 x 256 tiles' registers are full:
// 11 to 20 values a lane are in scratch, and one that a tile's beginning reads back waits for the stores of the last tile's end and the loads ahead of it, as all share a counter.
#include "dfk_moe_plan.h"
#include "dfk_tile.h"

namespace dfk {
namespace {

// kEpiRows: values whose largest is `top` are kept as halves times 2^(e - 14).
__device__ __forceinline__ int half_exponent(float top) { return top > 0.f ? max((int)(__float_as_uint(top) >> 23) - 127, -100) : 14; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

template <typename E>
__device__ __forceinline__ void store8(void* p, size_t i, const float (&v)[8]) {       // i a multiple of 8
    *(u32x4*)((uint16_t*)p + i) = u32x4{E::pack2(v[0], v[1]), E::pack2(v[2], v[3]), E::pack2(v[4], v[5]), E::pack2(v[6], v[7])};
}

// Workgroups b, b + 8, ... share an eighth of the tiles in order and count to take the next one (experts' last tiles are partial and take less time; which workgroup
// computes a tile changes nothing in it).  With `ahead` that happens some steps before it is needed, in four parts, each of which finds behind its barrier what the
// one before has asked for (dfk_moe_plan.h).
//
// Rows of B lie in LDS so that tiles 2p and 2p + 1 of a wavefront hold columns 32 p + 8 g + (0..3, 4..7) in the four rows of lane group g: a lane ends up with eight
// adjacent columns, 16 bytes.  Of the gated form the first half of a wavefront's tiles is gate, the other the same columns of up.
//
// LINES, for K off the multiples of 64, whose rows start anywhere in a cache line: a step brings in each row's own next line (one more than it has steps) instead of 64 k that
// straddle two, most of which would be asked for twice; an operand's 16-byte piece is found by its row's offset in this step's buffer or the next one's.  A step's lines have to
// be there one step sooner, so that this takes four buffers, and with them tiles of 128 x 128.  Whole call, us, straddling (128 x 256) / by lines: 300 tokens, 4 of 32 experts of 2888 x 1000
// 158 / 129, 600 tokens 215 / 171, 500, 2 of 8 of 3000 x 3000 213 / 157.
template <typename E, int EPI, int BM, int BN, int WM, int WN, int NS, int PER_CU, bool LINES>
__global__ __launch_bounds__(WM * WN * 64) void k_experts(TileArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int STAGE = (BM + BN) * 128, B_OFF = BM * 128;
    constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, LOADS = LA + LB;
    constexpr int CT = EPI == kEpiGated ? TN / 2 : TN, NCOLS = EPI == kEpiGated ? BN / 2 : BN;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM % 64 == 0 && BM / 64 <= NW && CT % (EPI == kEpiRows ? 4 : 2) == 0 && NW % 2 == 0, "whole loads, pairs of tiles, blocks of 64 columns");
    int* const next_slots = (int*)(lds + NS * STAGE);          // of the next tile's rows
    int4* const next_tile = (int4*)(next_slots + BM);          // its expert and rows, and
    int* const next_index = (int*)(next_tile + 1);             // its place in the order
    const int tid = threadIdx.x, lane = tid & 63, q = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int n_tiles = (a.N + NCOLS - 1) / NCOLS, m_tiles = *a.plan.n_tiles;
    const int total = m_tiles * n_tiles, per = (total + 7) / 8, part = (int)blockIdx.x & 7;
    const int begin = part * per, end = min(total, begin + per), index = begin + ((int)blockIdx.x >> 3);
    if (index >= end) return;
    constexpr int NEWER = LOADS * experts_newer_steps(NS, LINES);     // loads that may be under way when the next step's have to be there
    static_assert(NEWER >= 0, "depth");
    static_assert(LINES || NEWER <= LOADS * experts_look_gap(NS), "the next tile's words are older than the loads that may be under way when they are read");
    const int steps = (a.K + kTileStepK - 1) / kTileStepK;
    const bool ahead = EPI == kEpiRows && !LINES && steps >= experts_look_steps(NS);     // else a tile begins when the one before has ended
    const unsigned rb = (unsigned)a.K * 2, k_left = rb - (unsigned)(steps - 1) * (kTileStepK * 2);
    const auto piece_of = [&](int l) { return (unsigned)((((l & 7) ^ (l >> 4)) & 7) * 16) ^ ((wave & 1) ? 64u : 0u); };
    const unsigned tail_off = piece_of(lane) + 16 > k_left ? piece_of(lane) + 16 - k_left : 0u;

    // (For what is needed once a tile: values of the lane made anew, or the compiler keeps them all and pushes the steps' own out of the registers.)
    const auto new_lane = [&]() {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };

    struct Tile { int group, row0, rows, nt; };
    const auto tile_of_words = [&](int4 t, int nt) {
        return Tile{__builtin_amdgcn_readfirstlane(t.x), __builtin_amdgcn_readfirstlane(t.y), __builtin_amdgcn_readfirstlane(t.z), nt};
    };
    const auto request_slots = [&](const Tile& t) {            // rows past the end: the last one's
        if (EPI == kEpiGated && wave < BM / 64)
            __builtin_amdgcn_global_load_lds(a.plan.slot + (size_t)t.row0 + min(wave * 64 + new_lane(), t.rows - 1), DFK_LDS_PTR(next_slots + wave * 64), 4, 0, 0);
    };
    const char *base_a, *base_b, *base_u = nullptr;
    unsigned off_a[LA], off_b[LB];
    int at_a[LINES ? LA : 1], at_b[LINES ? LB : 1];            // LINES: place of a load's piece in its row, less what the row is off its line
    int o_off[2][LINES ? TM + 4 : 1];                          // and of this lane's operands: place in LDS, and whether in the next step's buffer
    bool o_next[2][LINES ? TM + 4 : 1];
    // once, rot: as in k_tile.  256 rows are chosen where experts have 200 and more, whose weights several workgroups read.
    const bool alone = BM < 256 && a.alone, once = alone && (a.K % kTileStepK == 0 || LINES);
    const int whole = a.K / kTileStepK;
    int rot = 0;
    int ls = 0;                                                // step that is loaded next
    const auto begin_loads = [&](const Tile& t) {
        const int l = new_lane(), prow = l >> 3;
        const unsigned kb = piece_of(l);
        unsigned top_k = (unsigned)a.top_k;
        asm volatile("" : "+s"(top_k));
        rot = alone && whole > 0 ? (int)((unsigned)t.nt % (unsigned)whole) : 0;
        const int n0 = t.nt * NCOLS, n_last = a.N - n0 - 1;
        const size_t b0 = ((size_t)t.group * a.N + n0) * rb;
        base_a = (const char*)a.A + (EPI == kEpiGated ? 0 : (size_t)t.row0 * rb);
        base_b = (const char*)a.B + b0;
        if (EPI == kEpiGated) base_u = (const char*)a.B2 + b0;
#pragma unroll
        for (int i = 0; i < LA; ++i) {
            const int r = 8 * (wave + NW * i) + prow;
            // (at most 65536 tokens of 64 KB, below 4 GiB)
            off_a[i] = __umul24(EPI == kEpiGated ? (unsigned)next_slots[r] / top_k : (unsigned)min(r, t.rows - 1), rb) + (LINES ? 0u : kb);
            if constexpr (LINES) at_a[i] = (int)kb - ((int)((uintptr_t)base_a + off_a[i]) & 127);
            asm("" : "+v"(off_a[i]));
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            const int r = 8 * (wave + NW * i) + prow, w = (r >> 4) / TN, f = (r >> 4) % TN % CT;
            const int col = (w * CT + (f & ~1)) * 16 + 8 * ((r & 15) >> 2) + 4 * (f & 1) + (r & 3);
            off_b[i] = __umul24((unsigned)min(col, n_last), rb) + (LINES ? 0u : kb);
            if constexpr (LINES) at_b[i] = (int)kb - ((int)((uintptr_t)(EPI == kEpiGated && (r >> 4) % TN >= CT ? base_u : base_b) + off_b[i]) & 127);
            asm("" : "+v"(off_b[i]));
        }
        if constexpr (LINES) {
            const int q = l & 15, g = l >> 4;
            const auto place = [&](int i, const char* row) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int p = 4 * j + g + (int)((uintptr_t)row & 127) / 16;
                    o_off[j][i] = q * 128 + ((p ^ (q >> 1)) & 7) * 16;
                    o_next[j][i] = p >= 8;
                }
            };
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const int r = (wm * TM + m) * 16 + q;
                place(m, base_a + __umul24(EPI == kEpiGated ? (unsigned)next_slots[r] / top_k : (unsigned)min(r, t.rows - 1), rb));
            }
            // (32 rows of B are a multiple of 128 bytes: tiles differ by the four rows of every second one, and by gate's and up's base)
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                const unsigned row = __umul24((unsigned)(8 * (q >> 2) + 4 * f + (q & 3)), rb);
                place(TM + f, base_b + row);
                if (EPI == kEpiGated) place(TM + 2 + f, base_u + row);
            }
        }
        ls = 0;
    };
    const auto load = [&](int i, int buf) {
        unsigned o = i < LA ? off_a[i] : off_b[i - LA];
        size_t k = 0;
        if constexpr (LINES) {                                 // lines 0 .. steps of a row; pieces outside it are its first or last one
            o += (unsigned)min(max(min(ls, steps) * (kTileStepK * 2) + (i < LA ? at_a[i] : at_b[i - LA]), 0), (int)rb - 16);
            asm("" : "+v"(o));
        } else {
            const int t = min(ls, steps - 1);                  // a step past the last one is the last one again
            int tr = t;
            if (BM < 256 && t < whole) tr = t + rot >= whole ? t + rot - whole : t + rot;
            k = (size_t)tr * (kTileStepK * 2);
            asm("" : "+v"(o));
            o -= t == steps - 1 ? tail_off : 0u;
        }
        const int j = NW * (i < LA ? i : i - LA);
        const char* p = i < LA ? base_a : EPI == kEpiGated && ((wave + j) >> 1) % TN >= CT ? base_u : base_b;
        unsigned char* const dst = lds + buf * STAGE + wave * 1024 + j * 1024;
        if (i >= LA && once) __builtin_amdgcn_global_load_lds(p + k + o, DFK_LDS_PTR(dst + B_OFF), 16, 0, kAuxNonTemporal);
        else __builtin_amdgcn_global_load_lds(p + k + o, DFK_LDS_PTR(dst + (i < LA ? 0 : B_OFF)), 16, 0, 0);
    };

    int mt, nt;
    tile_at(index, m_tiles, n_tiles, mt, nt);
    Tile cur = tile_of_words(a.plan.tiles[mt], nt), nxt = cur;
    int ticket = 0;
    bool more = false;
    const auto look_ahead = [&](int stage) {
        if (stage == 0) {
            if (tid == 0) ticket = atomicAdd(a.plan.taken + (EPI == kEpiGated ? 0 : 8 * kTakenPitch) + part * kTakenPitch, 1);
        } else if (stage == 1) {
            if (tid == 0) {
                const int idx = begin + ((int)gridDim.x >> 3) + ticket;
                *next_index = idx;
                if (idx < end) {
                    int m, n;
                    tile_at(idx, m_tiles, n_tiles, m, n);
                    __builtin_amdgcn_global_load_lds(a.plan.tiles + m, DFK_LDS_PTR(next_tile), 16, 0, 0);
                }
            }
        } else if (stage == 2) {
            const int idx = __builtin_amdgcn_readfirstlane(*next_index);
            more = idx < end;
            if (more) {
                int m, n;
                tile_at(idx, m_tiles, n_tiles, m, n);
                nxt = tile_of_words(*next_tile, n);
                request_slots(nxt);
            }
        } else if (more) {
            begin_loads(nxt);
        }
    };

    constexpr auto c0 = std::integral_constant<int, 0>{};
    constexpr auto c1 = std::integral_constant<int, 1>{};
    constexpr auto yes = std::true_type{};
    constexpr auto no = std::false_type{};

    request_slots(cur);
    bool filled = false;
    int buf = 0;
#pragma unroll 1
    for (;;) {
        if (!filled) {
            tile_wait_const<0>();
            lds_barrier();
            begin_loads(cur);
#pragma unroll 1
            for (int s = 0; s < NS; ++s) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) load(i, s);
                ++ls;
            }
            tile_wait_const<LOADS * (NS - (LINES ? 2 : 1))>();
            lds_barrier();
            buf = 0;
        }
        f32x4 acc[TN][TM];
        u32x4 x[2][TM], w[2][TN];
        const int lo = q * 128 + ((g ^ (q >> 1)) & 7) * 16;
        const int a_tile = wm * TM * kTile16, b_tile = B_OFF + wn * TN * kTile16;
        const auto o_a = [](int m) { return LINES ? m : 0; };
        const auto o_b = [](int n) { return LINES ? TM + (n & 1) + (EPI == kEpiGated && n >= CT ? 2 : 0) : 0; };
        // as in k_tile
        const auto half = [&](auto cur_, auto read_, int buf, auto load_, int lbuf) {
            constexpr int now = decltype(cur_)::value, nxt = now ^ 1, H = nxt;
            constexpr bool READ = decltype(read_)::value, LOAD = decltype(load_)::value;
            int at = lo;
            asm volatile("" : "+v"(at));                   // (one register for both halves of both operands)
            at ^= 64 * H;
            const unsigned char* as = lds + buf * STAGE + a_tile + (LINES ? 0 : at);
            const unsigned char* bs = lds + buf * STAGE + b_tile + (LINES ? 0 : at);
            const int on = buf + 1 == NS ? -(NS - 1) * STAGE : STAGE;
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                if (READ) {
#pragma unroll
                    for (int m = n * TM / TN; m < (n + 1) * TM / TN; ++m) x[nxt][m] = *(const u32x4*)(as + m * kTile16 + (LINES ? o_off[H][o_a(m)] + (o_next[H][o_a(m)] ? on : 0) : 0));
                    w[nxt][n] = *(const u32x4*)(bs + n * kTile16 + (LINES ? o_off[H][o_b(n)] + (o_next[H][o_b(n)] ? on : 0) : 0));
                }
                if (LOAD) {
#pragma unroll
                    for (int i = n * LOADS / TN; i < (n + 1) * LOADS / TN; ++i) load(i, lbuf);
                }
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int m = 0; m < TM; ++m) acc[n][m] = mfma16<E>(w[now][n], x[now][m], acc[n][m]);
                __builtin_amdgcn_s_setprio(0);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        const auto cut = [&](auto cur_) {                          // operands past the end of the last step
            constexpr int now = decltype(cur_)::value;
            if ((unsigned)(4 * now + g) * 16 >= k_left) {
#pragma unroll
                for (int m = 0; m < TM; ++m) x[now][m] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int n = 0; n < TN; ++n) w[now][n] = u32x4{0, 0, 0, 0};
            }
        };
        const bool idle = wm * TM * 16 >= cur.rows;            // rows past the end alone: this wavefront only loads
        const auto look = [&](int s) {
            if (ahead)
                if (const int part = experts_look_part(s, steps, NS); part >= 0) look_ahead(part);
        };
        int row_value[TM];                                     // weights (fp32) or slots of lane q's rows
        if (idle) {
#pragma unroll 1
            for (int s = 0; s < steps; ++s) {
                tile_wait_const<NEWER>();
                lds_barrier();
                look(s);
#pragma unroll
                for (int i = 0; i < LOADS; ++i) load(i, buf);
                ++ls;
                buf = buf + 1 == NS ? 0 : buf + 1;
            }
        } else {
#pragma unroll
            for (int n = 0; n < TN; ++n)
#pragma unroll
                for (int m = 0; m < TM; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < TM; ++m) x[0][m] = *(const u32x4*)(lds + buf * STAGE + a_tile + m * kTile16 + (LINES ? o_off[0][o_a(m)] + (o_next[0][o_a(m)] ? STAGE : 0) : lo));
#pragma unroll
            for (int n = 0; n < TN; ++n) w[0][n] = *(const u32x4*)(lds + buf * STAGE + b_tile + n * kTile16 + (LINES ? o_off[0][o_b(n)] + (o_next[0][o_b(n)] ? STAGE : 0) : lo));
#pragma unroll 1
            for (int s = 0; s + 1 < steps; ++s) {
                const int next = buf + 1 == NS ? 0 : buf + 1;
                half(c0, yes, buf, no, 0);
                tile_wait_const<NEWER>();
                lds_barrier();
                look(s);
                half(c1, yes, next, yes, buf);
                ++ls;
                buf = next;
            }
            cut(c0);
            half(c0, yes, buf, no, 0);
            tile_wait_const<NEWER>();
            lds_barrier();
            const int q = new_lane() & 15;
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const size_t r = (size_t)cur.row0 + min((wm * TM + m) * 16 + q, cur.rows - 1);
                row_value[m] = EPI == kEpiGated ? __float_as_int(a.plan.weight[r]) : a.plan.slot[r];
            }
            cut(c1);
            half(c1, no, 0, yes, buf);
            ++ls;
            buf = buf + 1 == NS ? 0 : buf + 1;
        }
        if (!idle) {
            const int n0 = cur.nt * NCOLS + wn * CT * 16, l = new_lane(), q = l & 15, g = l >> 4;
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                const int r = (wm * TM + m) * 16 + q;
                if constexpr (EPI == kEpiGated) {
#pragma unroll
                    for (int p = 0; p < CT; p += 2) {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = __int_as_float(row_value[m]) * silu_mul_fast(acc[p + i / 4][m][i & 3], acc[CT + p + i / 4][m][i & 3]);
                        const int col = n0 + p * 16 + 8 * g;
                        if (r < cur.rows && col < a.N) store8<E>(a.out, ((size_t)cur.row0 + r) * a.N + col, v);
                    }
                } else {
                    const size_t slot = (size_t)row_value[m];
                    if constexpr (!kHalfRows<E>) {             // (halves again would be as much error as the operands' rounding)
#pragma unroll
                        for (int p = 0; p < CT; ++p) {
                            const int col = n0 + (p & ~1) * 16 + 8 * g + 4 * (p & 1);
                            if (r < cur.rows && col < a.N) FP32::store4(a.out, slot * a.N + col, acc[p][m][0], acc[p][m][1], acc[p][m][2], acc[p][m][3]);
                        }
                    } else {
                    // 64 columns of a row share a power of two that brings the largest (finite) one to 2^14.
#pragma unroll
                    for (int b = 0; b < CT; b += 4) {
                        float top = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float v = fabsf(acc[b + i / 4][m][i & 3]);
                            top = fmaxf(top, v < INFINITY && (!LINES || n0 + (b + i / 4 / 2 * 2) * 16 + 8 * g < a.N) ? v : 0.f);     // (LINES: columns that there are)
                        }
                        top = fmaxf(top, __shfl_xor(top, 16));
                        top = fmaxf(top, __shfl_xor(top, 32));
                        const int e = half_exponent(top);
                        const float up = power_of_two(14 - e);
#pragma unroll
                        for (int p = b; p < b + 4; p += 2) {
                            float v[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = up * acc[p + i / 4][m][i & 3];
                            const int col = n0 + p * 16 + 8 * g;
                            if (r < cur.rows && col < a.N) store8<FP16>(a.out, slot * a.N + col, v);
                        }
                        const int col = n0 + b * 16;
                        if (g == 0 && r < cur.rows && col < a.N) a.scale[slot * ((a.N + 63) / 64) + col / 64] = power_of_two(e - 14);
                    }
                    }
                }
            }
        }
        if (!ahead) {
            look_ahead(0);
            look_ahead(1);
            tile_wait_const<0>();
            lds_barrier();                                     // (nobody reads operands any more)
            look_ahead(2);
        }
        if (!more) break;
        cur = nxt;
        filled = ahead;
    }
    tile_wait_const<0>();                                      // (the repeated loads)
}

template <typename E, int EPI, int BM, int BN, int WM, int WN, int NS, int PER_CU, bool LINES = false>
hipError_t launch_experts(const TileArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    constexpr size_t lds = (size_t)NS * (BM + BN) * 128 + BM * 4 + 32;
    static_assert(lds <= (size_t)kLdsLimit, "buffers fit LDS");
    if (hipError_t e = allow_lds(allowed, (const void*)k_experts<E, EPI, BM, BN, WM, WN, NS, PER_CU, LINES>, lds); e != hipSuccess) return e;
    return launch_kernel(k_experts<E, EPI, BM, BN, WM, WN, NS, PER_CU, LINES>, dim3(experts_grid(ExpertsForm{BM, BN, NS, PER_CU, LINES}, a.plan.max_tiles, a.N, EPI == kEpiGated)),
                         dim3(WM * WN * 64), lds, st, a);
}

template <typename E, int EPI>
hipError_t launch_of(const TileArgs& a, hipStream_t st) {
    const auto launch = [&](auto form_, auto wm_, auto wn_) {
        constexpr ExpertsForm F = kExpertsForms[decltype(form_)::value];
        return launch_experts<E, EPI, F.bm, F.bn, decltype(wm_)::value, decltype(wn_)::value, F.ns, F.per_cu, F.lines>(a, st);
    };
    constexpr auto two = std::integral_constant<int, 2>{};
    constexpr auto four = std::integral_constant<int, 4>{};
    switch (experts_form(a.plan.tile_rows, a.plan.max_tiles, a.N, a.K, EPI == kEpiGated)) {
        case 0: return launch(std::integral_constant<int, 0>{}, two, two);
        case 1: return launch(std::integral_constant<int, 1>{}, four, two);
        case 2: return launch(std::integral_constant<int, 2>{}, four, two);
        case 3: return launch(std::integral_constant<int, 3>{}, two, four);
        case 4: return launch(std::integral_constant<int, 4>{}, four, two);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_experts_tile(const TileArgs& a, dfk_dtype_t dtype, int epi, hipStream_t st) {
    if (epi == kEpiGated) return dtype == DFK_BF16 ? launch_of<BF16, kEpiGated>(a, st) : launch_of<FP16, kEpiGated>(a, st);
    return dtype == DFK_BF16 ? launch_of<BF16, kEpiRows>(a, st) : launch_of<FP16, kEpiRows>(a, st);
}

}  // namespace dfk
