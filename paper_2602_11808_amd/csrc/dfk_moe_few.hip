// Experts with few tokens: two launches that stream the weights of the experts that are taken, once.
//
// k_moe_gateup_few: a workgroup owns 16 (or 8) rows of W_gate and the same of W_up of one entry's expert, finds the slots of that expert by itself
// (a list of up to 64 tokens' experts is a few loads), and leaves w * A_2 of its rows.  Entries are the slots where there are no more of
// them than experts (a slot whose expert an earlier one has does nothing), else the experts.
// k_moe_down_few: a workgroup owns 16 (or 8) columns of Y and all the experts, so nothing is summed across workgroups: its wavefronts take the taken experts
// in turn (or parts of their d_ff, where they are fewer), add each expert's rows to sums of their own per token in LDS, and those
// meet at the end.  The order of every sum is that of the entries: deterministic.
#include <algorithm>

#include "dfk_stream.h"

namespace dfk {
namespace {

// Rings of two chunks leave room for two to three workgroups of the gate/up kernel on a CU: what bounds it is workgroups waiting for their first
// tiles (16 tokens, 6 of 64 experts of 2048 x 1408: 135 us, three chunks deep 139, with eight wavefronts 163).
constexpr int kGateWaves = 4, kDownWaves = 8;

// The products of up to 16 TT rows (slots rows[0 .. count)) with 16 weight rows of gate and up, and their epilogue.
template <typename E, int TT, int XR, int D, int WR>
__device__ __forceinline__ void gateup_rows(const MoeFewArgs& a, unsigned char* lds, const int* rows, const float* row_weight, int count, int e, int j0) {
    constexpr int NW = kGateWaves;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned rb = (unsigned)a.d_model * 2;
    f32x4 acc[2][TT];
    const char* wb[2];
    unsigned wr[2][2], xr[XR / 8];
    const size_t first = ((size_t)e * a.d_ff + j0) * rb;
    wb[0] = (const char*)a.Wg + first;
    wb[1] = (const char*)a.Wu + first;
#pragma unroll
    for (int h = 0; h < 2; ++h) wr[0][h] = wr[1][h] = (unsigned)min(8 * h + (lane >> 3), a.d_ff - 1 - j0) * rb;
#pragma unroll
    for (int h = 0; h < XR / 8; ++h) xr[h] = (unsigned)(rows[min(8 * h + (lane >> 3), count - 1)] / a.top_k) * rb;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    stream_dot<E, NW, 2, TT, XR, D, 1, WR>(acc, lds, wave, wb, wr, (const char*)a.X, xr, a.d_model, wave, NW);
    f32x4* const sums = (f32x4*)lds;
    lds_barrier();
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int t = 0; t < TT; ++t) sums[((wave * 2 + n) * TT + t) * 64 + lane] = acc[n][t];
    __syncthreads();
    for (int i = tid; i < TT * 64; i += NW * 64) {
        f32x4 gt = sums[i], up = sums[TT * 64 + i];
#pragma unroll
        for (int w = 1; w < NW; ++w) { gt += sums[w * 2 * TT * 64 + i]; up += sums[(w * 2 + 1) * TT * 64 + i]; }
        const int m = (i >> 6) * 16 + (i & 15), col = j0 + 4 * ((i >> 4) & 3);
        if (m < count && ((i >> 4) & 3) < WR / 4 && col < a.d_ff) {
            const int slot = rows[m];
            const float w = row_weight[m];
            E::store4(a.a2, (size_t)slot * a.d_ff + col, w * silu_mul_fast(gt[0], up[0]), w * silu_mul_fast(gt[1], up[1]),
                      w * silu_mul_fast(gt[2], up[2]), w * silu_mul_fast(gt[3], up[3]));
        }
    }
    __syncthreads();
}

// R: most tokens of a launch: 8, 16 or 64 (how many rows the rings hold).  WR: rows of W_gate and of W_up, or of W_down_t, that a workgroup owns: 16, or 8 for up to 8 tokens.
template <typename E, int R, int WR>
__global__ __launch_bounds__(kGateWaves * 64) void k_moe_gateup_few(MoeFewArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    __shared__ int rows[kMoeFewTokens];
    __shared__ float row_weights[kGateWaves][kMoeFewTokens];      // (added to: a list for each wavefront)
    float* const row_weight = row_weights[__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)];
    const int lane = threadIdx.x & 63, y = (int)blockIdx.y, j0 = (int)blockIdx.x * WR;
    const int slots = a.M * a.top_k;
    int e = y;
    if (a.by_slot) {
        e = __builtin_amdgcn_readfirstlane(a.experts[y]);
        if ((unsigned)e >= (unsigned)a.n_experts) e = -1;
    }
    // The expert's slots in order; every wavefront finds them and writes the same list.  A token's slots are neighbours, so a slot whose predecessor among those of
    // this expert is of the same token repeats it: its weight is added to that one's.
    int count = 0, last = -1;                      // rows so far, the last slot of this expert
    bool later = false;
    if (e >= 0) {
        constexpr int B = 4;                       // loads of the list under way
        for (int s1 = 0; s1 < slots; s1 += 64 * B) {
            int have[B];
            float weight[B];
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int s = s1 + 64 * b + lane;
                have[b] = s < slots ? a.experts[s] : -1;
                weight[b] = s < slots ? a.weights[s] : 0.f;
            }
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int s0 = s1 + 64 * b, s = s0 + lane;
                const bool hit = have[b] == e;
                const unsigned long long hits = __ballot(hit), before = hits & ((1ull << lane) - 1ull);
                if (hits == 0) continue;
                const int prev = before ? s0 + 63 - __builtin_clzll(before) : last;
                const bool first = hit && (prev < 0 || prev / a.top_k != s / a.top_k);
                const unsigned long long firsts = __ballot(first);
                if (a.by_slot && last < 0 && s0 + (int)__builtin_ctzll(hits) < y) later = true;
                if (first) {
                    const int at = count + __builtin_popcountll(firsts & ((1ull << lane) - 1ull));
                    rows[at] = s;
                    row_weight[at] = weight[b];
                }
                unsigned long long again = hits & ~firsts;
                while (again) {                    // (rare; one after the other, in order)
                    const int l = __builtin_ctzll(again), at = count + __builtin_popcountll(firsts & ((1ull << l) - 1ull)) - 1;
                    if (lane == l) row_weight[at] += weight[b];
                    again &= again - 1;
                }
                count += __builtin_popcountll(firsts);
                last = s0 + 63 - (int)__builtin_clzll(hits);
            }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");       // (its own lanes' entries of the list)
    __builtin_amdgcn_wave_barrier();
    if (later) count = 0;                          // an earlier slot's entry has this expert
    if (y == 0 && a.down_groups > 1)               // arrival counters of the next launch
        for (int i = (int)(blockIdx.x * blockDim.x + threadIdx.x); i < (a.d_model + 15) / 16; i += (int)(gridDim.x * blockDim.x)) a.tickets[i] = 0;
    if (blockIdx.x == 0 && threadIdx.x < 64) {
        if (lane == 0) a.entry[y] = make_int2(e, count);
        if (lane < count) a.rows[(size_t)y * a.M + lane] = rows[lane];
    }
    if (count == 0) return;
    if (R == 8) {
        gateup_rows<E, 1, 8, WR == 8 ? 3 : 2, WR>(a, lds, rows, row_weight, count, e, j0);
    } else if (count <= 16) {
        gateup_rows<E, 1, 16, 2, 16>(a, lds, rows, row_weight, count, e, j0);
    } else {
        for (int r0 = 0; r0 < count; r0 += 32) gateup_rows<E, 2, 32, 1, 16>(a, lds, rows + r0, row_weight + r0, min(32, count - r0), e, j0);
    }
}

template <typename E, int R, int WR>
__global__ __launch_bounds__(kDownWaves * 64) void k_moe_down_few(MoeFewArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    // entries that have an expert: number, expert, slots
    __shared__ unsigned short taken[kMoeFewSlots], taken_expert[kMoeFewSlots];
    __shared__ unsigned char taken_count[kMoeFewSlots];
    __shared__ int last;
    constexpr int NW = kDownWaves, XR = R == 8 ? 8 : 16, D = WR == 8 ? 5 : 3;
    const int tid = threadIdx.x, lane = tid & 63, q = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = (int)blockIdx.x * WR;
    const unsigned rb = (unsigned)a.d_ff * 2;
    const int rings = NW * stream_ring_bytes<kDownWaves, 1, XR, D, WR>(a.d_ff);
    float* const sums = (float*)(lds + rings) + wave * a.M * 16;      // [token][column]
    for (int i = lane; i < a.M * 4; i += 64) *(f32x4*)(sums + 4 * i) = f32x4{0.f, 0.f, 0.f, 0.f};
    int n_taken = 0;
    constexpr int B = 4;
    for (int y1 = 0; y1 < a.entries; y1 += 64 * B) {
        int2 have[B];
#pragma unroll
        for (int b = 0; b < B; ++b) have[b] = y1 + 64 * b + lane < a.entries ? a.entry[y1 + 64 * b + lane] : make_int2(-1, 0);
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const unsigned long long mask = __ballot(have[b].y > 0);
            if (have[b].y > 0) {                   // (the same from every wavefront)
                const int at = n_taken + __builtin_popcountll(mask & ((1ull << lane) - 1ull));
                taken[at] = (unsigned short)(y1 + 64 * b + lane);
                taken_expert[at] = (unsigned short)have[b].x;
                taken_count[at] = (unsigned char)have[b].y;
            }
            n_taken += __builtin_popcountll(mask);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
    // The NW * groups wavefronts of these columns take the (expert, part of d_ff) pairs in turn, an expert's slots XR at a time.  The slots of the next are requested
    // before the products of this one: a pair's loads would otherwise start a trip to memory late.
    const int takers = NW * a.down_groups, parts = n_taken == 0 ? 1 : min((takers + n_taken - 1) / n_taken, (a.d_ff + kChunkK - 1) / kChunkK);
    struct Work { int u, r0, count, expert, part; };
    const auto at = [&](int u) {
        Work w{u, 0, 0, 0, 0};
        if (u < n_taken * parts) {
            const int i = u / parts;
            w.part = u - i * parts;
            w.expert = __builtin_amdgcn_readfirstlane((int)taken_expert[i]);
            w.count = __builtin_amdgcn_readfirstlane((int)taken_count[i]);
        }
        return w;
    };
    int row[XR / 8], mine;                         // slots of this lane's loads, and of its column
    const auto request = [&](const Work& w) {
        const int y = __builtin_amdgcn_readfirstlane((int)taken[w.u / parts]), c = min(XR, w.count - w.r0);
        if (a.M == 1 && a.by_slot) {               // the entry's one slot is itself: no trip to memory
#pragma unroll
            for (int h = 0; h < XR / 8; ++h) row[h] = y;
            mine = y;
            return;
        }
        const int* rows = a.rows + (size_t)y * a.M + w.r0;
#pragma unroll
        for (int h = 0; h < XR / 8; ++h) row[h] = rows[min(8 * h + (lane >> 3), c - 1)];
        mine = rows[min(q, c - 1)];
    };
    Work now = at((int)blockIdx.y * NW + wave);
    if (now.count > 0) request(now);
    while (now.count > 0) {
        const int c = min(XR, now.count - now.r0), slot = mine;
        const char* wb[1] = {(const char*)a.Wd + ((size_t)now.expert * a.d_model + n0) * rb};
        unsigned wr[1][2], xr[XR / 8];
#pragma unroll
        for (int h = 0; h < 2; ++h) wr[0][h] = (unsigned)min(8 * h + (lane >> 3), a.d_model - 1 - n0) * rb;
#pragma unroll
        for (int h = 0; h < XR / 8; ++h) xr[h] = (unsigned)row[h] * rb;
        Work next = now;
        next.r0 += XR;
        if (next.r0 >= now.count) next = at(now.u + takers);
        if (next.count > 0) request(next);
        f32x4 acc[1][1] = {{f32x4{0.f, 0.f, 0.f, 0.f}}};
        stream_dot<E, NW, 1, 1, XR, D, 1 + R, WR>(acc, lds, wave, wb, wr, (const char*)a.a2, xr, a.d_ff, now.part, parts);
        if (q < c && g < WR / 4) {
            f32x4* const s = (f32x4*)(sums + slot / a.top_k * 16 + 4 * g);
            *s = *s + acc[0][0];
        }
        now = next;
    }
    __syncthreads();
    const float* const own = (const float*)(lds + rings);
    const auto sum_of_waves = [&](int i) {
        f32x4 s = *(const f32x4*)(own + i * 4);
        for (int w = 1; w < NW; ++w) s += *(const f32x4*)(own + i * 4 + w * a.M * 16);
        return s;
    };
    if (a.down_groups == 1) {
        for (int i = tid; i < a.M * 4; i += NW * 64) {
            const int m = i >> 2, col = n0 + 4 * (i & 3);
            const f32x4 s = sum_of_waves(i);
            if ((i & 3) < WR / 4 && col < a.d_model) store4_plus<E>(a.Y, a.resid, (size_t)m * a.d_model + col, make_float4(s[0], s[1], s[2], s[3]));
        }
        return;
    }
    // Several workgroups share these columns: each publishes its sums, the last to arrive adds them up in order.
    const size_t blk = (size_t)a.M * a.d_model;
    for (int i = tid; i < a.M * 4; i += NW * 64) {
        const int m = i >> 2, col = n0 + 4 * (i & 3);
        const f32x4 s = sum_of_waves(i);
        if ((i & 3) < WR / 4 && col < a.d_model) store4_device(a.partial + blockIdx.y * blk + (size_t)m * a.d_model + col, s[0], s[1], s[2], s[3]);
    }
    drain_own_memory_ops();
    __syncthreads();
    if (tid == 0) last = arrive_last_acquire(a.tickets + blockIdx.x, (unsigned)a.down_groups);
    __syncthreads();
    if (!last) return;
    for (int i = tid; i < a.M * 4; i += NW * 64) {
        const int m = i >> 2, col = n0 + 4 * (i & 3);
        if ((i & 3) >= WR / 4 || col >= a.d_model) continue;
        const size_t at = (size_t)m * a.d_model + col;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int y = 0; y < a.down_groups; ++y) {
            const float4 v = *(const float4*)(a.partial + y * blk + at);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        store4_plus<E>(a.Y, a.resid, at, s);
    }
}

template <typename E, int R, int WR>
hipError_t launch_gate(const MoeFewArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    const size_t ring = (size_t)(WR == 8   ? stream_ring_bytes<kGateWaves, 2, 8, 3, 8>(a.d_model)
                                 : R == 8  ? stream_ring_bytes<kGateWaves, 2, 8, 2>(a.d_model)
                                 : R == 16 ? stream_ring_bytes<kGateWaves, 2, 16, 2>(a.d_model)
                                           : std::max(stream_ring_bytes<kGateWaves, 2, 16, 2>(a.d_model), stream_ring_bytes<kGateWaves, 2, 32, 1>(a.d_model)));
    static_assert(stream_ring_bytes<kGateWaves, 2, 8, 3, 8>(64) >= 2048 && stream_ring_bytes<kGateWaves, 2, 8, 2>(64) >= 2048 && stream_ring_bytes<kGateWaves, 2, 16, 2>(64) >= 4096, "the sums of gate and up take the rings' place");
    if (hipError_t e = allow_lds(allowed, (const void*)k_moe_gateup_few<E, R, WR>, kGateWaves * ring); e != hipSuccess) return e;
    return launch_kernel(k_moe_gateup_few<E, R, WR>, dim3((unsigned)(a.d_ff + WR - 1) / WR, (unsigned)a.entries), dim3(kGateWaves * 64), kGateWaves * ring, st, a);
}

template <typename E, int R, int WR>
hipError_t launch_down(const MoeFewArgs& a, hipStream_t st) {
    static LdsAllowance allowed;
    const size_t lds = kDownWaves * ((size_t)stream_ring_bytes<kDownWaves, 1, R == 8 ? 8 : 16, WR == 8 ? 5 : 3, WR>(a.d_ff) + (size_t)a.M * 64);
    if (hipError_t e = allow_lds(allowed, (const void*)k_moe_down_few<E, R, WR>, lds); e != hipSuccess) return e;
    return launch_kernel(k_moe_down_few<E, R, WR>, dim3((unsigned)(a.d_model + WR - 1) / WR, (unsigned)a.down_groups), dim3(kDownWaves * 64), lds, st, a);
}

template <typename E>
hipError_t launch_of(const MoeFewArgs& a, hipStream_t st) {
    // Up to 8 tokens tiles of 8 rows where 16 would make few workgroups: twice as many, and deeper rings.  Whole call, us, 16 / 8 rows: gate/up, 1 token, 1 of 16 experts of 4096 x 2048
    // (128 workgroups of 16 rows) 17.7 / 15.9, 8 of 128 of 2048 x 768 (384) 20.7 / 19.6, 2 tokens of these (768) 33.7 / 33.3, 8, 4 of 16 of 1024 x 1024 (1024) 24.4 / 25.1;
    // down, 1 token, 6 of 64 of 2048 x 1408 (128) 27.6 / 25.3, 2, 8 of 128 of 2048 x 768 (128) 33.7 / 30.7, 1, 4 of 60 of 2304 x 1408 (144) 20.9 / 23.8.
    const bool narrow_gate = a.M <= 8 && a.entries * ((a.d_ff + 15) / 16) < 1024, narrow_down = a.M <= 8 && a.down_groups == 1 && a.d_model <= 2048;
    hipError_t e = narrow_gate ? launch_gate<E, 8, 8>(a, st) : a.M <= 8 ? launch_gate<E, 8, 16>(a, st) : a.M <= 16 ? launch_gate<E, 16, 16>(a, st) : launch_gate<E, 64, 16>(a, st);
    if (e != hipSuccess) return e;
    return narrow_down ? launch_down<E, 8, 8>(a, st) : a.M <= 8 ? launch_down<E, 8, 16>(a, st) : a.M <= 16 ? launch_down<E, 16, 16>(a, st) : launch_down<E, 64, 16>(a, st);
}

}  // namespace

hipError_t launch_moe_few(const MoeFewArgs& a, dfk_dtype_t dtype, hipStream_t st) {
    if (a.M > kMoeFewTokens || a.M * a.top_k > kMoeFewSlots || a.entries > kMoeFewSlots) return hipErrorInvalidValue;
    return dtype == DFK_BF16 ? launch_of<BF16>(a, st) : launch_of<FP16>(a, st);
}

}  // namespace dfk
