// Mixture of experts: the rows of each expert gathered on the device, the launches of dfk_moe_mlp_wdt, its checks.
//
// A chunk of tokens is a list of slots t * top_k + j.  k_moe_count and k_moe_place sort the slots that take part by expert into rows and cut each expert's rows
// into row tiles (5 and 11 us of 4096 tokens with 8 of 64 experts; one launch, of 6 us at 1200 slots, up to 2048); the gate/up product gathers X by row and leaves w * A_2 in the row order;
// the down product's rows go to P[slot], and k_moe_sum adds a token's up in order of its slots (28 us, 6.2 TB/s; in half,
// whose rows are fp32, 52 us, 5.8 TB/s).  In 16 bits w * A_2 is rounded once: it is an operand of the matrix
// instructions.  The order of rows within an expert is
// that in which atomics placed them: it varies from run to run, but a row's sums do not depend on
// its place in a tile, so the results do not.
#include <algorithm>

#include "dfk_epilogue.h"
#include "dfk_moe_plan.h"

namespace dfk {
namespace {

// The plan's workgroups own whole tokens, of kPlanSlots slots or a few more.
// (us of the plan's launches with 512 threads and 1024 slots / 1024 and 2048: 1200 slots of 32 experts 9.3 / 5.9, 4096 of 64 12.8 / 13.7, 32768 of 256 19.3 / 16.7.)
constexpr int kPlanThreads = 1024, kPlanSlots = 2048;
constexpr int kPlanExperts = DFK_MAX_EXPERTS / kPlanThreads;      // of a thread

__host__ __device__ inline int plan_tokens(int top_k) { return (kPlanSlots + top_k - 1) / top_k; }

// The expert of slot j of a token's list, or -1 where it takes no part: out of range, or listed before.
__device__ __forceinline__ int taken_expert(const int* list, int j, int n_experts) {
    const int e = list[j];
    bool out = (unsigned)e >= (unsigned)n_experts;
#pragma unroll 4
    for (int i = 0; i < j; ++i) out |= list[i] == e;
    return out ? -1 : e;
}

// Sum over the workgroup's earlier threads, and over all.
__device__ __forceinline__ int scan_before(int v, int* part, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(s, o);
        if (lane >= o) s += t;
    }
    __syncthreads();
    if (lane == 63) part[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) before += part[w];
        all += part[w];
    }
    *total = all;
    return before + s - v;
}

// This workgroup's slots [first, first + n) into LDS, and how many of them each expert has.
__device__ __forceinline__ void plan_count(const int* experts, int first, int n, int top_k, int n_experts, int* list, int* count) {
    for (int e = threadIdx.x; e < n_experts; e += kPlanThreads) count[e] = 0;
    for (int i = threadIdx.x; i < n; i += kPlanThreads) list[i] = experts[first + i];
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int j = i % top_k, e = taken_expert(list + i - j, j, n_experts);
        if (e >= 0) atomicAdd(&count[e], 1);
    }
    __syncthreads();
}

__global__ __launch_bounds__(kPlanThreads) void k_moe_count(const int* experts, int tokens, int top_k, int n_experts, MoePlan p) {
    __shared__ int list[kPlanSlots + DFK_MAX_TOP_K];
    __shared__ int count[DFK_MAX_EXPERTS];
    const int per = plan_tokens(top_k), t0 = (int)blockIdx.x * per;
    plan_count(experts, t0 * top_k, min(per, tokens - t0) * top_k, top_k, n_experts, list, count);
    for (int e = threadIdx.x; e < n_experts; e += kPlanThreads) p.counts[(size_t)blockIdx.x * n_experts + e] = count[e];
}

// Every workgroup counts its own slots (again); where there are several, the others' counts are k_moe_count's.
__global__ __launch_bounds__(kPlanThreads) void k_moe_place(const int* experts, const float* weights, int tokens, int top_k, int n_experts, MoePlan p) {
    __shared__ int list[kPlanSlots + DFK_MAX_TOP_K];
    __shared__ int count[DFK_MAX_EXPERTS];
    __shared__ int sum_all[DFK_MAX_EXPERTS], sum_before[DFK_MAX_EXPERTS];
    __shared__ int part[kPlanThreads / 64];
    const int per = plan_tokens(top_k), t0 = (int)blockIdx.x * per, first = t0 * top_k, n = min(per, tokens - t0) * top_k;
    plan_count(experts, first, n, top_k, n_experts, list, count);
    // All workgroups' counts and those of the ones before: every thread adds its share of the table, which is read in one go.
    if (gridDim.x > 1) {
        for (int e = threadIdx.x; e < n_experts; e += kPlanThreads) sum_all[e] = sum_before[e] = 0;
        __syncthreads();
        const int size = (int)gridDim.x * n_experts;
#pragma unroll 8
        for (int i = threadIdx.x; i < size; i += kPlanThreads) {
            const int c = p.counts[i];
            if (c) {
                const int g = i / n_experts, e = i - g * n_experts;
                atomicAdd(&sum_all[e], c);
                if (g < (int)blockIdx.x) atomicAdd(&sum_before[e], c);
            }
        }
        __syncthreads();
    }
    // thread t: experts kPlanExperts t ..
    int all[kPlanExperts], before[kPlanExperts], rows = 0, tiles = 0;
#pragma unroll
    for (int k = 0; k < kPlanExperts; ++k) {
        const int e = (int)threadIdx.x * kPlanExperts + k;
        all[k] = e >= n_experts ? 0 : gridDim.x == 1 ? count[e] : sum_all[e];
        before[k] = e >= n_experts || gridDim.x == 1 ? 0 : sum_before[e];
        rows += all[k];
        tiles += (all[k] + p.tile_rows - 1) / p.tile_rows;
    }
    int total, n_tiles;
    int row0 = scan_before(rows, part, &total), tile0 = scan_before(tiles, part, &n_tiles);
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.n_tiles = n_tiles;
    if (blockIdx.x == 0 && threadIdx.x < 16) p.taken[threadIdx.x * kTakenPitch] = 0;
#pragma unroll
    for (int k = 0; k < kPlanExperts; ++k) {
        const int e = (int)threadIdx.x * kPlanExperts + k;
        if (e < n_experts) count[e] = row0 + before[k];      // from here on: where the expert's next row of this workgroup goes
        if (blockIdx.x == 0)
            for (int r = 0; r < all[k]; r += p.tile_rows) p.tiles[tile0++] = make_int4(e, row0 + r, min(p.tile_rows, all[k] - r), 0);
        row0 += all[k];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int j = i % top_k, e = taken_expert(list + i - j, j, n_experts);
        if (e < 0) continue;
        float w = weights[first + i];
        bool again = false;
#pragma unroll 4
        for (int k = j + 1; k < top_k; ++k) again |= list[i - j + k] == e;
        if (again)
            for (int k = j + 1; k < top_k; ++k)
                if (list[i - j + k] == e) w += weights[first + i - j + k];
        const int r = atomicAdd(&count[e], 1);
        p.slot[r] = first + i;
        p.weight[r] = w;
    }
}

// Y of a token: the residual and its slots' rows in order.  The rows of bf16 calls are halves times a power of two per 64 columns: 11 bits each, an eighth of the error of rounding
// Y, for half the traffic of fp32 rows, which is what this pass is made of (4096 tokens, 8 of 64 experts of 2048 x 1024, whole call 566 -> 534 us).  With half inputs that would be a third error
// of the size of those of w * A_2 and of Y (3.6e-4 for 3.0e-4 against 64 bits); their fp32 rows take this call from 521 to 568 us.
template <typename E>
__global__ __launch_bounds__(256) void k_moe_sum(const void* P, const float* scale, const int* experts, const void* resid, void* Y, int top_k, int n_experts, int d_model) {
    constexpr int C = kHalfRows<E> ? 8 : 4, B = 8;       // columns of a thread; slots whose loads are under way
    const int t = (int)blockIdx.y, n = ((int)blockIdx.x * 256 + (int)threadIdx.x) * C;
    if (n >= d_model) return;
    const int* list = experts + (size_t)t * top_k;
    const int blocks = (d_model + 63) / 64;
    float s[C];
#pragma unroll
    for (int c = 0; c < C; ++c) s[c] = 0.f;
    for (int j0 = 0; j0 < top_k; j0 += B) {
        u32x4 v[B];
        float f[B];
        bool take[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            take[b] = j0 + b < top_k && taken_expert(list, j0 + b, n_experts) >= 0;
            const size_t slot = (size_t)t * top_k + (take[b] ? j0 + b : 0);
            v[b] = *(const u32x4*)((const char*)P + (slot * d_model + n) * (C == 4 ? 4 : 2));
            f[b] = C == 4 ? 1.f : scale[slot * blocks + n / 64];
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (!take[b]) continue;
            float x[C];
            if constexpr (C == 4) FP32::widen(v[b], x); else FP16::widen(v[b], x);
#pragma unroll
            for (int c = 0; c < C; ++c) s[c] += f[b] * x[c];
        }
    }
#pragma unroll
    for (int c = 0; c < C; c += 4) store4_plus<E>(Y, resid, (size_t)t * d_model + n + c, make_float4(s[c], s[c + 1], s[c + 2], s[c + 3]));
}

// ---------------------------------------------------------------- host side
constexpr int kMaxSlots = 65536;     // of a chunk of tokens: offsets of rows stay below 4 GiB, and P within 64 KB x 65536 x 2

int moe_tile_rows(int M, int n_experts, int top_k, int d_model, int d_ff, dfk_dtype_t dtype) {
    return dtype == DFK_FP32 ? kTileRowsF32 : experts_tile_rows(M, n_experts, top_k, d_model, d_ff);
}
int chunk_tokens(int M, int top_k) { return std::min(M, std::min(kMaxSlots / top_k, 65535)); }

int plan_groups(int tokens, int top_k) { return (tokens + plan_tokens(top_k) - 1) / plan_tokens(top_k); }

struct MoeLayout { size_t n_tiles, taken, tiles, counts, slot, weight, entry, rows, tickets, a2, p, scale, total; int max_tiles, entries; };

struct Taker {
    size_t at = 0;
    size_t operator()(size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; }
};

MoeLayout moe_layout(int M, int n_experts, int top_k, int d_model, int d_ff, dfk_dtype_t dtype, int tile_rows) {
    const size_t slots = (size_t)chunk_tokens(M, top_k) * top_k;
    MoeLayout l{};
    l.max_tiles = experts_max_tiles((int)slots, n_experts, tile_rows);
    Taker take;
    l.n_tiles = take(4);
    l.taken = take(16 * kTakenPitch * 4);
    l.tiles = take((size_t)l.max_tiles * sizeof(int4));
    l.counts = take((size_t)plan_groups(chunk_tokens(M, top_k), top_k) * n_experts * 4);
    l.slot = take(slots * 4);
    l.weight = take(slots * 4);
    l.a2 = take(slots * d_ff * elt_bytes(dtype));
    l.p = take(slots * d_model * (dtype == DFK_BF16 ? 2 : 4));
    l.scale = take(dtype == DFK_BF16 ? slots * ((d_model + 63) / 64) * 4 : 0);
    l.total = take.at;
    return l;
}

// Few tokens: workgroups of the down projection that share 16 columns.  Several cost a meeting at the end, about 1 us, and pay where there are few columns
// and much to read for each: whole call, us, with 1 / 2 / 4: 1 token, 8 of 128 experts of 2048 x 768 (200 KB for 16 columns) 20.3 / 21.5 / 24.7, 4 tokens (700 KB)
// 55.7 / 52.6 / 56.1; 32 tokens, 4 of 16 of 1024 x 1024 (500 KB) 37.3 / 32.7 / 30.3; 24, 4 of 60 of 2304 x 1408 (2 MB) 142.7 / 146.0 / 139.0;
// 8, 4 of 16 of 4096 x 1024 59.3 / 64.6 / 71.0.
int moe_down_groups(int M, int n_experts, int top_k, int d_model, int d_ff) {
    const int columns = (d_model + 15) / 16;
    const size_t each = (size_t)std::min(M * top_k, n_experts) * d_ff * 32;
    return columns >= 256 || each < 400000 ? 1 : columns >= 128 && each < 1000000 ? 2 : 4;
}

MoeLayout moe_few_layout(int M, int n_experts, int top_k, int d_model, int d_ff) {
    const size_t slots = (size_t)M * top_k;
    MoeLayout l{};
    l.entries = (int)std::min<size_t>(slots, n_experts);
    Taker take;
    l.entry = take((size_t)l.entries * sizeof(int2));
    l.rows = take((size_t)l.entries * M * 4);
    l.tickets = take((size_t)(d_model + 15) / 16 * 4);
    l.a2 = take(slots * d_ff * 2);
    l.p = take((size_t)(d_model < 4096 ? 4 : 0) * M * d_model * 4);      // of up to four groups: no more for fewer tokens
    l.total = take.at;
    return l;
}

// The launches that stream the weights, up to 64 tokens: where experts have 8 rows at most on the average (16 rows to a weight tile then nearly always) and the lists
// are short.  Whole call, us, streaming / with tiles: 16 tokens, 2 of 4 experts of 4096 x 4096 (8 rows) 69.8 / 83.0, 32 tokens 84.2 / 84.7, 64 tokens 130.7 / 86.8;
// 64, 4 of 32 of 4096 x 1024 (256 slots) 136 / 155, 4 of 60 of 2304 x 1408 197 / 182, 8 of 128 of 2048 x 768 (512 slots) 227 / 192.
bool moe_few(int M, int n_experts, int top_k, dfk_dtype_t dtype) {
    return dtype != DFK_FP32 && M <= kMoeFewTokens && M * top_k <= 8 * n_experts && M * top_k <= kMoeFewSlots;
}

size_t moe_workspace(int M, int n_experts, int top_k, int d_model, int d_ff, dfk_dtype_t dtype) {
    // (64: the smallest row tiles make the longest list of them)
    return std::max(moe_layout(M, n_experts, top_k, d_model, d_ff, dtype, 64).total,
                    moe_few_layout(std::min(M, kMoeFewTokens), n_experts, top_k, d_model, d_ff).total);
}

bool moe_shape(int M, int n_experts, int top_k, int d_model, int d_ff) {
    return M >= 1 && M <= DFK_MAX_ROWS && n_experts >= 1 && n_experts <= DFK_MAX_EXPERTS && top_k >= 1 && top_k <= DFK_MAX_TOP_K &&
           d_model >= 8 && d_model <= kMaxDModel && d_model % 8 == 0 && d_ff >= 8 && d_ff <= kMaxDModel && d_ff % 8 == 0;
}

template <typename E>
hipError_t launch_moe_sum(const void* P, const float* scale, const int* experts, const void* resid, void* Y, int tokens, int top_k, int n_experts, int d_model, hipStream_t st) {
    return launch_kernel(k_moe_sum<E>, dim3((unsigned)((d_model * (kHalfRows<E> ? 2 : 4) + 4095) / 4096), (unsigned)tokens), dim3(256), 0, st, P, scale, experts, resid, Y, top_k, n_experts, d_model);
}

}  // namespace
}  // namespace dfk

using namespace dfk;

extern "C" {

dfk_status_t dfk_moe_mlp_wdt(const void* X, const int* experts, const float* weights,
                             const void* W_gate, const void* W_up, const void* W_down_t,
                             const void* residual, void* Y,
                             int M, int n_experts, int top_k, int d_model, int d_ff, dfk_dtype_t dtype,
                             void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !experts || !weights || !W_gate || !W_up || !W_down_t || !Y) return DFK_ERR_INVALID_ARG;
    if (M < 1 || n_experts < 1 || top_k < 1 || d_model < 1 || d_ff < 1 || !known_dtype(dtype)) return DFK_ERR_INVALID_ARG;
    if (!moe_shape(M, n_experts, top_k, d_model, d_ff)) return DFK_ERR_UNSUPPORTED_SHAPE;
    if ((uintptr_t)X % 16 || (uintptr_t)W_gate % 16 || (uintptr_t)W_up % 16 || (uintptr_t)W_down_t % 16 || (uintptr_t)residual % 16 ||
        (uintptr_t)Y % 16 || (uintptr_t)experts % 4 || (uintptr_t)weights % 4 || (uintptr_t)workspace % 256)
        return DFK_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < moe_workspace(M, n_experts, top_k, d_model, d_ff, dtype)) return DFK_ERR_WORKSPACE;
    const size_t es = elt_bytes(dtype), nx = (size_t)M * d_model * es, nw = (size_t)n_experts * d_ff * d_model * es, nk = (size_t)M * top_k * 4;
    const auto hits = [&](const void* p, size_t n) { return overlaps(Y, nx, p, n) || overlaps(workspace, workspace_bytes, p, n); };
    if (hits(X, nx) || hits(experts, nk) || hits(weights, nk) || hits(W_gate, nw) || hits(W_up, nw) || hits(W_down_t, nw) ||
        overlaps(workspace, workspace_bytes, Y, nx) || (residual && residual != Y && hits(residual, nx)))
        return DFK_ERR_ALIAS;

    const hipStream_t st = (hipStream_t)stream;
    unsigned char* const ws = (unsigned char*)workspace;
    if (moe_few(M, n_experts, top_k, dtype)) {
        const MoeLayout l = moe_few_layout(M, n_experts, top_k, d_model, d_ff);
        const MoeFewArgs f{X, experts, weights, W_gate, W_up, W_down_t, residual, Y, M, n_experts, top_k, d_model, d_ff,
                           M * top_k <= n_experts, l.entries, (int2*)(ws + l.entry), (int*)(ws + l.rows), ws + l.a2,
                           moe_down_groups(M, n_experts, top_k, d_model, d_ff), (unsigned*)(ws + l.tickets), (float*)(ws + l.p)};
        const hipError_t e = launch_moe_few(f, dtype, st);
        return e == hipSuccess ? DFK_OK : hip_fail(e);
    }
    const int tile_rows = moe_tile_rows(M, n_experts, top_k, d_model, d_ff, dtype);
    const MoeLayout l = moe_layout(M, n_experts, top_k, d_model, d_ff, dtype, tile_rows);
    TileArgs a{};
    a.top_k = top_k;
    a.scale = (float*)(ws + l.scale);
    // Start rotation and no place in the caches for the weights (dfk_tile.h): us without / with, 64 rows an expert (512 tokens, 8 of 64 of 2048 x 1024) 221 / 211, 38 (300, 4 of 32
    // of 4096 x 1024) 196 / 173, 19 (300, 8 of 128 of 2048 x 768) 251 / 236; 128 (1024 tokens, 8 of 64) 236 / 244.
    a.alone = 2ll * M * top_k <= (long long)tile_rows * n_experts;
    a.plan = MoePlan{(int*)(ws + l.n_tiles), (int4*)(ws + l.tiles), (int*)(ws + l.counts), (int*)(ws + l.slot), (float*)(ws + l.weight), (int*)(ws + l.taken), tile_rows, l.max_tiles};
    const int per = chunk_tokens(M, top_k);
    for (int m0 = 0; m0 < M; m0 += per) {
        const int n = std::min(per, M - m0);
        const int* ex = experts + (size_t)m0 * top_k;
        const float* wt = weights + (size_t)m0 * top_k;
        const unsigned groups = (unsigned)plan_groups(n, top_k);
        if (groups > 1)
            if (hipError_t e = launch_kernel(k_moe_count, dim3(groups), dim3(kPlanThreads), 0, st, ex, n, top_k, n_experts, a.plan); e != hipSuccess) return hip_fail(e);
        if (hipError_t e = launch_kernel(k_moe_place, dim3(groups), dim3(kPlanThreads), 0, st, ex, wt, n, top_k, n_experts, a.plan); e != hipSuccess) return hip_fail(e);
        a.A = (const char*)X + (size_t)m0 * d_model * es;
        a.B = W_gate; a.B2 = W_up; a.N = d_ff; a.K = d_model; a.out = ws + l.a2;
        if (hipError_t e = dtype == DFK_FP32 ? launch_experts_f32(a, kEpiGated, st) : launch_experts_tile(a, dtype, kEpiGated, st); e != hipSuccess) return hip_fail(e);
        a.A = ws + l.a2; a.B = W_down_t; a.B2 = nullptr; a.N = d_model; a.K = d_ff; a.out = ws + l.p;
        if (hipError_t e = dtype == DFK_FP32 ? launch_experts_f32(a, kEpiRows, st) : launch_experts_tile(a, dtype, kEpiRows, st); e != hipSuccess) return hip_fail(e);
        const size_t at = (size_t)m0 * d_model * es;
        const void* r = residual ? (const char*)residual + at : nullptr;
        void* y = (char*)Y + at;
        const void* P = ws + l.p;
        const float* f = (const float*)(ws + l.scale);
        const hipError_t e = dtype == DFK_FP32   ? launch_moe_sum<FP32>(P, f, ex, r, y, n, top_k, n_experts, d_model, st)
                             : dtype == DFK_BF16 ? launch_moe_sum<BF16>(P, f, ex, r, y, n, top_k, n_experts, d_model, st)
                                                 : launch_moe_sum<FP16>(P, f, ex, r, y, n, top_k, n_experts, d_model, st);
        if (e != hipSuccess) return hip_fail(e);
    }
    return DFK_OK;
}

size_t dfk_moe_workspace_bytes(int M_max, int n_experts, int top_k, int d_model, int d_ff, dfk_dtype_t dtype) {
    if (!known_dtype(dtype) || !moe_shape(M_max, n_experts, top_k, d_model, d_ff)) return 0;
    return moe_workspace(M_max, n_experts, top_k, d_model, d_ff, dtype);
}

}  // extern "C"
