// Choice of experts: scores, groups, top-k and weights of dfk_moe_route, its checks.
//
// A token is handled by L lanes of one wavefront (16, four tokens beside each other, 32 or all 64) that hold V of its experts each,
// expert v L + l in value v of lane l.  What is compared is one double per expert that no other expert of the token has: the selection score's
// upper 54 bits with the expert's index in place of the lower 10, turned so that of equal scores the lower index is the larger number.
// The maximum of those is one instruction whatever is compared, where a pair of score and index takes a compare and three selects, and
// the next pick is the maximum of what is below the last one.
// Where the order of the scores is that of the logits (no bias, and no sums of scores for groups) the logit takes the
// score's place and no exponential is needed to choose: that is the form BY_LOGIT, whose weights are computed in fp32.  The other one computes
// all scores in 64 bits: two scores that differ by less than 2^-42 of themselves count as equal.
#include <cmath>

#include "dfk_device.h"
#include "dfk_ops.h"

namespace dfk {
namespace {

struct RouteArgs {
    const void* logits;
    const float* bias;
    int* experts;
    float* weights;
    int M, E, K, dtype, sigmoid;
    int n_groups, group_size, top_groups, group_top;
    int renormalise;
    float scale;
};

constexpr int kTagBits = 10;
static_assert(DFK_MAX_EXPERTS <= 1 << kTagBits, "an expert's index in the lower bits");
constexpr unsigned kTagMask = (1u << kTagBits) - 1u;

// ---- across the L lanes of a token: every lane gets the result ----
template <int CTRL>
__device__ __forceinline__ unsigned dpp(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(v);
    return __longlong_as_double((long long)(((unsigned long long)dpp<CTRL>((unsigned)(u >> 32)) << 32) | dpp<CTRL>((unsigned)u)));
}
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __uint_as_float(dpp<CTRL>(__float_as_uint(v))); }

// The two values whose combination is the next step's: rows of 16 lanes (ROW) or halves (not ROW) exchanged.
template <bool ROW>
__device__ __forceinline__ void swapped(unsigned v, unsigned& a, unsigned& b) {
    const auto r = ROW ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
    a = r[0]; b = r[1];
}
template <bool ROW>
__device__ __forceinline__ void swapped(float v, float& a, float& b) {
    unsigned x, y;
    swapped<ROW>(__float_as_uint(v), x, y);
    a = __uint_as_float(x); b = __uint_as_float(y);
}
template <bool ROW>
__device__ __forceinline__ void swapped(double v, double& a, double& b) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(v);
    unsigned al, bl, ah, bh;
    swapped<ROW>((unsigned)u, al, bl);
    swapped<ROW>((unsigned)(u >> 32), ah, bh);
    a = __longlong_as_double((long long)(((unsigned long long)ah << 32) | al));
    b = __longlong_as_double((long long)(((unsigned long long)bh << 32) | bl));
}
template <int L, typename T, typename F>
__device__ __forceinline__ T across(T v, F f) {
    v = f(v, dpp<0x128>(v));     // rotations within a row of 16 lanes, by 8, 4, 2, 1
    v = f(v, dpp<0x124>(v));
    v = f(v, dpp<0x122>(v));
    v = f(v, dpp<0x121>(v));
    T a, b;
    if (L >= 32) {
        swapped<true>(v, a, b);
        v = f(a, b);
    }
    if (L == 64) {
        swapped<false>(v, a, b);
        v = f(a, b);
    }
    return v;
}
template <int L> __device__ __forceinline__ double max_across(double v) { return across<L>(v, [](double a, double b) { return __builtin_fmax(a, b); }); }
template <int L> __device__ __forceinline__ float max_across(float v) { return across<L>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int L> __device__ __forceinline__ unsigned or_across(unsigned v) { return across<L>(v, [](unsigned a, unsigned b) { return a | b; }); }
template <int L, typename T> __device__ __forceinline__ T sum_across(T v) { return across<L>(v, [](T a, T b) { return a + b; }); }

// exp(x) to about 2 units in the last place, -745 <= x <= 709: 2^n exp(r) with |r| <= ln(2)/2 and the series of exp up to r^12
// (the next term is below 2^-52).
__device__ __forceinline__ double exp64(double x) {
    const double n = __builtin_rint(x * 1.4426950408889634);
    double r = __builtin_fma(n, -0.69314718036912382, x);        // ln 2 in two parts, the first with 32 bits
    r = __builtin_fma(n, -1.9082149292705877e-10, r);
    double p = 1.0 / 479001600.0;
    p = __builtin_fma(p, r, 1.0 / 39916800.0);
    p = __builtin_fma(p, r, 1.0 / 3628800.0);
    p = __builtin_fma(p, r, 1.0 / 362880.0);
    p = __builtin_fma(p, r, 1.0 / 40320.0);
    p = __builtin_fma(p, r, 1.0 / 5040.0);
    p = __builtin_fma(p, r, 1.0 / 720.0);
    p = __builtin_fma(p, r, 1.0 / 120.0);
    p = __builtin_fma(p, r, 1.0 / 24.0);
    p = __builtin_fma(p, r, 1.0 / 6.0);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_ldexp(p, (int)n);
}
// 1 / d for 1 <= d: the hardware's start and two steps of Newton's method.  Infinity gives 0.
__device__ __forceinline__ double recip64(double d) {
    double y = __builtin_amdgcn_rcp(d);
    if (d > 1e300) return y;
    y = __builtin_fma(__builtin_fma(-d, y, 1.0), y, y);
    return __builtin_fma(__builtin_fma(-d, y, 1.0), y, y);
}
__device__ __forceinline__ double sigmoid64(double x) {
    // (below -708 the exponential overflows; those scores are below 1e-307.  Above 40 the 1 is all there is; infinity has no exp64.)
    return x < -708.0 ? 0.0 : recip64(1.0 + exp64(__builtin_fmax(-x, -40.0)));
}

// A score and its index as one number; -infinity and NaN become -infinity, +infinity the largest number, -0 becomes 0.
__device__ __forceinline__ double tagged(double score, unsigned index) {
    const double s = __builtin_fmin(score, 1.7976931348623157e308) + 0.0;
    const unsigned long long u = (unsigned long long)__double_as_longlong(s);
    const unsigned hi = (unsigned)(u >> 32), tag = (kTagMask - index) ^ ((unsigned)((int)hi >> 31) & kTagMask);   // (kTagMask - index is its complement)
    const unsigned long long v = ((unsigned long long)hi << 32) | ((unsigned)u & ~kTagMask) | tag;
    return score > -HUGE_VAL ? __longlong_as_double((long long)v) : -HUGE_VAL;
}
__device__ __forceinline__ unsigned index_of(double key) {
    const long long u = __double_as_longlong(key);
    const unsigned tag = (unsigned)u & kTagMask;
    return u < 0 ? tag : kTagMask - tag;
}

// key where it is below `last`, else a number that is no key (none is below kNone, logits and biases being fp32): only the upper word is selected.
constexpr double kNone = -1e308;
__device__ __forceinline__ double below(double key, double last) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(key);
    const unsigned hi = key < last ? (unsigned)(u >> 32) : 0xFFEFFFFFu;
    return __longlong_as_double((long long)(((unsigned long long)hi << 32) | (unsigned)u));
}

__device__ __forceinline__ float logit_at(const RouteArgs& a, size_t i) {
    return a.dtype == DFK_FP32 ? ((const float*)a.logits)[i] : a.dtype == DFK_BF16 ? BF16::load1(a.logits, i) : FP16::load1(a.logits, i);
}

constexpr int kRouteWaves = 4;

// GROUPS: keys of the workgroup's tokens go through LDS (`keys`: E doubles and one of padding per token), where a lane per group finds the
// group's best.
template <int L, int V, bool BY_LOGIT, bool GROUPS>
__global__ __launch_bounds__(kRouteWaves * 64) void k_route(RouteArgs a) {
    extern __shared__ __attribute__((aligned(16))) double keys[];
    constexpr int PER_WAVE = 64 / L;
    const int tid = threadIdx.x, lane = tid & (L - 1), local = tid / L;
    const int token = (int)blockIdx.x * (kRouteWaves * PER_WAVE) + local;
    const bool live = token < a.M;                 // (a token past the end repeats the last one and stores nothing)
    const size_t row = (size_t)min(token, a.M - 1) * a.E;

    float x[V];
    unsigned bad = 0;
    const auto read = [&](auto load) {             // (the type is asked for once, and every lane loads: no branches between the loads)
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = load(row + min(v * L + lane, a.E - 1));
    };
    if (a.dtype == DFK_FP32) read([&](size_t i) { return ((const float*)a.logits)[i]; });
    else if (a.dtype == DFK_BF16) read([&](size_t i) { return BF16::load1(a.logits, i); });
    else read([&](size_t i) { return FP16::load1(a.logits, i); });
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v * L + lane >= a.E) x[v] = -INFINITY;
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (x[v] != x[v] || (x[v] == INFINITY && !a.sigmoid)) { bad = 1; x[v] = -INFINITY; }
        top = fmaxf(top, x[v]);
    }
    bad = or_across<L>(bad);
    double key[V], total = 1.0, shift = 0.0;
    if (!a.sigmoid) {
        top = max_across<L>(top);
        if (top == -INFINITY) top = 0.f;
        shift = (double)top;
    }
    if constexpr (BY_LOGIT) {
        if (!a.sigmoid) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) s += __builtin_amdgcn_exp2f((x[v] - top) * 1.44269504088896341f);
            total = (double)sum_across<L>(s);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = tagged((double)x[v], v * L + lane);
    } else {
        double s = 0.0, score[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const double d = (double)x[v] - shift;
            if (a.sigmoid) score[v] = sigmoid64(d);
            else { score[v] = d < -745.0 ? 0.0 : exp64(d); s += score[v]; }
        }
        double norm = 1.0;
        if (!a.sigmoid) {
            total = sum_across<L>(s);
            norm = total > 0.0 ? 1.0 / total : 0.0;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = v * L + lane;
            double c = a.sigmoid ? score[v] : score[v] * norm;
            if (a.bias && e < a.E) c += (double)a.bias[e];
            key[v] = tagged(x[v] == -INFINITY ? -HUGE_VAL : c, e);
        }
    }

    if constexpr (GROUPS) {
        double* mine = keys + (size_t)local * (a.E + 1);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v * L + lane < a.E) mine[v * L + lane] = key[v];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        __builtin_amdgcn_wave_barrier();           // a token's lanes are in one wavefront
        constexpr int VG = 64 / L;
        double group[VG];
#pragma unroll
        for (int v = 0; v < VG; ++v) {
            const int gr = v * L + lane;
            double b1 = -HUGE_VAL, b2 = -HUGE_VAL;
            if (gr < a.n_groups) {
                const double* k = mine + gr * a.group_size;
                const auto take = [&](double y) {
                    b2 = __builtin_fmax(b2, __builtin_fmin(b1, y));
                    b1 = __builtin_fmax(b1, y);
                };
                int i = 0;
                for (; i + 8 <= a.group_size; i += 8) {
                    double y[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) y[u] = k[i + u];
#pragma unroll
                    for (int u = 0; u < 8; ++u) take(y[u]);
                }
                for (; i < a.group_size; ++i) take(k[i]);
            }
            // The tags of the keys would count in the sum: without them, groups of equal scores are equal.
            const auto bare = [](double k) { return __longlong_as_double(__double_as_longlong(k) & ~(long long)kTagMask); };
            double c = b1;
            if (b1 > -HUGE_VAL) c = bare(b1) + (a.group_top == 2 && b2 > -HUGE_VAL ? bare(b2) : 0.0);
            group[v] = tagged(c, gr);
        }
        unsigned lo = 0, hi = 0;                   // the groups that are taken
        double last = HUGE_VAL;
        for (int i = 0; i < a.top_groups; ++i) {
            double m = -HUGE_VAL;
#pragma unroll
            for (int v = 0; v < VG; ++v) m = __builtin_fmax(m, group[v] < last ? group[v] : -HUGE_VAL);
            m = max_across<L>(m);
            if (m == -HUGE_VAL) break;
            last = m;
            const unsigned gr = index_of(m);
            if (gr < 32) lo |= 1u << gr; else hi |= 1u << (gr - 32);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const unsigned gr = (unsigned)(v * L + lane) / (unsigned)a.group_size;
            const unsigned bit = gr < 32 ? lo >> gr : gr < 64 ? hi >> (gr - 32) : 0u;
            if (!(bit & 1u)) key[v] = -HUGE_VAL;
        }
    }

    double pick = -HUGE_VAL, last = HUGE_VAL;      // lane j keeps the j-th
    for (int j = 0; j < a.K; ++j) {
        double m = -HUGE_VAL;
#pragma unroll
        for (int v = 0; v < V; ++v) m = __builtin_fmax(m, below(key[v], last));
        last = max_across<L>(m);
        if (lane == j) pick = last;
    }
    const bool some = lane < a.K && pick > kNone;
    const int e = some ? (int)index_of(pick) : -1;
    // (64 bits here: sigmoids that fp32 cannot hold have proportions all the same)
    double s = 0.0;
    if (some) {
        const double d = (double)logit_at(a, row + e) - shift;
        s = a.sigmoid ? sigmoid64(d) : (d < -745.0 ? 0.0 : exp64(d)) / total;
    }
    if (a.renormalise) {
        const double all = sum_across<L>(s);
        s = all > 0.0 ? s / all : 0.0;
    }
    const float w = (float)((double)a.scale * s);
    if (live && lane < a.K) {
        const size_t at = (size_t)token * a.K + lane;
        a.experts[at] = e;
        a.weights[at] = bad ? NAN : w;
    }
}

template <int L, int V>
hipError_t launch_route(const RouteArgs& a, bool by_logit, hipStream_t st) {
    constexpr int tokens = kRouteWaves * 64 / L;
    const dim3 grid((unsigned)((a.M + tokens - 1) / tokens)), block(kRouteWaves * 64);
    if (a.n_groups > 1) {
        const size_t lds = (size_t)tokens * (a.E + 1) * sizeof(double);   // at most 16 x 257, 8 x 513 or 4 x 1025 doubles: below 64 KB
        return by_logit ? launch_kernel(k_route<L, V, true, true>, grid, block, lds, st, a) : launch_kernel(k_route<L, V, false, true>, grid, block, lds, st, a);
    }
    return by_logit ? launch_kernel(k_route<L, V, true, false>, grid, block, 0, st, a) : launch_kernel(k_route<L, V, false, false>, grid, block, 0, st, a);
}

template <int L>
hipError_t launch_route(const RouteArgs& a, bool by_logit, hipStream_t st) {
    const int v = (a.E + L - 1) / L;
    if (v <= 1) return launch_route<L, 1>(a, by_logit, st);
    if (v <= 2) return launch_route<L, 2>(a, by_logit, st);
    if (v <= 4) return launch_route<L, 4>(a, by_logit, st);
    if (v <= 8) return launch_route<L, 8>(a, by_logit, st);
    return launch_route<L, 16>(a, by_logit, st);
}

}  // namespace
}  // namespace dfk

using namespace dfk;

extern "C" dfk_status_t dfk_moe_route(const void* logits, const float* bias, int* experts, float* weights,
                                      int M, int n_experts, int top_k, dfk_dtype_t dtype, dfk_score_t score,
                                      int n_groups, int top_groups, int group_top, int renormalise, float scale, void* stream) {
    if (!logits || !experts || !weights || M < 1 || n_experts < 1 || top_k < 1) return DFK_ERR_INVALID_ARG;
    if (!known_dtype(dtype) || (score != DFK_SCORE_SOFTMAX && score != DFK_SCORE_SIGMOID)) return DFK_ERR_INVALID_ARG;
    if (n_groups < 1 || top_groups < 1 || top_groups > n_groups || group_top < 1 || group_top > 2 || !std::isfinite(scale)) return DFK_ERR_INVALID_ARG;
    if (M > DFK_MAX_ROWS || n_experts > DFK_MAX_EXPERTS || top_k > DFK_MAX_TOP_K || n_groups > 64 || n_experts % n_groups ||
        top_k > n_experts / n_groups * top_groups)
        return DFK_ERR_UNSUPPORTED_SHAPE;
    if ((uintptr_t)logits % elt_bytes(dtype) || (uintptr_t)bias % 4 || (uintptr_t)experts % 4 || (uintptr_t)weights % 4) return DFK_ERR_ALIGNMENT;
    const size_t nl = (size_t)M * n_experts * elt_bytes(dtype), nk = (size_t)M * top_k * 4, nb = bias ? (size_t)n_experts * 4 : 0;
    if (overlaps(experts, nk, weights, nk) || overlaps(experts, nk, logits, nl) || overlaps(weights, nk, logits, nl) ||
        (bias && (overlaps(experts, nk, bias, nb) || overlaps(weights, nk, bias, nb))))
        return DFK_ERR_ALIAS;
    const RouteArgs a{logits, bias, experts, weights, M, n_experts, top_k, (int)dtype, score == DFK_SCORE_SIGMOID,
                      n_groups, n_experts / n_groups, top_groups, group_top, renormalise, scale};
    const bool by_logit = !bias && (n_groups == 1 || group_top == 1);
    // Lanes of a token: 16 spend the fewest instructions (their reductions take four steps, and serve four tokens at once); with fewer tokens, more lanes
    // have fewer one after the other.  us with 16 / 32 / 64, 8 of 256 experts by biased sigmoids: 1024 tokens 10.6 / 7.1 / 5.3, 4096 10.8 / 8.6 / 8.5,
    // 16384 20.3 / 20.8 / 24.7; 8 of 128 by logits: 2048 5.1 / 4.1 / 4.6, 8192 6.0 / 6.7 / 9.7.
    int lanes = M <= 1024 || (M <= 2048 && n_experts > 192) ? 64 : M <= 4096 || (M <= 8192 && n_experts > 192) ? 32 : 16;
    if (lanes == 16 && (top_k > 16 || n_experts > 256)) lanes = 32;
    if (n_experts > 512) lanes = 64;
    const hipError_t e = lanes == 64   ? launch_route<64>(a, by_logit, (hipStream_t)stream)
                         : lanes == 32 ? launch_route<32>(a, by_logit, (hipStream_t)stream)
                                       : launch_route<16>(a, by_logit, (hipStream_t)stream);
    return e == hipSuccess ? DFK_OK : hip_fail(e);
}
