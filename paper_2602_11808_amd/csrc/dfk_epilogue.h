// Epilogues of the linear layers and of the experts (device code).
#pragma once

#include <type_traits>

#include "dfk_device.h"
#include "dfk_ops.h"

namespace dfk {

// kEpiRows: rows of bf16 calls are halves times a power of two per 64 columns, those of the other types fp32.
template <typename E> constexpr bool kHalfRows = false;
template <> inline constexpr bool kHalfRows<BF16> = true;

// The activations in fp32: a result may be stored as fp32.
// GELU: Phi(-|v|) = exp(-v^2 / 2) P(t), t = 1 / (1 + 0.291 |v|), P a polynomial without constant term that is fitted to 0 <= |v| <= 13.3, where results end: off by
// 3.3e-9 (1 + 4 v^2) of the value, less than the exponent's roundings (so that the hardware's exp2 and reciprocal, about 1 ulp each, do).  It is that of the smaller side, so that
// nothing cancels for negative v: of v / 2 (1 + erf) nothing is left at -6.  What GELU takes of 4096 x 4096 -> 14336 with fp32 results: 19 us, with 1 + erff
// 45, with erfcf 75.
__device__ __forceinline__ float apply_act(float v, int act) {
    switch (act) {
        case DFK_ACT_RELU: return v > 0.f ? v : (v != v ? v : 0.f);
        case DFK_ACT_GELU: {
            const float t = __builtin_amdgcn_rcpf(1.f + 0.291f * fabsf(v));
            const float p = t * (0.115935067f + t * (0.118786174f + t * (0.0869164702f + t * (0.162575332f + t * (-0.1178174f + t * (0.277196456f + t * (-0.18102303f + t * 0.0374309335f)))))));
            const float tail = p * __builtin_amdgcn_exp2f(v * (v * -0.72134752044448170f));       // 1 - Phi(|v|)
            return v * (v >= 0.f ? 1.f - tail : tail);
        }
        // v/2 (1 + tanh(u)) = v Sigmoid(2u)
        case DFK_ACT_GELU_TANH: return v / (1.f + expf(-1.5957691216057308f * (v + 0.044715f * v * v * v)));
        case DFK_ACT_SILU: return v / (1.f + expf(-v));
    }
    return v;
}

// The same for results that are rounded to 16 bits next, on the hardware's exp2 and reciprocal too; GELU's polynomial has two terms less and is off by 1.7e-7 (1 + 4 v^2) of the value:
// at most 3 % of half a step, in bf16 at -13 and in half at -4.2, where its normal results end.  What the activation alone takes of 4096 x 4096 -> 14336: GELU 41 us.
__device__ __forceinline__ float apply_act_fast(float v, int act) {
    const float kLog2e = 1.44269504088896341f;
    switch (act) {
        case DFK_ACT_RELU: return v > 0.f ? v : (v != v ? v : 0.f);
        case DFK_ACT_GELU: {
            const float t = __builtin_amdgcn_rcpf(1.f + 0.293f * fabsf(v));
            const float p = t * (0.117896462f + t * (0.104079986f + t * (0.170835252f + t * (-0.0737567082f + t * (0.267643269f + t * -0.0866983449f)))));
            const float tail = p * __builtin_amdgcn_exp2f(v * (v * (-0.5f * kLog2e)));       // 1 - Phi(|v|)
            return v * (v >= 0.f ? 1.f - tail : tail);
        }
        case DFK_ACT_GELU_TANH: {
            const float c = -kLog2e * 1.5957691216057308f;
            return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * (c + 0.044715f * c * (v * v))));
        }
        case DFK_ACT_SILU: return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * v));
    }
    return v;
}

// Four elements from element i on, wherever they start: one access all the same, which the hardware takes at any alignment.
struct alignas(4) FourFloats { float v[4]; };
struct alignas(2) FourHalves { uint16_t v[4]; };
template <typename T>
__device__ __forceinline__ void load4_anywhere(const void* p, size_t i, float (&f)[4]) {
    if constexpr (T::BYTES == 4) {
        const FourFloats t = *(const FourFloats*)((const float*)p + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = t.v[k];
    } else {
        const FourHalves t = *(const FourHalves*)((const uint16_t*)p + i);
        T::widen2((unsigned)t.v[0] | (unsigned)t.v[1] << 16, f[0], f[1]);
        T::widen2((unsigned)t.v[2] | (unsigned)t.v[3] << 16, f[2], f[3]);
    }
}
template <typename T>
__device__ __forceinline__ void store4_anywhere(void* p, size_t i, const float (&f)[4]) {
    if constexpr (T::BYTES == 4) {
        *(FourFloats*)((float*)p + i) = FourFloats{f[0], f[1], f[2], f[3]};
    } else {
        const unsigned lo = T::pack2(f[0], f[1]), hi = T::pack2(f[2], f[3]);
        *(FourHalves*)((uint16_t*)p + i) = FourHalves{(uint16_t)lo, (uint16_t)(lo >> 16), (uint16_t)hi, (uint16_t)(hi >> 16)};
    }
}

// Columns n .. n+3 of row m of a linear layer (those below N): bias (unless the sums have it), activation, residual, one rounding to OUT.  (Results of 50257 columns one at a time:
// 1000 x 1024 182 us, four at a time 149.)
template <typename E, typename OUT, bool BIAS = true>
__device__ __forceinline__ void linear_store4(const TileArgs& a, size_t m, int n, const float (&sum)[4]) {
    const size_t at = m * (size_t)a.N + n;
    const auto whole = [&](auto vec_) {
        constexpr bool VEC = decltype(vec_)::value;
        float v[4] = {sum[0], sum[1], sum[2], sum[3]}, t[4];
        if (BIAS && a.bias) {
            if constexpr (VEC) E::load4(a.bias, n, t); else load4_anywhere<E>(a.bias, n, t);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += t[i];
        }
        if (a.act != DFK_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = OUT::BYTES == 2 ? apply_act_fast(v[i], a.act) : apply_act(v[i], a.act);
        }
        if (a.resid) {
            if constexpr (VEC) OUT::load4(a.resid, at, t); else load4_anywhere<OUT>(a.resid, at, t);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += t[i];
        }
        if constexpr (VEC) OUT::store4(a.out, at, v[0], v[1], v[2], v[3]); else store4_anywhere<OUT>(a.out, at, v);
    };
    if (a.vec4) {
        if (n < a.N) whole(std::true_type{});
    } else if (n + 4 <= a.N) {
        whole(std::false_type{});
    } else {
        for (int i = 0; i < a.N - n; ++i) {          // (the last columns)
            float x = i == 0 ? sum[0] : i == 1 ? sum[1] : sum[2];
            if (BIAS && a.bias) x += E::load1(a.bias, n + i);
            x = OUT::BYTES == 2 ? apply_act_fast(x, a.act) : apply_act(x, a.act);
            if (a.resid) x += OUT::load1(a.resid, at + i);
            OUT::store(a.out, at + i, x);
        }
    }
}

}  // namespace dfk
