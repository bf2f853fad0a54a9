// Epilogues of the linear layers (device code).
#pragma once

#include "dfk_device.h"
#include "dfk_ops.h"

namespace dfk {

// The activations in fp32, each with the library's own exp and erf: a result may be stored as fp32.
__device__ __forceinline__ float apply_act(float v, int act) {
    switch (act) {
        case DFK_ACT_RELU: return v > 0.f ? v : (v != v ? v : 0.f);
        case DFK_ACT_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
        // v/2 (1 + tanh(u)) = v Sigmoid(2u)
        case DFK_ACT_GELU_TANH: return v / (1.f + expf(-1.5957691216057308f * (v + 0.044715f * v * v * v)));
        case DFK_ACT_SILU: return v / (1.f + expf(-v));
    }
    return v;
}

// Columns n .. n+3 of row m of a linear layer (those below N): bias, activation, residual, one rounding to OUT.
template <typename E, typename OUT>
__device__ __forceinline__ void linear_store4(const TileArgs& a, size_t m, int n, const float (&sum)[4]) {
    const size_t at = m * (size_t)a.N + n;
    float v[4] = {sum[0], sum[1], sum[2], sum[3]}, t[4];
    if (a.vec4) {
        if (n >= a.N) return;
        if (a.bias) {
            E::load4(a.bias, n, t);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += t[i];
        }
        if (a.act != DFK_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = apply_act(v[i], a.act);
        }
        if (a.resid) {
            OUT::load4(a.resid, at, t);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += t[i];
        }
        OUT::store4(a.out, at, v[0], v[1], v[2], v[3]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n + i < a.N) {
            float x = v[i];
            if (a.bias) x += E::load1(a.bias, n + i);
            x = apply_act(x, a.act);
            if (a.resid) x += OUT::load1(a.resid, at + i);
            OUT::store(a.out, at + i, x);
        }
    }
}

}  // namespace dfk
