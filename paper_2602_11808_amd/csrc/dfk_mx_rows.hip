// MX from rows of 16 or 32 bits and back, and the residual's addition with the RMS norm whose result may be MX.
#include "dfk_mx_device.h"

namespace dfk {
namespace {

// The largest magnitude of a block whose 32 values four neighbouring lanes hold.
__device__ __forceinline__ unsigned mx_top_of_quad(unsigned t) {
    t = max(t, (unsigned)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, true));        // lane ^ 1
    return max(t, (unsigned)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, true));     // lane ^ 2
}

// Eight elements, vector i of a tensor.
template <typename E>
__device__ __forceinline__ void load8(const void* p, size_t i, float (&f)[8]) {
    if constexpr (E::BYTES == 2) {
        E::widen(ld16(p, i), f);
    } else {
        float a[4], b[4];
        FP32::widen(ld16(p, 2 * i), a);
        FP32::widen(ld16(p, 2 * i + 1), b);
#pragma unroll
        for (int k = 0; k < 4; ++k) { f[k] = a[k]; f[4 + k] = b[k]; }
    }
}
template <typename E>
__device__ __forceinline__ void store8(void* p, size_t i, const float (&f)[8]) {
    if constexpr (E::BYTES == 2) {
        u32x4 v;
        v.x = E::pack2(f[0], f[1]); v.y = E::pack2(f[2], f[3]); v.z = E::pack2(f[4], f[5]); v.w = E::pack2(f[6], f[7]);
        ((u32x4*)p)[i] = v;
    } else {
        FP32::store4(p, 8 * i, f[0], f[1], f[2], f[3]);
        FP32::store4(p, 8 * i + 4, f[4], f[5], f[6], f[7]);
    }
}

// Eight values as a quarter of a block, vector i of the MX tensor; all four lanes of a block call it.
template <int MX>
__device__ __forceinline__ void store_mx8(unsigned char* q, unsigned char* s, size_t i, const float (&f)[8]) {
    unsigned top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = mx_top(top, f[k]);
    const unsigned scale = mx_scale_of<MX>(mx_top_of_quad(top));
    const float a[4] = {f[0], f[1], f[2], f[3]}, b[4] = {f[4], f[5], f[6], f[7]};
    if constexpr (MX == DFK_MXFP4) ((unsigned*)q)[i] = mx_elements<MX>(a, scale) | (mx_elements<MX>(b, scale) << 16);
    else ((uint2*)q)[i] = make_uint2(mx_elements<MX>(a, scale), mx_elements<MX>(b, scale));
    if ((i & 3) == 0) s[i >> 2] = (unsigned char)scale;
}

template <typename E, int MX>
__global__ __launch_bounds__(256) void k_mx_quantize(const void* X, unsigned char* q, unsigned char* s, size_t vecs) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= vecs) return;                     // (whole blocks: a multiple of 4)
    float f[8];
    load8<E>(X, i, f);
    store_mx8<MX>(q, s, i, f);
}

template <typename E, int MX>
__global__ __launch_bounds__(256) void k_mx_dequantize(const unsigned char* q, const unsigned char* s, void* Y, size_t vecs) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= vecs) return;
    const int e = s[i >> 2];
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 v[4];
    if constexpr (MX == DFK_MXFP4) {
        const unsigned w = ((const unsigned*)q)[i];
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
    } else {
        const uint2 w = ((const uint2*)q)[i];
        v[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false);
        v[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
        v[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false);
        v[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
    }
    float f[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = e == 255 ? __builtin_nanf("") : __builtin_ldexpf(v[k / 2][k % 2], e - 127);
    store8<E>(Y, i, f);
}

// A row per workgroup, its sums H + delta kept in registers between the sum of their squares and the results.  Squares and their sum have 64 bits, so that neither large nor small rows leave their
// range, which hides beside the loads (4096 rows of 4096 into MXFP8 25.4 -> 25.7 us; the products too would be 26.9).  Bound by memory: 118 MB at 4.6 TB/s in and out, a large copy's rate being 5.0.
template <typename E, int NT, int NV>
__global__ __launch_bounds__(NT) void k_add_rmsnorm(AddNormArgs a) {
    __shared__ double part[NT / 64];
    const int tid = threadIdx.x, vecs = a.d / 8;
    const size_t row = (size_t)blockIdx.x * vecs;
    float f[NV][8];
    double sq = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + NT * j;
        if (v >= vecs) continue;
        load8<E>(a.H, row + v, f[j]);
        if (a.delta) {
            float g[8];
            load8<E>(a.delta, row + v, g);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[j][k] += g[k];
            store8<E>(a.H_out, row + v, f[j]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sq += (double)f[j][k] * f[j][k];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sq += __shfl_xor(sq, o);
    if (NT > 64) {
        if ((tid & 63) == 0) part[tid >> 6] = sq;
        __syncthreads();
        sq = 0.0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) sq += part[w];
    }
    const float r = (float)(1.0 / sqrt(sq / a.d + (double)a.eps));
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + NT * j;
        if (v >= vecs) continue;
        float w[8];
        load8<E>(a.w, v, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[j][k] = f[j][k] * r * w[k];
        if (a.N) store8<E>(a.N, row + v, f[j]);
        if (a.q) {
            if (a.mx == DFK_MXFP4) store_mx8<DFK_MXFP4>(a.q, a.s, row + v, f[j]);
            else store_mx8<DFK_MXFP8>(a.q, a.s, row + v, f[j]);
        }
    }
}

template <typename E>
hipError_t norm_of(const AddNormArgs& a, hipStream_t st) {
    const int vecs = a.d / 8;
    const dim3 grid((unsigned)a.rows);
    if (vecs <= 64) return launch_kernel(k_add_rmsnorm<E, 64, 1>, grid, dim3(64), 0, st, a);
    if (vecs <= 128) return launch_kernel(k_add_rmsnorm<E, 128, 1>, grid, dim3(128), 0, st, a);
    if (vecs <= 256) return launch_kernel(k_add_rmsnorm<E, 256, 1>, grid, dim3(256), 0, st, a);
    if (vecs <= 512) return launch_kernel(k_add_rmsnorm<E, 256, 2>, grid, dim3(256), 0, st, a);
    if (vecs <= 1024) return launch_kernel(k_add_rmsnorm<E, 256, 4>, grid, dim3(256), 0, st, a);
    if (vecs <= 2048) return launch_kernel(k_add_rmsnorm<E, 512, 4>, grid, dim3(512), 0, st, a);
    if (vecs <= 4096) return launch_kernel(k_add_rmsnorm<E, 1024, 4>, grid, dim3(1024), 0, st, a);
    return hipErrorInvalidValue;
}

constexpr size_t kVecsOfLaunch = (size_t)1 << 31;      // (a launch has fewer than 2^32 threads)

// Runs `one` on a tensor's vectors of 8 elements, as many at a time as a launch takes: one(first, count, grid).
template <typename F>
hipError_t by_vecs(size_t vecs, F one) {
    for (size_t v = 0; v < vecs; v += kVecsOfLaunch) {
        const size_t n = vecs - v < kVecsOfLaunch ? vecs - v : kVecsOfLaunch;
        if (const hipError_t e = one(v, n, dim3((unsigned)((n + 255) / 256))); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename E, int MX>
hipError_t quantize_of(const void* X, unsigned char* q, unsigned char* s, size_t vecs, hipStream_t st) {
    return by_vecs(vecs, [&](size_t v, size_t n, dim3 grid) {
        return launch_kernel(k_mx_quantize<E, MX>, grid, dim3(256), 0, st, (const void*)((const char*)X + v * 8 * E::BYTES), q + v * (MX == DFK_MXFP4 ? 4 : 8), s + v / 4, n);
    });
}
template <typename E, int MX>
hipError_t dequantize_of(const unsigned char* q, const unsigned char* s, void* Y, size_t vecs, hipStream_t st) {
    return by_vecs(vecs, [&](size_t v, size_t n, dim3 grid) {
        return launch_kernel(k_mx_dequantize<E, MX>, grid, dim3(256), 0, st, q + v * (MX == DFK_MXFP4 ? 4 : 8), s + v / 4, (void*)((char*)Y + v * 8 * E::BYTES), n);
    });
}

}  // namespace

hipError_t launch_mx_quantize(const void* X, unsigned char* q, unsigned char* s, size_t elems, dfk_dtype_t dtype, int mx, hipStream_t st) {
    return dtype == DFK_BF16   ? (mx == DFK_MXFP4 ? quantize_of<BF16, DFK_MXFP4> : quantize_of<BF16, DFK_MXFP8>)(X, q, s, elems / 8, st)
           : dtype == DFK_FP16 ? (mx == DFK_MXFP4 ? quantize_of<FP16, DFK_MXFP4> : quantize_of<FP16, DFK_MXFP8>)(X, q, s, elems / 8, st)
                               : (mx == DFK_MXFP4 ? quantize_of<FP32, DFK_MXFP4> : quantize_of<FP32, DFK_MXFP8>)(X, q, s, elems / 8, st);
}
hipError_t launch_mx_dequantize(const unsigned char* q, const unsigned char* s, void* Y, size_t elems, dfk_dtype_t dtype, int mx, hipStream_t st) {
    return dtype == DFK_BF16   ? (mx == DFK_MXFP4 ? dequantize_of<BF16, DFK_MXFP4> : dequantize_of<BF16, DFK_MXFP8>)(q, s, Y, elems / 8, st)
           : dtype == DFK_FP16 ? (mx == DFK_MXFP4 ? dequantize_of<FP16, DFK_MXFP4> : dequantize_of<FP16, DFK_MXFP8>)(q, s, Y, elems / 8, st)
                               : (mx == DFK_MXFP4 ? dequantize_of<FP32, DFK_MXFP4> : dequantize_of<FP32, DFK_MXFP8>)(q, s, Y, elems / 8, st);
}
hipError_t launch_add_rmsnorm(const AddNormArgs& a, dfk_dtype_t dtype, hipStream_t st) {
    return dtype == DFK_BF16 ? norm_of<BF16>(a, st) : dtype == DFK_FP16 ? norm_of<FP16>(a, st) : norm_of<FP32>(a, st);
}

}  // namespace dfk
