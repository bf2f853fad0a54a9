// Matrix products of the fp32 type on the fp32 matrix instructions (gfx950), any shape.
//
// out[m, n] = sum_k A[m, k] B[n, k].  A workgroup of four wavefronts
// owns 64 rows x 64 columns; 32 k a step are staged through registers into LDS, padded so that the 16 rows of an operand read
// start in different banks.  Within 16 k lane (q, g) of an operand holds row q, k = 4g .. 4g+3, read at once; v_mfma_f32_16x16x4
// number i takes element i of both, so the k order differs from the memory's but is the same for both operands.
// D: lane (q, g) holds row q of A and columns 4g .. 4g+3, which are stored together.
#include "dfk_epilogue.h"

namespace dfk {
namespace {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

constexpr int kStepK = 32;
constexpr int kPitch = kStepK + 4;   // floats

template <int EPI>
__global__ __launch_bounds__(256) void k_tile_f32(TileArgs a) {
    using E = FP32;
    constexpr int NB = EPI == kEpiGated ? 2 : 1;
    constexpr bool GROUPS = EPI != kEpiLinear;
    __shared__ float lds_a[64 * kPitch];
    __shared__ float lds_b[NB][64 * kPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane & 15, g = lane >> 4;
    const int mt = (int)blockIdx.y, n0 = (int)blockIdx.x * 64;
    size_t row0 = (size_t)mt * 64;
    int rows, group = 0;
    if (GROUPS) {
        if (mt >= *a.plan.n_tiles) return;
        const int4 t = a.plan.tiles[mt];
        group = t.x; row0 = (size_t)t.y; rows = t.z;
    } else {
        rows = min(64, a.M - (int)row0);
    }
    // The staging: thread tid moves VPT 16-byte vectors of each operand per step: vector v of row v / VR.
    constexpr int VR = kStepK / E::VEC, VPT = 64 * VR / 256;
    const char* pa[VPT];
    const char* pb[NB][VPT];
    bool oka[VPT], okb[VPT];
    const size_t rb = (size_t)a.K * E::BYTES;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = tid + 256 * i, r = v / VR, c = v % VR;
        oka[i] = r < rows;
        okb[i] = n0 + r < a.N;
        size_t src = row0 + r;
        if (EPI == kEpiGated && oka[i]) src = (size_t)(a.plan.slot[row0 + r] / a.top_k);
        pa[i] = (const char*)a.A + (oka[i] ? src : 0) * rb + c * 16;
        const size_t bo = ((size_t)group * a.N + (okb[i] ? n0 + r : 0)) * rb + c * 16;
        pb[0][i] = (const char*)a.B + bo;
        if (NB == 2) pb[NB - 1][i] = (const char*)a.B2 + bo;
    }
    f32x4 acc[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto put = [&](float* dst, const char* p, bool ok, int i, int k0) {
        const int v = tid + 256 * i, r = v / VR, c = v % VR;
        u32x4 raw = u32x4{0, 0, 0, 0};
        if (ok && k0 + c * E::VEC < a.K) raw = *(const u32x4*)(p + (size_t)k0 * E::BYTES);   // (K is a multiple of 8: whole vectors)
        *(u32x4*)(dst + r * kPitch + c * E::VEC) = raw;
    };
    for (int k0 = 0; k0 < a.K; k0 += kStepK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            put(lds_a, pa[i], oka[i], i, k0);
#pragma unroll
            for (int b = 0; b < NB; ++b) put(lds_b[b], pb[b][i], okb[i], i, k0);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < kStepK / 16; ++h) {
            const f32x4 x = *(const f32x4*)(lds_a + (wave * 16 + q) * kPitch + 16 * h + 4 * g);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const f32x4 w = *(const f32x4*)(lds_b[b] + (t * 16 + q) * kPitch + 16 * h + 4 * g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[b][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], x[i], acc[b][t], 0, 0, 0);
                }
        }
    }
    const int r = wave * 16 + q;
    if (r >= rows) return;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int n = n0 + t * 16 + 4 * g;
        float v[4] = {acc[0][t][0], acc[0][t][1], acc[0][t][2], acc[0][t][3]};
        if (EPI == kEpiLinear) {
            linear_store4<E, E>(a, row0 + r, n, v);
        } else if (n < a.N) {   // (d_model and d_ff are multiples of 8)
            if (EPI == kEpiGated) {
                const float w = a.plan.weight[row0 + r];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = w * silu_mul(v[i], acc[NB - 1][t][i]);
                E::store4(a.out, (row0 + r) * (size_t)a.N + n, v[0], v[1], v[2], v[3]);
            } else {
                FP32::store4(a.out, (size_t)a.plan.slot[row0 + r] * a.N + n, v[0], v[1], v[2], v[3]);
            }
        }
    }
}

}  // namespace

hipError_t launch_linear_f32(const TileArgs& a, hipStream_t st) {
    return launch_kernel(k_tile_f32<kEpiLinear>, dim3((unsigned)((a.N + 63) / 64), (unsigned)((a.M + 63) / 64)), dim3(256), 0, st, a);
}

hipError_t launch_experts_f32(const TileArgs& a, int epi, hipStream_t st) {
    const dim3 grid((unsigned)((a.N + 63) / 64), (unsigned)a.plan.max_tiles);
    return epi == kEpiGated ? launch_kernel(k_tile_f32<kEpiGated>, grid, dim3(256), 0, st, a)
                            : launch_kernel(k_tile_f32<kEpiRows>, grid, dim3(256), 0, st, a);
}

}  // namespace dfk
