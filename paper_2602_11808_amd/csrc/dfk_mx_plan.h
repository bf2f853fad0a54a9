// Which kernel and tile a product with MXFP4 weights runs on.  Free of device code, so that a host program can check it.
#pragma once

#include "dfk_linear_plan.h"

namespace dfk {

// MXFP8 activations: whether their large and small elements are multiplied apart (dfk_mx_device.h), which loses nothing and takes twice as many instructions.  Up to 64 rows the
// weights' bytes are what counts; beyond, it is for fp32 results only, as the error, 1.3e-5 of the result on the root-mean-square for normally distributed ones, is 1/130 of what
// rounding to bf16 leaves and 1/15 of half's.
constexpr int kMxExactRows = 64;
inline bool mx_exact_sums(int M, int out_fp32) { return M <= kMxExactRows || out_fp32; }

// The weight stream (dfk_mx_stream.hip): NT tiles of 16 weight rows a wavefront, TT tiles of activations, NW wavefronts, rings of D chunks of 256 k.
constexpr int kMxStreamDepth = 4, kMxStreamDepthGated = 3;
constexpr int kMxStreamHalf = 80 * 1024 - 128;       // of LDS: two workgroups a CU
constexpr int mx_stream_stage(int NT, bool words) { return NT * 2048 + (words ? 256 * ((NT + 1) / 2) : 512 * NT); }
constexpr int mx_x_pitch(bool x8, int K) { return ((x8 ? K : K / 2) + 1023) / 1024 * 1024 + 16; }
inline size_t mx_stream_lds(bool x8, int NT, int TT, int NW, int D, bool words, int M, int K) {
    return (size_t)NW * D * mx_stream_stage(NT, words) + (size_t)NW * NT * TT * 1024 + (size_t)M * mx_x_pitch(x8, K) + ((size_t)M * (K / 32) + 1039) / 1024 * 1024;
}
// Whether the activations fit beside the rings.
inline bool mx_stream_fits(int M, int K, bool x8, bool gated) {
    const int TT = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    return M <= 64 && mx_stream_lds(x8, gated ? 2 : 1, TT, 8, gated ? kMxStreamDepthGated : kMxStreamDepth, K % 128 == 0, M, K) <= 160 * 1024 - 256;
}

}  // namespace dfk
