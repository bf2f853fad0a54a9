// Microscaled (MX) tensors: storage, arguments of their calls and launchers shared by their files.
//
// 32 neighbours of a row, a block, share a scale 2^(s - 127), s a byte (255: the block is NaN).  MXFP4: elements e2m1 (0 .5 1 1.5 2 3 4 6 and a sign), element 2j of a
// row in the low half of its byte j.  MXFP8: elements e4m3 (up to 448).  A row of K has K / 2 or K bytes of elements and K / 32 of scales, rows follow each other.
#pragma once

#include "dfk_ops.h"

namespace dfk {

constexpr int kMxBlock = 32;
inline bool known_mx(int mx) { return mx == DFK_MXFP4 || mx == DFK_MXFP8; }
inline size_t mx_data_bytes(size_t elems, int mx) { return mx == DFK_MXFP4 ? elems / 2 : elems; }

// Products with MXFP4 weights.  t: the linear layer's epilogue (A, B, B2: elements, K: length of the sum).
struct MxArgs {
    TileArgs t;
    const unsigned char* As;       // scales of A, B and B2
    const unsigned char* Bs;
    const unsigned char* B2s;
    int dtype;                     // dfk_dtype_t of bias and of a 16-bit result
    int out_mx;                    // gated half: format of the result, or -1: 16 bits into t.out
    unsigned char* q;              // its elements and scales
    unsigned char* qs;
};

struct AddNormArgs {
    const void* H;
    const void* delta;             // or NULL, as H_out then
    const void* w;
    void* H_out;
    void* N;                       // either may be NULL
    unsigned char* q;
    unsigned char* s;
    float eps;
    int rows, d, mx;
};

// rows (dfk_mx_rows.hip)
hipError_t launch_mx_quantize(const void* X, unsigned char* q, unsigned char* s, size_t elems, dfk_dtype_t dtype, int mx, hipStream_t st);
hipError_t launch_mx_dequantize(const unsigned char* q, const unsigned char* s, void* Y, size_t elems, dfk_dtype_t dtype, int mx, hipStream_t st);
hipError_t launch_add_rmsnorm(const AddNormArgs& a, dfk_dtype_t dtype, hipStream_t st);

// many rows (dfk_mx_tile.hip); x_mx: format of A
hipError_t launch_mx_linear_tile(const MxArgs& a, int x_mx, int tile, hipStream_t st);
hipError_t launch_mx_gateup_tile(const MxArgs& a, int x_mx, int tile, hipStream_t st);

// few rows (dfk_mx_stream.hip), form and tile: mx_plan
hipError_t launch_mx_linear_stream(const MxArgs& a, int x_mx, int form, hipStream_t st);
hipError_t launch_mx_gateup_stream(const MxArgs& a, int x_mx, int form, hipStream_t st);

}  // namespace dfk
