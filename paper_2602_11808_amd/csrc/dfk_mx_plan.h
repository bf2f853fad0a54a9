// Which kernel and tile a product with MXFP4 weights runs on.  Free of device code, so that a host program can check it.
#pragma once

#include "dfk_linear_plan.h"

namespace dfk {

// MXFP8 activations: whether their large and small elements are multiplied apart (dfk_mx_device.h), which loses nothing and takes twice as many instructions.  Up to 64 rows the
// weights' bytes are what counts; beyond, it is for fp32 results only, as the error, 1.3e-5 of the result on the root-mean-square for normally distributed ones, is 1/130 of what
// rounding to bf16 leaves and 1/15 of half's.
constexpr int kMxExactRows = 64;
inline bool mx_exact_sums(int M, int out_fp32) { return M <= kMxExactRows || out_fp32; }

}  // namespace dfk
