// Linear layers: argument checks and dispatch of dfk_linear.
#include "dfk_linear_plan.h"
#include "dfk_ops.h"

namespace dfk {
namespace {

constexpr int kMaxIn = 131072, kMaxOut = 1 << 20;

bool linear_shape(int M, int n_out, int n_in) {
    return M >= 1 && M <= DFK_MAX_ROWS && n_out >= 1 && n_out <= kMaxOut && n_in >= 8 && n_in <= kMaxIn && n_in % 8 == 0;
}

size_t linear_workspace(int M, int n_out) { return 256 + linear_partial_bound(M, n_out); }

}  // namespace
}  // namespace dfk

using namespace dfk;

extern "C" {

dfk_status_t dfk_linear(const void* X, const void* W, const void* bias, const void* residual, void* Y,
                        int M, int n_out, int n_in, dfk_dtype_t dtype, dfk_dtype_t out_dtype, dfk_act_t act,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !W || !Y || M < 1 || n_out < 1 || n_in < 1) return DFK_ERR_INVALID_ARG;
    if (!known_dtype(dtype) || (out_dtype != dtype && out_dtype != DFK_FP32)) return DFK_ERR_INVALID_ARG;
    if ((int)act < DFK_ACT_NONE || (int)act > DFK_ACT_SILU) return DFK_ERR_INVALID_ARG;
    if (!linear_shape(M, n_out, n_in)) return DFK_ERR_UNSUPPORTED_SHAPE;
    const size_t es = elt_bytes(dtype), os = elt_bytes(out_dtype);
    if ((uintptr_t)X % 16 || (uintptr_t)W % 16 || (uintptr_t)bias % es || (uintptr_t)residual % os || (uintptr_t)Y % os ||
        (uintptr_t)workspace % 256)
        return DFK_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < linear_workspace(M, n_out)) return DFK_ERR_WORKSPACE;
    const size_t nx = (size_t)M * n_in * es, nw = (size_t)n_out * n_in * es, nb = bias ? n_out * es : 0, ny = (size_t)M * n_out * os;
    const auto hits = [&](const void* p, size_t n) { return n && (overlaps(Y, ny, p, n) || overlaps(workspace, workspace_bytes, p, n)); };
    if (hits(X, nx) || hits(W, nw) || hits(bias, nb) || overlaps(workspace, workspace_bytes, Y, ny)) return DFK_ERR_ALIAS;
    if (residual && residual != Y && hits(residual, ny)) return DFK_ERR_ALIAS;

    TileArgs a{};
    a.A = X; a.B = W; a.out = Y; a.bias = bias; a.resid = residual;
    a.M = M; a.N = n_out; a.K = n_in; a.act = (int)act;
    a.out_fp32 = out_dtype == DFK_FP32; a.splits = 1;
    a.partial = (float*)workspace; a.partial_bytes = workspace_bytes; a.pitch = (n_out + 3) / 4 * 4;
    a.vec4 = n_out % 4 == 0 && (uintptr_t)Y % (4 * os) == 0 && (uintptr_t)residual % (4 * os) == 0 && (uintptr_t)bias % (4 * es) == 0;
    hipError_t e;
    if (dtype == DFK_FP32) {
        e = launch_linear_f32(a, (hipStream_t)stream);
    } else {
        const LinearPlan p = linear_plan(M, n_out, n_in);
        a.splits = p.splits;
        e = p.stream ? launch_linear_stream(a, dtype, p.nt, (hipStream_t)stream) : launch_linear_tile(a, dtype, p.tile, (hipStream_t)stream);
    }
    return e == hipSuccess ? DFK_OK : hip_fail(e);
}

size_t dfk_linear_workspace_bytes(int M_max, int n_out, int n_in, dfk_dtype_t dtype) {
    if (!known_dtype(dtype) || !linear_shape(M_max, n_out, n_in)) return 0;
    return linear_workspace(M_max, n_out);
}

}  // extern "C"
