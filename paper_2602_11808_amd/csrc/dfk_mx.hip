// Microscaled tensors: argument checks and dispatch of their calls.
#include "dfk_mx.h"
#include "dfk_mx_plan.h"

namespace dfk {
namespace {

constexpr int kMxMaxIn = 131072, kMxMaxOut = 1 << 20;

bool mx_rows_shape(int rows, int cols) { return rows >= 1 && rows <= DFK_MAX_ROWS && cols >= kMxBlock && cols <= kMxMaxIn && cols % kMxBlock == 0; }
bool mx_linear_shape(int M, int n_out, int n_in) { return mx_rows_shape(M, n_in) && n_out >= 1 && n_out <= kMxMaxOut; }
bool mx_gateup_shape(int M, int d_ff, int d_model) { return mx_rows_shape(M, d_model) && mx_rows_shape(1, d_ff); }

size_t mx_workspace(int M, int n_out) { return 256 + linear_partial_bound(M, n_out); }
constexpr size_t kMxGateupWorkspace = 256;     // (nothing is split across workgroups)

// Rows of a launch: its threads are counted in 32 bits.
constexpr int kMxLaunchRows = 1 << 18;

// Runs `one` on a call's rows, kMxLaunchRows at a time.
template <typename F>
hipError_t by_launch(const MxArgs& a, int x_mx, size_t out_row, F one) {
    const size_t rows = (size_t)a.t.M;
    for (size_t m0 = 0; m0 < rows; m0 += kMxLaunchRows) {
        MxArgs b = a;
        b.t.M = (int)(rows - m0 < kMxLaunchRows ? rows - m0 : kMxLaunchRows);
        const size_t at = m0 * out_row, blocks = m0 * (a.t.K / kMxBlock);
        b.t.A = (const char*)a.t.A + blocks * (x_mx == DFK_MXFP4 ? 16 : 32);
        b.As = a.As + blocks;
        if (a.t.out) b.t.out = (char*)a.t.out + at;
        if (a.t.resid) b.t.resid = (const char*)a.t.resid + at;
        if (a.q) {
            b.q = a.q + at;
            b.qs = a.qs + m0 * (a.t.N / kMxBlock);
        }
        if (const hipError_t e = one(b); e != hipSuccess) return e;
    }
    return hipSuccess;
}

// One of a call's buffers.
struct Span {
    const void* p;
    size_t n;
    bool hits(const Span& o) const { return p && o.p && n && o.n && overlaps(p, n, o.p, o.n); }
};
// Whether an output overlaps an input or another output.
template <int NO, int NI>
bool any_overlap(const Span (&outs)[NO], const Span (&ins)[NI]) {
    for (int i = 0; i < NO; ++i) {
        for (int j = 0; j < NI; ++j)
            if (outs[i].hits(ins[j])) return true;
        for (int j = 0; j < i; ++j)
            if (outs[i].hits(outs[j])) return true;
    }
    return false;
}

}  // namespace
}  // namespace dfk

using namespace dfk;

extern "C" {

dfk_status_t dfk_mx_quantize(const void* X, void* Q, void* S, int rows, int cols, dfk_dtype_t dtype, dfk_mx_t mx, void* stream) {
    if (!X || !Q || !S || rows < 1 || cols < 1 || !known_dtype(dtype) || !known_mx((int)mx)) return DFK_ERR_INVALID_ARG;
    if (!mx_rows_shape(rows, cols)) return DFK_ERR_UNSUPPORTED_SHAPE;
    if ((uintptr_t)X % 16 || (uintptr_t)Q % 16 || (uintptr_t)S % 16) return DFK_ERR_ALIGNMENT;
    const size_t n = (size_t)rows * cols;
    const Span outs[] = {{Q, mx_data_bytes(n, (int)mx)}, {S, n / kMxBlock}}, ins[] = {{X, n * elt_bytes(dtype)}};
    if (any_overlap(outs, ins)) return DFK_ERR_ALIAS;
    const hipError_t e = launch_mx_quantize(X, (unsigned char*)Q, (unsigned char*)S, n, dtype, (int)mx, (hipStream_t)stream);
    return e == hipSuccess ? DFK_OK : hip_fail(e);
}

dfk_status_t dfk_mx_dequantize(const void* Q, const void* S, void* Y, int rows, int cols, dfk_mx_t mx, dfk_dtype_t dtype, void* stream) {
    if (!Q || !S || !Y || rows < 1 || cols < 1 || !known_dtype(dtype) || !known_mx((int)mx)) return DFK_ERR_INVALID_ARG;
    if (!mx_rows_shape(rows, cols)) return DFK_ERR_UNSUPPORTED_SHAPE;
    if ((uintptr_t)Y % 16 || (uintptr_t)Q % 16 || (uintptr_t)S % 16) return DFK_ERR_ALIGNMENT;
    const size_t n = (size_t)rows * cols;
    const Span outs[] = {{Y, n * elt_bytes(dtype)}}, ins[] = {{Q, mx_data_bytes(n, (int)mx)}, {S, n / kMxBlock}};
    if (any_overlap(outs, ins)) return DFK_ERR_ALIAS;
    const hipError_t e = launch_mx_dequantize((const unsigned char*)Q, (const unsigned char*)S, Y, n, dtype, (int)mx, (hipStream_t)stream);
    return e == hipSuccess ? DFK_OK : hip_fail(e);
}

dfk_status_t dfk_add_rmsnorm(const void* H, const void* delta, const void* norm_weight, float eps, void* H_out, void* N, void* Q, void* S,
                             int M, int d_model, dfk_dtype_t dtype, dfk_mx_t mx, void* stream) {
    if (!H || !norm_weight || (delta != nullptr) != (H_out != nullptr) || (Q != nullptr) != (S != nullptr) || (!N && !Q)) return DFK_ERR_INVALID_ARG;
    if (M < 1 || d_model < 1 || !known_dtype(dtype) || (Q && !known_mx((int)mx)) || !(eps >= 0.f) || eps > 3.0e38f) return DFK_ERR_INVALID_ARG;
    if (M > DFK_MAX_ROWS || d_model > kMaxDModel || d_model % (Q ? kMxBlock : 8) != 0) return DFK_ERR_UNSUPPORTED_SHAPE;
    const void* all[] = {H, delta, norm_weight, H_out, N, Q, S};
    for (const void* p : all)
        if ((uintptr_t)p % 16) return DFK_ERR_ALIGNMENT;
    const size_t n = (size_t)M * d_model, es = elt_bytes(dtype);
    // H_out may be H or delta itself: each element is read and then written by one thread
    const Span outs[] = {{N, n * es}, {Q, mx_data_bytes(n, (int)mx)}, {S, n / kMxBlock}};
    const Span ins[] = {{H, n * es}, {delta, n * es}, {norm_weight, (size_t)d_model * es}, {H_out, n * es}};
    if (any_overlap(outs, ins)) return DFK_ERR_ALIAS;
    const Span h{H_out, n * es};
    if ((H_out != H && h.hits(ins[0])) || (H_out != delta && h.hits(ins[1])) || h.hits(ins[2])) return DFK_ERR_ALIAS;
    AddNormArgs a{H, delta, norm_weight, H_out, N, (unsigned char*)Q, (unsigned char*)S, eps, M, d_model, (int)mx};
    const hipError_t e = launch_add_rmsnorm(a, dtype, (hipStream_t)stream);
    return e == hipSuccess ? DFK_OK : hip_fail(e);
}

dfk_status_t dfk_mx_linear(const void* Xq, const void* Xs, dfk_mx_t x_mx, const void* Wq, const void* Ws, const void* bias, const void* residual, void* Y,
                           int M, int n_out, int n_in, dfk_dtype_t dtype, dfk_dtype_t out_dtype, dfk_act_t act,
                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!Xq || !Xs || !Wq || !Ws || !Y || M < 1 || n_out < 1 || n_in < 1 || !known_mx((int)x_mx)) return DFK_ERR_INVALID_ARG;
    if ((dtype != DFK_BF16 && dtype != DFK_FP16) || (out_dtype != dtype && out_dtype != DFK_FP32)) return DFK_ERR_INVALID_ARG;
    if ((int)act < DFK_ACT_NONE || (int)act > DFK_ACT_SILU) return DFK_ERR_INVALID_ARG;
    if (!mx_linear_shape(M, n_out, n_in)) return DFK_ERR_UNSUPPORTED_SHAPE;
    const size_t es = elt_bytes(dtype), os = elt_bytes(out_dtype);
    if ((uintptr_t)Xq % 16 || (uintptr_t)Xs % 16 || (uintptr_t)Wq % 16 || (uintptr_t)Ws % 16 || (uintptr_t)bias % es || (uintptr_t)residual % os ||
        (uintptr_t)Y % os || (uintptr_t)workspace % 256)
        return DFK_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < mx_workspace(M, n_out)) return DFK_ERR_WORKSPACE;
    const size_t nx = (size_t)M * n_in, nw = (size_t)n_out * n_in, ny = (size_t)M * n_out * os;
    const Span outs[] = {{Y, ny}, {workspace, workspace_bytes}};
    const Span ins[] = {{Xq, mx_data_bytes(nx, (int)x_mx)}, {Xs, nx / kMxBlock}, {Wq, nw / 2}, {Ws, nw / kMxBlock}, {bias, n_out * es}};
    if (any_overlap(outs, ins)) return DFK_ERR_ALIAS;
    const Span r{residual, ny};
    if (outs[1].hits(r) || (residual != Y && outs[0].hits(r))) return DFK_ERR_ALIAS;

    MxArgs a{};
    a.t.A = Xq; a.t.B = Wq; a.t.out = Y; a.t.bias = bias; a.t.resid = residual;
    a.t.M = M; a.t.N = n_out; a.t.K = n_in; a.t.act = (int)act;
    a.t.out_fp32 = out_dtype == DFK_FP32; a.t.splits = 1;
    a.t.partial = (float*)workspace; a.t.partial_bytes = workspace_bytes; a.t.pitch = (n_out + 3) / 4 * 4;
    a.t.vec4 = n_out % 4 == 0 && (uintptr_t)Y % (4 * os) == 0 && (uintptr_t)residual % (4 * os) == 0 && (uintptr_t)bias % (4 * es) == 0;
    a.As = (const unsigned char*)Xs; a.Bs = (const unsigned char*)Ws;
    a.dtype = (int)dtype; a.out_mx = -1;
    const hipError_t e = by_launch(a, (int)x_mx, n_out * os, [&](MxArgs& b) {
        const MxPlan p = mx_plan(b.t.M, n_out, n_in, x_mx == DFK_MXFP8, false, b.t.out_fp32);
        b.t.splits = p.splits;
        return p.form >= 0 ? launch_mx_linear_stream(b, (int)x_mx, p.form, (hipStream_t)stream) : launch_mx_linear_tile(b, (int)x_mx, p.tile, (hipStream_t)stream);
    });
    return e == hipSuccess ? DFK_OK : hip_fail(e);
}

size_t dfk_mx_linear_workspace_bytes(int M_max, int n_out, int n_in) { return mx_linear_shape(M_max, n_out, n_in) ? mx_workspace(M_max, n_out) : 0; }

dfk_status_t dfk_mx_gateup(const void* Xq, const void* Xs, dfk_mx_t x_mx, const void* Wg_q, const void* Wg_s, const void* Wu_q, const void* Wu_s,
                           void* A2, dfk_dtype_t dtype, void* A2_q, void* A2_s, dfk_mx_t out_mx, int M, int d_model, int d_ff,
                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!Xq || !Xs || !Wg_q || !Wg_s || !Wu_q || !Wu_s || M < 1 || d_model < 1 || d_ff < 1 || !known_mx((int)x_mx)) return DFK_ERR_INVALID_ARG;
    if ((A2 != nullptr) == (A2_q != nullptr) || (A2_q != nullptr) != (A2_s != nullptr)) return DFK_ERR_INVALID_ARG;
    if (A2 ? (dtype != DFK_BF16 && dtype != DFK_FP16) : !known_mx((int)out_mx)) return DFK_ERR_INVALID_ARG;
    if (!mx_gateup_shape(M, d_ff, d_model)) return DFK_ERR_UNSUPPORTED_SHAPE;
    const void* all[] = {Xq, Xs, Wg_q, Wg_s, Wu_q, Wu_s, A2, A2_q, A2_s};
    for (const void* p : all)
        if ((uintptr_t)p % 16) return DFK_ERR_ALIGNMENT;
    if ((uintptr_t)workspace % 256) return DFK_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < kMxGateupWorkspace) return DFK_ERR_WORKSPACE;
    const size_t nx = (size_t)M * d_model, nw = (size_t)d_ff * d_model, ny = (size_t)M * d_ff;
    const Span outs[] = {{A2, ny * 2}, {A2_q, mx_data_bytes(ny, (int)out_mx)}, {A2_s, ny / kMxBlock}, {workspace, workspace_bytes}};
    const Span ins[] = {{Xq, mx_data_bytes(nx, (int)x_mx)}, {Xs, nx / kMxBlock}, {Wg_q, nw / 2}, {Wg_s, nw / kMxBlock}, {Wu_q, nw / 2}, {Wu_s, nw / kMxBlock}};
    if (any_overlap(outs, ins)) return DFK_ERR_ALIAS;

    MxArgs a{};
    a.t.A = Xq; a.t.B = Wg_q; a.t.B2 = Wu_q; a.t.out = A2;
    a.t.M = M; a.t.N = d_ff; a.t.K = d_model; a.t.splits = 1; a.t.vec4 = 1; a.t.pitch = d_ff;
    a.t.partial = (float*)workspace; a.t.partial_bytes = workspace_bytes;
    a.As = (const unsigned char*)Xs; a.Bs = (const unsigned char*)Wg_s; a.B2s = (const unsigned char*)Wu_s;
    a.dtype = (int)dtype; a.out_mx = A2 ? -1 : (int)out_mx; a.q = (unsigned char*)A2_q; a.qs = (unsigned char*)A2_s;
    const size_t row = A2 ? (size_t)d_ff * 2 : mx_data_bytes((size_t)d_ff, (int)out_mx);
    const hipError_t e = by_launch(a, (int)x_mx, row, [&](MxArgs& b) {
        const MxPlan p = mx_plan(b.t.M, d_ff, d_model, x_mx == DFK_MXFP8, true, false);
        return p.form >= 0 ? launch_mx_gateup_stream(b, (int)x_mx, p.form, (hipStream_t)stream) : launch_mx_gateup_tile(b, (int)x_mx, p.tile, (hipStream_t)stream);
    });
    return e == hipSuccess ? DFK_OK : hip_fail(e);
}

size_t dfk_mx_gateup_workspace_bytes(int M_max, int d_ff, int d_model) { return mx_gateup_shape(M_max, d_ff, d_model) ? kMxGateupWorkspace : 0; }

}  // extern "C"
