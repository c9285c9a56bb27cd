// C ABI of the operators of rotary, gated transformer blocks: checks of the arguments, then the launches of norm.hip, rotary.hip and
// ffn.hip.
#include <cmath>

#include "free_internal.h"

using namespace freemi;

namespace {

bool known(int32_t dtype) { return dtype == FREE_FP32 || dtype == FREE_BF16; }

bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int32_t check_workspace(const void* ws, size_t have, size_t need) {
    return !ws || !aligned(ws, 256) || have < need ? FREE_ERR_WORKSPACE : FREE_OK;
}

// what all four entry points of the layer norm check
int32_t check_norm(int32_t M, int32_t D, int32_t rows_per_sample, float eps, const float* vec, int32_t stride) {
    if (M < 0 || D < 1 || rows_per_sample < 1) return FREE_ERR_SHAPE;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return FREE_ERR_RANGE;
    if (!norm_covers(D)) return FREE_ERR_LIMIT;
    if (vec && M > rows_per_sample && stride < D) return FREE_ERR_SHAPE;
    return FREE_OK;
}

}  // namespace

extern "C" {

int32_t free_op_layer_norm(const void* x, int32_t x_dtype, const float* weight, const float* bias, int32_t wb_stride, int32_t plus_one,
                           float eps, int32_t M, int32_t D, int32_t rows_per_sample, int32_t dtype, void* out, void* stream) {
    if (!known(x_dtype) || !known(dtype)) return FREE_ERR_DTYPE;
    const int32_t st = check_norm(M, D, rows_per_sample, eps, weight ? weight : bias, wb_stride);
    if (st != FREE_OK) return st;
    if (M > 0 && (!x || !out)) return FREE_ERR_NULL;
    return launch_norm_forward(x, x_dtype, weight, bias, wb_stride, plus_one != 0, eps, M, D, rows_per_sample, dtype, out,
                               static_cast<hipStream_t>(stream));
}

size_t free_layer_norm_backward_workspace_bytes(int32_t M, int32_t D, int32_t rows_per_sample) {
    if (M < 0 || D < 1 || rows_per_sample < 1 || !norm_covers(D)) return 0;
    return norm_backward_workspace_bytes(M, D, rows_per_sample);
}

int32_t free_op_layer_norm_backward(const void* dout, int32_t dtype, const void* x, int32_t x_dtype, const float* weight,
                                    int32_t w_stride, int32_t plus_one, float eps, int32_t M, int32_t D, int32_t rows_per_sample,
                                    void* dx, float* dweight, float* dbias, int32_t grad_stride, void* workspace, size_t ws_bytes,
                                    void* stream) {
    if (!known(x_dtype) || !known(dtype)) return FREE_ERR_DTYPE;
    int32_t st = check_norm(M, D, rows_per_sample, eps, weight, w_stride);
    if (st == FREE_OK) st = check_norm(M, D, rows_per_sample, eps, dweight, grad_stride);
    if (st != FREE_OK) return st;
    if ((M > 0 && (!dout || !x || !dx)) || !dweight != !dbias) return FREE_ERR_NULL;
    if (dweight) {
        st = check_workspace(workspace, ws_bytes, norm_backward_workspace_bytes(M, D, rows_per_sample));
        if (st != FREE_OK) return st;
    }
    return launch_norm_backward(dout, dtype, x, x_dtype, weight, w_stride, plus_one != 0, eps, M, D, rows_per_sample, dx, dweight, dbias,
                                grad_stride, workspace, static_cast<hipStream_t>(stream));
}

int32_t free_op_rope_axes(const void* x, int64_t x_stride, const int32_t* pos, int32_t pos_rows, int32_t rows, int32_t heads, int32_t dh,
                          int32_t axes, const int32_t* axis_dims, double theta, int32_t pairing, int32_t inverse, int32_t dtype,
                          void* out, int64_t out_stride, void* stream) {
    if (!axis_dims) return FREE_ERR_NULL;
    if (!known(dtype)) return FREE_ERR_DTYPE;
    if (pairing != FREE_ROPE_PAIRS && pairing != FREE_ROPE_HALVES) return FREE_ERR_RANGE;
    if (!(theta >= 1.0) || !std::isfinite(theta)) return FREE_ERR_RANGE;
    if (rows < 0 || heads < 1 || !rope_covers(dh, axes, axis_dims)) return FREE_ERR_SHAPE;
    if (rows == 0) return FREE_OK;
    if (!x || !pos || !out) return FREE_ERR_NULL;
    const int64_t width = static_cast<int64_t>(heads) * dh;
    if (pos_rows < 1 || (rows > 1 && (x_stride < width || out_stride < width)) || (x == out && rows > 1 && x_stride != out_stride))
        return FREE_ERR_SHAPE;
    return launch_rope(x, x_stride, pos, pos_rows, rows, heads, dh, axes, axis_dims, theta, pairing == FREE_ROPE_PAIRS, inverse != 0, dtype,
                       out, out_stride, static_cast<hipStream_t>(stream));
}

static int32_t check_ffn(int32_t M, int32_t D, int32_t F, int32_t dtype, int32_t act) {
    if (!known(dtype)) return FREE_ERR_DTYPE;
    if (act != FREE_ACT_SILU && act != FREE_ACT_GELU) return FREE_ERR_RANGE;
    if (M < 0 || D < 1 || F < 1) return FREE_ERR_SHAPE;
    return ffn_covers(M, D, F, dtype) ? FREE_OK : FREE_ERR_LIMIT;
}

size_t free_gated_ffn_saved_bytes(int32_t M, int32_t D, int32_t F, int32_t dtype) {
    return check_ffn(M, D, F, dtype, FREE_ACT_SILU) == FREE_OK ? ffn_saved_bytes(M, D, F, dtype) : 0;
}

size_t free_gated_ffn_workspace_bytes(int32_t M, int32_t D, int32_t F, int32_t dtype, int32_t backward) {
    return check_ffn(M, D, F, dtype, FREE_ACT_SILU) == FREE_OK ? ffn_workspace_bytes(M, D, F, dtype, backward != 0) : 0;
}

int32_t free_op_gated_ffn(const void* x, const void* w_in, const void* w_out, int32_t M, int32_t D, int32_t F, int32_t dtype, int32_t act,
                          void* out, void* saved, size_t saved_bytes, void* workspace, size_t ws_bytes, void* stream) {
    int32_t st = check_ffn(M, D, F, dtype, act);
    if (st != FREE_OK) return st;
    if (M == 0) return FREE_OK;
    if (!x || !w_in || !w_out || !out) return FREE_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w_in, 16) || !aligned(w_out, 16) || !aligned(out, 16)) return FREE_ERR_SHAPE;
    if (saved && (!aligned(saved, 256) || saved_bytes < ffn_saved_bytes(M, D, F, dtype))) return FREE_ERR_WORKSPACE;
    st = check_workspace(workspace, ws_bytes, ffn_forward_bytes(M, D, F, dtype, saved != nullptr));
    if (st != FREE_OK) return st;
    return launch_ffn_forward(x, w_in, w_out, M, D, F, dtype, act, out, saved, workspace, static_cast<hipStream_t>(stream));
}

int32_t free_op_gated_ffn_backward(const void* dout, const void* x, const void* w_in, const void* w_out, const void* saved,
                                   size_t saved_bytes, int32_t M, int32_t D, int32_t F, int32_t dtype, int32_t act, void* dx, void* dw_in,
                                   void* dw_out, void* workspace, size_t ws_bytes, void* stream) {
    int32_t st = check_ffn(M, D, F, dtype, act);
    if (st != FREE_OK) return st;
    if (!w_in || !w_out || !dw_in || !dw_out || (M > 0 && (!dout || !x || !dx))) return FREE_ERR_NULL;
    for (const void* p : {dout, x, w_in, w_out, static_cast<const void*>(dx), static_cast<const void*>(dw_in), static_cast<const void*>(dw_out)})
        if (!aligned(p, 16)) return FREE_ERR_SHAPE;
    if (M > 0 && (!saved || !aligned(saved, 256) || saved_bytes < ffn_saved_bytes(M, D, F, dtype))) return FREE_ERR_WORKSPACE;
    st = check_workspace(workspace, ws_bytes, ffn_workspace_bytes(M, D, F, dtype, true));
    if (st != FREE_OK) return st;
    return launch_ffn_backward(dout, x, w_in, w_out, saved, M, D, F, dtype, act, dx, dw_in, dw_out, workspace,
                               static_cast<hipStream_t>(stream));
}

}  // extern "C"
