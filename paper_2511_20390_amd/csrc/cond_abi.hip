// C ABI of the operators of conditioned blocks: checks of the arguments, then the launches of cross_attn.hip, cross_attn_grad.hip and
// adapters.hip.
#include <algorithm>
#include <cmath>

#include "cross_attn.h"

using namespace freemi;

namespace {

bool known(int32_t dtype) { return dtype == FREE_FP32 || dtype == FREE_BF16; }

bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int32_t check_workspace(const void* ws, size_t have, size_t need) {
    return !ws || !aligned(ws, 256) || have < need ? FREE_ERR_WORKSPACE : FREE_OK;
}

constexpr int64_t kMaxStride = 1 << 22;          // 32-bit byte offsets within a tile of rows

int32_t check_cross_sizes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype) {
    if (!known(dtype)) return FREE_ERR_DTYPE;
    if (B < 0 || Nq < 0 || Nk < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0 || dh < 1) return FREE_ERR_SHAPE;
    const int64_t pairs = static_cast<int64_t>(B) * kv_heads, rows = static_cast<int64_t>(Nq) * (heads / kv_heads);
    if (dh > 128 || static_cast<int64_t>(heads) * dh > kMaxStride || rows > 0x7fffffff - 128 || Nk > 0x7fffffff - 128) return FREE_ERR_LIMIT;
    // (workgroups of 512 threads, 2^32 threads to a launch; blocks alone are up to 2^26)
    const int64_t most = std::max({rows, static_cast<int64_t>(Nk), int64_t{1}});
    return pairs >= 1 << 23 || pairs * ((most + 31) / 32) >= 1 << 23 ? FREE_ERR_LIMIT : FREE_OK;
}

bool element_aligned(const void* p, int32_t dtype) { return aligned(p, dtype == FREE_BF16 ? 2 : 4); }

// rows of `width` values, `n` of them
int32_t check_rows(const void* p, int64_t stride, int64_t n, int64_t width, int32_t dtype) {
    if (n > 0 && !p) return FREE_ERR_NULL;
    if (!element_aligned(p, dtype) || (n > 1 && stride < width)) return FREE_ERR_SHAPE;
    return n > 1 && stride > kMaxStride ? FREE_ERR_LIMIT : FREE_OK;
}

#define FREE_CHECK(call)                  \
    do {                                  \
        const int32_t st_ = (call);       \
        if (st_ != FREE_OK) return st_;   \
    } while (0)

}  // namespace

extern "C" {

size_t free_cross_attention_workspace_bytes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype,
                                            int32_t backward) {
    if (check_cross_sizes(B, Nq, Nk, heads, kv_heads, dh, dtype) != FREE_OK) return 0;
    const size_t forward = cross_forward_bytes(B, Nq, Nk, heads, kv_heads, dh, dtype);
    return backward ? std::max(forward, cross_backward_bytes(B, Nq, Nk, heads, kv_heads, dh, dtype)) : forward;
}

int32_t free_op_cross_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                const int32_t* key_len, const uint8_t* key_mask, int32_t B, int32_t Nq, int32_t Nk, int32_t heads,
                                int32_t kv_heads, int32_t dh, float scale, int32_t dtype, void* out, int64_t out_stride, float* lse,
                                void* workspace, size_t ws_bytes, void* stream) {
    FREE_CHECK(check_cross_sizes(B, Nq, Nk, heads, kv_heads, dh, dtype));
    if (!(scale >= 0x1p-64f && scale <= 0x1p64f)) return FREE_ERR_RANGE;
    const int64_t nq = static_cast<int64_t>(B) * Nq, nk = static_cast<int64_t>(B) * Nk, wq = static_cast<int64_t>(heads) * dh, wk = static_cast<int64_t>(kv_heads) * dh;
    if (nq == 0) return FREE_OK;
    FREE_CHECK(check_rows(q, q_stride, nq, wq, dtype));
    FREE_CHECK(check_rows(out, out_stride, nq, wq, dtype));
    FREE_CHECK(check_rows(k, k_stride, nk, wk, dtype));
    FREE_CHECK(check_rows(v, v_stride, nk, wk, dtype));
    if (!aligned(lse, 4) || !aligned(key_len, 4)) return FREE_ERR_SHAPE;
    FREE_CHECK(check_workspace(workspace, ws_bytes, cross_forward_bytes(B, Nq, Nk, heads, kv_heads, dh, dtype)));
    CrossArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_stride = q_stride;
    a.k_stride = nk > 1 ? k_stride : wk;         // (the distance to a next row that there is not)
    a.v_stride = nk > 1 ? v_stride : wk;
    a.key_len = key_len;
    a.key_mask = key_mask;
    a.B = B;
    a.Nq = Nq;
    a.Nk = Nk;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.dh = dh;
    a.scale = scale;
    a.out = out;
    a.out_stride = out_stride;
    a.lse = lse;
    return launch_cross_forward(a, dtype, workspace, static_cast<hipStream_t>(stream));
}

int32_t free_op_cross_attention_backward(const void* dout, int64_t dout_stride, const void* q, int64_t q_stride, const void* k,
                                         int64_t k_stride, const void* v, int64_t v_stride, const void* out, int64_t out_stride,
                                         const float* lse, const int32_t* key_len, const uint8_t* key_mask, int32_t B, int32_t Nq,
                                         int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, float scale, int32_t dtype, void* dq,
                                         int64_t dq_stride, void* dk, int64_t dk_stride, void* dv, int64_t dv_stride, void* workspace,
                                         size_t ws_bytes, void* stream) {
    FREE_CHECK(check_cross_sizes(B, Nq, Nk, heads, kv_heads, dh, dtype));
    if (!(scale >= 0x1p-64f && scale <= 0x1p64f)) return FREE_ERR_RANGE;
    const int64_t nq = static_cast<int64_t>(B) * Nq, nk = static_cast<int64_t>(B) * Nk, wq = static_cast<int64_t>(heads) * dh, wk = static_cast<int64_t>(kv_heads) * dh;
    if (nq == 0 && nk == 0) return FREE_OK;
    FREE_CHECK(check_rows(q, q_stride, nq, wq, dtype));
    FREE_CHECK(check_rows(dout, dout_stride, nq, wq, dtype));
    FREE_CHECK(check_rows(out, out_stride, nq, wq, dtype));
    FREE_CHECK(check_rows(dq, dq_stride, nq, wq, dtype));
    FREE_CHECK(check_rows(k, k_stride, nk, wk, dtype));
    FREE_CHECK(check_rows(v, v_stride, nk, wk, dtype));
    FREE_CHECK(check_rows(dk, dk_stride, nk, wk, dtype));
    FREE_CHECK(check_rows(dv, dv_stride, nk, wk, dtype));
    if (nq > 0 && !lse) return FREE_ERR_NULL;
    if (!aligned(lse, 4) || !aligned(key_len, 4)) return FREE_ERR_SHAPE;
    FREE_CHECK(check_workspace(workspace, ws_bytes, cross_backward_bytes(B, Nq, Nk, heads, kv_heads, dh, dtype)));
    CrossArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_stride = nq > 1 ? q_stride : wq;
    a.k_stride = nk > 1 ? k_stride : wk;
    a.v_stride = nk > 1 ? v_stride : wk;
    a.key_len = key_len;
    a.key_mask = key_mask;
    a.B = B;
    a.Nq = Nq;
    a.Nk = Nk;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.dh = dh;
    a.scale = scale;
    a.out = const_cast<void*>(out);
    a.out_stride = out_stride;
    a.lse = const_cast<float*>(lse);
    a.dout = dout;
    a.dout_stride = nq > 1 ? dout_stride : wq;
    a.dq = dq;
    a.dq_stride = dq_stride;
    a.dk = dk;
    a.dk_stride = dk_stride;
    a.dv = dv;
    a.dv_stride = dv_stride;
    return launch_cross_backward(a, dtype, workspace, static_cast<hipStream_t>(stream));
}

static int32_t check_adapters(int32_t M, int32_t K, int32_t N, int32_t r, int32_t n, int32_t rows_per_sample, int32_t dtype) {
    if (!known(dtype)) return FREE_ERR_DTYPE;
    if (M < 0 || K < 1 || N < 1 || r < 1 || n < 1 || rows_per_sample < 1) return FREE_ERR_SHAPE;
    return adapters_cover(M, K, N, r, n, dtype) ? FREE_OK : FREE_ERR_LIMIT;
}

size_t free_linear_adapters_saved_bytes(int32_t M, int32_t r, int32_t dtype) {
    return check_adapters(M, 1, 1, r, 1, 1, dtype) == FREE_OK ? adapters_saved_bytes(M, r, dtype) : 0;
}

size_t free_linear_adapters_workspace_bytes(int32_t M, int32_t K, int32_t N, int32_t r, int32_t n, int32_t dtype, int32_t backward) {
    return check_adapters(M, K, N, r, n, 1, dtype) == FREE_OK ? adapters_workspace_bytes(M, K, N, r, n, dtype, backward != 0) : 0;
}

int32_t free_op_linear_adapters(const void* x, const void* W, const float* bias, const void* A, const void* B, const float* scale,
                                const int32_t* adapter, int32_t rows_per_sample, int32_t M, int32_t K, int32_t N, int32_t r, int32_t n,
                                int32_t dtype, void* out, void* saved, size_t saved_bytes, void* workspace, size_t ws_bytes, void* stream) {
    FREE_CHECK(check_adapters(M, K, N, r, n, rows_per_sample, dtype));
    if (M == 0) return FREE_OK;
    if (!x || !W || !A || !B || !adapter || !out) return FREE_ERR_NULL;
    if (!aligned(x, 16) || !aligned(W, 16) || !aligned(out, 16) || !element_aligned(A, dtype) || !element_aligned(B, dtype) || !aligned(bias, 4) ||
        !aligned(scale, 4) || !aligned(adapter, 4))
        return FREE_ERR_SHAPE;
    if (saved && (!aligned(saved, 256) || saved_bytes < adapters_saved_bytes(M, r, dtype))) return FREE_ERR_WORKSPACE;
    FREE_CHECK(check_workspace(workspace, ws_bytes, adapters_workspace_bytes(M, K, N, r, n, dtype, false)));
    AdapterArgs a{x, W, A, B, bias, scale, adapter, rows_per_sample, saved, out, nullptr, nullptr, nullptr, nullptr};
    return launch_adapters_forward(a, M, K, N, r, n, dtype, workspace, static_cast<hipStream_t>(stream));
}

int32_t free_op_linear_adapters_backward(const void* dout, const void* x, const void* W, const void* A, const void* B, const float* scale,
                                         const int32_t* adapter, int32_t rows_per_sample, const void* saved, size_t saved_bytes, int32_t M,
                                         int32_t K, int32_t N, int32_t r, int32_t n, int32_t dtype, void* dx, void* dA, void* dB,
                                         void* workspace, size_t ws_bytes, void* stream) {
    FREE_CHECK(check_adapters(M, K, N, r, n, rows_per_sample, dtype));
    if (!W || !A || !B || !dA || !dB || (M > 0 && (!dout || !x || !dx || !adapter))) return FREE_ERR_NULL;
    if (!aligned(dout, 16) || !aligned(x, 16) || !aligned(W, 16) || !aligned(dx, 16)) return FREE_ERR_SHAPE;
    for (const void* p : {A, B, static_cast<const void*>(dA), static_cast<const void*>(dB)})
        if (!element_aligned(p, dtype)) return FREE_ERR_SHAPE;
    if (!aligned(scale, 4) || !aligned(adapter, 4)) return FREE_ERR_SHAPE;
    if (M > 0 && (!saved || !aligned(saved, 256) || saved_bytes < adapters_saved_bytes(M, r, dtype))) return FREE_ERR_WORKSPACE;
    FREE_CHECK(check_workspace(workspace, ws_bytes, adapters_workspace_bytes(M, K, N, r, n, dtype, true)));
    AdapterArgs a{x, W, A, B, nullptr, scale, adapter, rows_per_sample, const_cast<void*>(saved), nullptr, dout, dx, dA, dB};
    return launch_adapters_backward(a, M, K, N, r, n, dtype, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
