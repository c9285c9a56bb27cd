// Gated feed-forward block of a token row x [D], with w_in [2 F, D] (gate rows, then up rows) and w_out [D, F]:
//   [g | u] = x w_in^T,   h = act(g) u,   y = h w_out^T
// and its gradient:
//   dh = dy w_out,  dg = dh u act'(g),  du = dh act(g),
//   dx = [dg | du] w_in,  dw_in = [dg | du]^T x,  dw_out = dy^T h.
// g and u stay fp32 from the sums to the activation and, for the gradient, in the saved state; h, dg and du are rounded to the type of
// the block once, as operands of the next product.
#include <algorithm>

#include "free_internal.h"

namespace freemi {

namespace {

constexpr int kThreads = 256;

// act(v) and its derivative
__device__ __forceinline__ void act_of(float v, int act, float* f, float* df) {
    if (act == FREE_ACT_SILU) {
        const float sg = 1.0f / (1.0f + expf(-v));
        *f = v * sg;
        *df = sg * (1.0f + v * (1.0f - sg));
    } else {
        const float k = 0.7978845608028654f;
        const float t = tanhf(k * (v + 0.044715f * v * v * v));
        *f = 0.5f * v * (1.0f + t);
        *df = 0.5f * (1.0f + t) + 0.5f * v * (1.0f - t * t) * k * (1.0f + 3.0f * 0.044715f * v * v);
    }
}

// C[m, n] = sum_k A(m, k) B(n, k), element strides of both given: any layout, any size.  64 x 64 tile, 4 x 4 outputs per thread.
template <typename TA, typename TB, typename TC>
__global__ __launch_bounds__(kThreads) void product_kernel(const TA* A, int64_t am, int64_t ak, const TB* B, int64_t bn, int64_t bk,
                                                           int32_t M, int32_t N, int32_t K, TC* C) {
    constexpr int BM = 64, BK = 16;
    __shared__ float sA[BK][BM + 4], sB[BK][BM + 4];
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int tiles_n = (N + BM - 1) / BM;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x / tiles_n) * BM, n0 = static_cast<int64_t>(blockIdx.x % tiles_n) * BM;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += BK) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = threadIdx.x + kThreads * i, r = e / BK, kk = e % BK;
            const int64_t gm = m0 + r, gn = n0 + r, gk = k0 + kk;
            sA[kk][r] = gm < M && gk < K ? load_f(A + gm * am + gk * ak) : 0.f;
            sB[kk][r] = gn < N && gk < K ? load_f(B + gn * bn + gk * bk) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < BK; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sA[kk][ty * 4 + i], sB[kk][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t gm = m0 + ty * 4 + i, gn = n0 + tx * 4 + j;
            if (gm < M && gn < N) store_f(C + gm * N + gn, acc[i][j]);
        }
}

// h = act(g) u
template <typename T>
__global__ __launch_bounds__(kThreads) void gate_kernel(const float* gu, int64_t total, int32_t F, int32_t act, T* h) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t m = i / F;
        const float* row = gu + m * 2 * F + (i - m * F);
        float f, df;
        act_of(row[0], act, &f, &df);
        store_f(h + i, f * row[F]);
    }
}

// [dg | du] of dh
template <typename T>
__global__ __launch_bounds__(kThreads) void gate_backward_kernel(const float* gu, const float* dh, int64_t total, int32_t F, int32_t act, T* dgu) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t m = i / F, at = m * 2 * F + (i - m * F);
        float f, df;
        act_of(gu[at], act, &f, &df);
        store_f(dgu + at, dh[i] * gu[at + F] * df);
        store_f(dgu + at + F, dh[i] * f);
    }
}

template <typename TA, typename TB, typename TC>
int32_t product(const TA* A, int64_t am, int64_t ak, const TB* B, int64_t bn, int64_t bk, int32_t M, int32_t N, int32_t K, TC* C, hipStream_t s) {
    const int64_t tiles = static_cast<int64_t>((M + 63) / 64) * ((N + 63) / 64);
    if (tiles > (1 << 22)) return FREE_ERR_LIMIT;
    hipLaunchKernelGGL((product_kernel<TA, TB, TC>), dim3(static_cast<uint32_t>(tiles)), dim3(kThreads), 0, s, A, am, ak, B, bn, bk, M, N, K, C);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

int elementwise_blocks(int64_t total) { return static_cast<int>(std::min<int64_t>((total + kThreads - 1) / kThreads, 8192)); }

size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }

template <typename T>
int32_t forward_of(const T* x, const T* w_in, const T* w_out, int32_t M, int32_t D, int32_t F, int32_t act, T* out, char* keep, hipStream_t s) {
    float* gu = reinterpret_cast<float*>(keep);
    T* h = reinterpret_cast<T*>(keep + up(static_cast<size_t>(M) * 2 * F * sizeof(float)));
    const int64_t total = static_cast<int64_t>(M) * F;
    int32_t st = product(x, D, 1, w_in, D, 1, M, 2 * F, D, gu, s);
    if (st != FREE_OK) return st;
    hipLaunchKernelGGL(gate_kernel<T>, dim3(elementwise_blocks(total)), dim3(kThreads), 0, s, gu, total, F, act, h);
    if (!launch_ok()) return FREE_ERR_HIP;
    return product(h, F, 1, w_out, F, 1, M, D, F, out, s);
}

template <typename T>
int32_t backward_of(const T* dout, const T* x, const T* w_in, const T* w_out, const char* keep, int32_t M, int32_t D, int32_t F, int32_t act,
                    T* dx, T* dw_in, T* dw_out, char* ws, hipStream_t s) {
    const float* gu = reinterpret_cast<const float*>(keep);
    const T* h = reinterpret_cast<const T*>(keep + up(static_cast<size_t>(M) * 2 * F * sizeof(float)));
    const int64_t total = static_cast<int64_t>(M) * F;
    T* dgu = reinterpret_cast<T*>(ws);
    if (M > 0) {
        float* dh = reinterpret_cast<float*>(ws + up(static_cast<size_t>(M) * 2 * F * sizeof(T)));
        int32_t st = product(dout, D, 1, w_out, 1, F, M, F, D, dh, s);
        if (st != FREE_OK) return st;
        hipLaunchKernelGGL(gate_backward_kernel<T>, dim3(elementwise_blocks(total)), dim3(kThreads), 0, s, gu, dh, total, F, act, dgu);
        if (!launch_ok()) return FREE_ERR_HIP;
        st = product(dgu, 2 * F, 1, w_in, 1, D, M, D, 2 * F, dx, s);
        if (st != FREE_OK) return st;
    }
    int32_t st = product(dgu, 1, 2 * F, x, 1, D, 2 * F, D, M, dw_in, s);
    if (st != FREE_OK) return st;
    return product(dout, 1, D, h, 1, F, D, F, M, dw_out, s);
}

}  // namespace

bool ffn_covers(int32_t M, int32_t D, int32_t F, int32_t dtype) {
    (void)M; (void)dtype;
    return static_cast<int64_t>(F) * 2 < (1ll << 31) && D < (1 << 30);
}

size_t ffn_saved_bytes(int32_t M, int32_t D, int32_t F, int32_t dtype) {
    (void)D;
    const size_t es = dtype == FREE_BF16 ? 2 : 4;
    return up(static_cast<size_t>(M) * 2 * F * sizeof(float)) + up(static_cast<size_t>(M) * F * es) + 256;
}

size_t ffn_workspace_bytes(int32_t M, int32_t D, int32_t F, int32_t dtype, bool backward) {
    const size_t es = dtype == FREE_BF16 ? 2 : 4;
    const size_t forward = ffn_saved_bytes(M, D, F, dtype);
    const size_t back = up(static_cast<size_t>(M) * 2 * F * es) + up(static_cast<size_t>(M) * F * sizeof(float)) + 256;
    return backward ? std::max(forward, back) : forward;
}

int32_t launch_ffn_forward(const void* x, const void* w_in, const void* w_out, int32_t M, int32_t D, int32_t F, int32_t dtype, int32_t act,
                           void* out, void* saved, void* ws, hipStream_t s) {
    if (M == 0) return FREE_OK;
    char* keep = static_cast<char*>(saved ? saved : ws);
    if (dtype == FREE_BF16)
        return forward_of(static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(w_in), static_cast<const bf16_t*>(w_out), M, D, F, act, static_cast<bf16_t*>(out), keep, s);
    return forward_of(static_cast<const float*>(x), static_cast<const float*>(w_in), static_cast<const float*>(w_out), M, D, F, act, static_cast<float*>(out), keep, s);
}

int32_t launch_ffn_backward(const void* dout, const void* x, const void* w_in, const void* w_out, const void* saved, int32_t M, int32_t D,
                            int32_t F, int32_t dtype, int32_t act, void* dx, void* dw_in, void* dw_out, void* ws, hipStream_t s) {
    const char* keep = static_cast<const char*>(saved);
    char* w = static_cast<char*>(ws);
    if (dtype == FREE_BF16)
        return backward_of(static_cast<const bf16_t*>(dout), static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(w_in), static_cast<const bf16_t*>(w_out),
                           keep, M, D, F, act, static_cast<bf16_t*>(dx), static_cast<bf16_t*>(dw_in), static_cast<bf16_t*>(dw_out), w, s);
    return backward_of(static_cast<const float*>(dout), static_cast<const float*>(x), static_cast<const float*>(w_in), static_cast<const float*>(w_out),
                       keep, M, D, F, act, static_cast<float*>(dx), static_cast<float*>(dw_in), static_cast<float*>(dw_out), w, s);
}

}  // namespace freemi
