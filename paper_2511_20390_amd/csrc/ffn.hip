// Gated feed-forward block of a token row x [D], with w_in [2 F, D] (gate rows, then up rows) and w_out [D, F]:
//   [g | u] = x w_in^T,   h = act(g) u,   y = h w_out^T
// and its gradient:
//   dh = dy w_out,  dg = dh u act'(g),  du = dh act(g),
//   dx = [dg | du] w_in,  dw_in = [dg | du]^T x,  dw_out = dy^T h.
// g and u stay fp32 from the sums to the activation and, for the gradient, in the saved state: rounded to bf16 there they would add an
// error of their own to dg and du, three roundings on the way to a gradient in place of two.  h, dg and du are rounded to the type of the
// block once, as operands of the next product.
//
// The products want widths that are multiples of 64 (16-byte rows, whole slices of K).  Other widths go through zero-padded copies in
// the workspace, results through a cropping copy: zeros in D add nothing to a sum, zero rows of w_in give h = 0.
// bf16: ffn_mfma.hip, operands read in either layout.  fp32: the products of three bf16 parts per value of gemm_f32.hip, which want K
// next to each other; the gradient's factors are transposed in the workspace first.
#include <algorithm>

#include "ffn_mfma.h"
#include "free_internal.h"

namespace freemi {

namespace {

constexpr int kThreads = 256;

// act(v) and its derivative
__device__ __forceinline__ void act_of(float v, int act, float* f, float* df) {
    if (act == FREE_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-v));
        *f = v * s;
        *df = s == 0.f || s == 1.f ? s : s * (1.0f + v * (1.0f - s));
    } else {
        const float k = 0.7978845608028654f;
        const float v2 = v * v, t = tanhf(k * (v + 0.044715f * v2 * v));
        *f = 0.5f * v * (1.0f + t);
        // (1 - t^2) times what grows with v^3: 0 where t is one to the last bit
        *df = fabsf(t) == 1.f ? 0.5f * (1.0f + t) : 0.5f * (1.0f + t) + 0.5f * v * (1.0f - t * t) * k * (1.0f + 3.0f * 0.044715f * v2);
    }
}

// fp32: h = act(g) u
__global__ __launch_bounds__(kThreads) void ffn_gate_kernel(const float* gu, int64_t total4, int32_t F, int32_t act, float* h) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total4; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t m = i / (F / 4), c = i - m * (F / 4);
        const float4 g = reinterpret_cast<const float4*>(gu + m * 2 * F)[c], u = reinterpret_cast<const float4*>(gu + m * 2 * F + F)[c];
        float4 f, df;
        act_of(g.x, act, &f.x, &df.x);
        act_of(g.y, act, &f.y, &df.y);
        act_of(g.z, act, &f.z, &df.z);
        act_of(g.w, act, &f.w, &df.w);
        reinterpret_cast<float4*>(h)[i] = make_float4(f.x * u.x, f.y * u.y, f.z * u.z, f.w * u.w);
    }
}

// fp32: [dg | du] of dh
__global__ __launch_bounds__(kThreads) void ffn_gate_grad_kernel(const float* gu, const float* dh, int64_t total4, int32_t F, int32_t act, float* dgu) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total4; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t m = i / (F / 4), c = i - m * (F / 4);
        const float4 g = reinterpret_cast<const float4*>(gu + m * 2 * F)[c], u = reinterpret_cast<const float4*>(gu + m * 2 * F + F)[c];
        const float4 d = reinterpret_cast<const float4*>(dh)[i];
        float4 f, df;
        act_of(g.x, act, &f.x, &df.x);
        act_of(g.y, act, &f.y, &df.y);
        act_of(g.z, act, &f.z, &df.z);
        act_of(g.w, act, &f.w, &df.w);
        reinterpret_cast<float4*>(dgu + m * 2 * F)[c] = make_float4(d.x * u.x * df.x, d.y * u.y * df.y, d.z * u.z * df.z, d.w * u.w * df.w);
        reinterpret_cast<float4*>(dgu + m * 2 * F + F)[c] = make_float4(d.x * f.x, d.y * f.y, d.z * f.z, d.w * f.w);
    }
}

// dst [rows_to, cols_to] = src [rows, cols], cropped or filled with zeros; elements of 2 or 4 bytes
template <typename T>
__global__ __launch_bounds__(kThreads) void ffn_fit_kernel(const T* src, int32_t rows, int32_t cols, T* dst, int32_t rows_to, int32_t cols_to) {
    const int64_t total = static_cast<int64_t>(rows_to) * cols_to;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t r = i / cols_to, c = i - r * cols_to;
        dst[i] = r < rows && c < cols ? src[r * cols + c] : T(0);
    }
}

// dst [cols, rows_to] = src [rows, cols]^T, columns past rows zero; 64 x 64 per workgroup, a tile per blockIdx.x
__global__ __launch_bounds__(kThreads) void ffn_transpose_kernel(const float* src, int32_t rows, int32_t cols, float* dst, int32_t rows_to) {
    __shared__ float t[64][65];
    const int tiles_c = (cols + 63) / 64;
    const int64_t r0 = static_cast<int64_t>(blockIdx.x / tiles_c) * 64, c0 = static_cast<int64_t>(blockIdx.x % tiles_c) * 64;
    const int x = threadIdx.x % 64, y = threadIdx.x / 64;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int64_t r = r0 + y + 4 * k, c = c0 + x;
        t[y + 4 * k][x] = r < rows && c < cols ? src[r * cols + c] : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int64_t c = c0 + y + 4 * k, r = r0 + x;
        if (c < cols && r < rows_to) dst[c * rows_to + r] = t[x][y + 4 * k];
    }
}

constexpr int kMaxBlocks = 1 << 16;

int grid_of(int64_t items) { return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>((items + kThreads - 1) / kThreads, kMaxBlocks))); }

template <typename T>
int32_t fit(const T* src, int32_t rows, int32_t cols, T* dst, int32_t rows_to, int32_t cols_to, hipStream_t s) {
    using U = typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type;
    hipLaunchKernelGGL(ffn_fit_kernel<U>, dim3(grid_of(static_cast<int64_t>(rows_to) * cols_to)), dim3(kThreads), 0, s, reinterpret_cast<const U*>(src),
                       rows, cols, reinterpret_cast<U*>(dst), rows_to, cols_to);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

int32_t transpose(const float* src, int32_t rows, int32_t cols, float* dst, int32_t rows_to, hipStream_t s) {
    const int64_t blocks = static_cast<int64_t>((rows_to + 63) / 64) * ((cols + 63) / 64);
    if (blocks > (1 << 23)) return FREE_ERR_LIMIT;
    hipLaunchKernelGGL(ffn_transpose_kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, s, src, rows, cols, dst, rows_to);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

int32_t up_to(int32_t v, int32_t step) { return (v + step - 1) / step * step; }

// The sizes of a block and where the parts of its saved state and of its workspaces lie
struct Sizes {
    int32_t M, D, F;                 // as given
    int32_t Dp, Fp;                  // as the products have them
    int32_t Mk;                      // rows as a summed dimension of fp32 products
    size_t es;
    bool padded;
    Sizes(int32_t m, int32_t d, int32_t f, int32_t dtype)
        : M(m), D(d), F(f), Dp(up_to(d, 64)), Fp(up_to(f, 64)), Mk(up_to(m, 32)), es(dtype == FREE_BF16 ? 2 : 4), padded(Dp != d || Fp != f) {}
    size_t gu_bytes() const {        // bf16: blocks of 32 x 32 (ffn_mfma.h); fp32: rows [g | u]
        return static_cast<size_t>(es == 2 ? up_to(M, 32) : M) * 2 * Fp * sizeof(float);
    }
    size_t act_bytes(int32_t width) const { return static_cast<size_t>(M) * width * es; }
    size_t weight_bytes(int32_t n) const { return static_cast<size_t>(n) * Dp * Fp * es; }
};

struct Carve {
    char* base;
    size_t at = 0;
    template <typename T>
    T* take(size_t bytes) {
        T* p = reinterpret_cast<T*>(base + at);
        at += (bytes + 255) / 256 * 256;
        return p;
    }
};

// bf16: the products of the two passes
struct ForwardProducts {
    FfnProduct up, down;
    ForwardProducts(const Sizes& z, const bf16_t* x, const bf16_t* w_in, const bf16_t* w_out, int32_t act, bf16_t* y, float* gu, bf16_t* h, bool keep)
        : up{keep ? FFN_GATE_KEEP : FFN_GATE, x, w_in, z.Dp, z.Dp, z.M, z.Fp, z.Dp, h, z.Fp, gu, act},
          down{FFN_ROWS, h, w_out, z.Fp, z.Fp, z.M, z.Dp, z.Fp, y, z.Dp} {}
    size_t room() const { return std::max(ffn_products_part_bytes(&up, 1), ffn_products_part_bytes(&down, 1)); }
};

struct BackwardProducts {
    FfnProduct gate, rows, weights[2];
    BackwardProducts(const Sizes& z, const bf16_t* dy, const bf16_t* x, const bf16_t* w_in, const bf16_t* w_out, float* gu, const bf16_t* h,
                     int32_t act, bf16_t* dgu, bf16_t* dx, bf16_t* dw_in, bf16_t* dw_out)
        : gate{FFN_GATE_GRAD, dy, w_out, z.Dp, z.Fp, z.M, z.Fp, z.Dp, dgu, 2 * z.Fp, gu, act},
          rows{FFN_ROWS_BY_K, dgu, w_in, 2 * z.Fp, z.Dp, z.M, z.Dp, 2 * z.Fp, dx, z.Dp},
          weights{{FFN_K_BY_K, dgu, x, 2 * z.Fp, z.Dp, 2 * z.Fp, z.Dp, z.M, dw_in, z.Dp}, {FFN_K_BY_K, dy, h, z.Dp, z.Fp, z.Dp, z.Fp, z.M, dw_out, z.Fp}} {}
    size_t room() const {
        return std::max({ffn_products_part_bytes(&gate, 1), ffn_products_part_bytes(&rows, 1), ffn_products_part_bytes(weights, 2)});
    }
};

template <typename T>
struct Saved {
    float* gu;
    T* h;
    size_t bytes;
    Saved(const Sizes& z, char* base) {
        Carve c{base};
        gu = c.take<float>(z.gu_bytes());
        h = c.take<T>(z.act_bytes(z.Fp));
        bytes = c.at + 256;
    }
};

template <typename T>
struct ForwardSpace {
    T *x, *w_in, *w_out, *y, *h;
    float *gu, *room;            // room: bf16 the parts of a product, fp32 a bias of zeros
    size_t bytes;
    ForwardSpace(const Sizes& z, char* base) {
        Carve c{base};
        gu = c.take<float>(z.es == 4 ? z.gu_bytes() : 0);
        h = c.take<T>(z.act_bytes(z.Fp));
        room = c.take<float>(z.es == 4 ? sizeof(float) * std::max(2 * z.Fp, z.Dp)
                                       : ForwardProducts(z, nullptr, nullptr, nullptr, 0, nullptr, nullptr, nullptr, false).room());
        x = w_in = w_out = y = nullptr;
        if (z.padded) {
            x = c.take<T>(z.act_bytes(z.Dp));
            w_in = c.take<T>(z.weight_bytes(2));
            w_out = c.take<T>(z.weight_bytes(1));
            y = c.take<T>(z.act_bytes(z.Dp));
        }
        bytes = c.at + 256;
    }
};

template <typename T>
struct BackwardSpace {
    T *dgu, *x, *dy, *w_in, *w_out, *dx, *dw_in, *dw_out;
    float *dh, *room, *t1, *t2;
    size_t bytes;
    BackwardSpace(const Sizes& z, char* base) {
        Carve c{base};
        dgu = c.take<T>(z.act_bytes(2 * z.Fp));
        dh = t1 = t2 = nullptr;
        room = c.take<float>(z.es == 4 ? sizeof(float) * std::max(2 * z.Fp, z.Dp)
                                       : BackwardProducts(z, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr, nullptr, nullptr, nullptr).room());
        if (z.es == 4) {
            dh = c.take<float>(z.act_bytes(z.Fp));
            // transposed factors: a weight, or two of rows Mk
            t1 = c.take<float>(std::max(z.weight_bytes(2), static_cast<size_t>(z.Mk) * std::max(2 * z.Fp, z.Dp) * 4));
            t2 = c.take<float>(static_cast<size_t>(z.Mk) * std::max(z.Fp, z.Dp) * 4);
        }
        x = dy = w_in = w_out = dx = dw_in = dw_out = nullptr;
        if (z.padded) {
            x = c.take<T>(z.act_bytes(z.Dp));
            dy = c.take<T>(z.act_bytes(z.Dp));
            dx = c.take<T>(z.act_bytes(z.Dp));
            w_in = c.take<T>(z.weight_bytes(2));
            w_out = c.take<T>(z.weight_bytes(1));
            dw_in = c.take<T>(z.weight_bytes(2));
            dw_out = c.take<T>(z.weight_bytes(1));
        }
        bytes = c.at + 256;
    }
};

#define FREE_STEP(call)                     \
    do {                                    \
        const int32_t st_ = (call);         \
        if (st_ != FREE_OK) return st_;     \
    } while (0)

template <typename T>
int32_t pad_weights(const Sizes& z, const T* w_in, const T* w_out, T* w_in_p, T* w_out_p, hipStream_t s) {
    FREE_STEP(fit(w_in, z.F, z.D, w_in_p, z.Fp, z.Dp, s));
    FREE_STEP(fit(w_in + static_cast<size_t>(z.F) * z.D, z.F, z.D, w_in_p + static_cast<size_t>(z.Fp) * z.Dp, z.Fp, z.Dp, s));
    return fit(w_out, z.D, z.F, w_out_p, z.Dp, z.Fp, s);
}

int32_t product_f32(const float* X, const float* W, const float* zero, int32_t M, int32_t N, int32_t K, float* out, hipStream_t s) {
    if (!linear_f32_covers(X, W, M, N, K)) return FREE_ERR_LIMIT;
    return launch_linear_f32(X, W, zero, M, N, K, FREE_EPI_BIAS, out, nullptr, RowVec{nullptr, 0, 1}, s);
}

int32_t products_forward(const Sizes& z, const bf16_t* x, const bf16_t* w_in, const bf16_t* w_out, int32_t act, bf16_t* y, float* gu,
                         bf16_t* h, bool keep, float* room, hipStream_t s) {
    const ForwardProducts p(z, x, w_in, w_out, act, y, gu, h, keep);
    FREE_STEP(launch_ffn_products(&p.up, 1, room, s));
    return launch_ffn_products(&p.down, 1, room, s);
}

int32_t products_forward(const Sizes& z, const float* x, const float* w_in, const float* w_out, int32_t act, float* y, float* gu, float* h,
                         bool, float* zero, hipStream_t s) {
    FREE_STEP(fit(x, 0, 0, zero, 1, std::max(2 * z.Fp, z.Dp), s));
    FREE_STEP(product_f32(x, w_in, zero, z.M, 2 * z.Fp, z.Dp, gu, s));
    const int64_t total4 = static_cast<int64_t>(z.M) * z.Fp / 4;
    hipLaunchKernelGGL(ffn_gate_kernel, dim3(grid_of(total4)), dim3(kThreads), 0, s, gu, total4, z.Fp, act, h);
    if (!launch_ok()) return FREE_ERR_HIP;
    return product_f32(h, w_out, zero, z.M, z.Dp, z.Fp, y, s);
}

int32_t products_backward(const Sizes& z, const bf16_t* dy, const bf16_t* x, const bf16_t* w_in, const bf16_t* w_out, const Saved<bf16_t>& kept,
                          int32_t act, const BackwardSpace<bf16_t>& w, bf16_t* dx, bf16_t* dw_in, bf16_t* dw_out, hipStream_t s) {
    const BackwardProducts p(z, dy, x, w_in, w_out, kept.gu, kept.h, act, w.dgu, dx, dw_in, dw_out);
    FREE_STEP(launch_ffn_products(&p.gate, 1, w.room, s));
    FREE_STEP(launch_ffn_products(&p.rows, 1, w.room, s));
    return launch_ffn_products(p.weights, 2, w.room, s);
}

int32_t products_backward(const Sizes& z, const float* dy, const float* x, const float* w_in, const float* w_out, const Saved<float>& kept,
                          int32_t act, const BackwardSpace<float>& w, float* dx, float* dw_in, float* dw_out, hipStream_t s) {
    const int32_t F2 = 2 * z.Fp;
    FREE_STEP(fit(x, 0, 0, w.room, 1, std::max(F2, z.Dp), s));
    FREE_STEP(transpose(w_out, z.Dp, z.Fp, w.t1, z.Dp, s));
    FREE_STEP(product_f32(dy, w.t1, w.room, z.M, z.Fp, z.Dp, w.dh, s));
    const int64_t total4 = static_cast<int64_t>(z.M) * z.Fp / 4;
    hipLaunchKernelGGL(ffn_gate_grad_kernel, dim3(grid_of(total4)), dim3(kThreads), 0, s, kept.gu, w.dh, total4, z.Fp, act, w.dgu);
    if (!launch_ok()) return FREE_ERR_HIP;
    FREE_STEP(transpose(w_in, F2, z.Dp, w.t1, F2, s));
    FREE_STEP(product_f32(w.dgu, w.t1, w.room, z.M, z.Dp, F2, dx, s));
    FREE_STEP(transpose(w.dgu, z.M, F2, w.t1, z.Mk, s));
    FREE_STEP(transpose(x, z.M, z.Dp, w.t2, z.Mk, s));
    FREE_STEP(product_f32(w.t1, w.t2, w.room, F2, z.Dp, z.Mk, dw_in, s));
    FREE_STEP(transpose(dy, z.M, z.Dp, w.t1, z.Mk, s));
    FREE_STEP(transpose(kept.h, z.M, z.Fp, w.t2, z.Mk, s));
    return product_f32(w.t1, w.t2, w.room, z.Dp, z.Fp, z.Mk, dw_out, s);
}

template <typename T>
int32_t forward_of(const Sizes& z, const T* x, const T* w_in, const T* w_out, int32_t act, T* out, char* saved, char* ws, hipStream_t s) {
    ForwardSpace<T> w(z, ws);
    float* gu = w.gu;
    T* h = w.h;
    if (saved) {
        const Saved<T> k(z, saved);
        gu = k.gu;
        h = k.h;
    }
    if (!saved && ffn_rows_pay(z.M, z.D, z.F, z.es == 2 ? FREE_BF16 : FREE_FP32)) return launch_ffn_rows(x, w_in, w_out, z.M, z.D, z.F, act, h, out, s);
    T* y = out;
    if (z.padded) {
        FREE_STEP(fit(x, z.M, z.D, w.x, z.M, z.Dp, s));
        FREE_STEP(pad_weights(z, w_in, w_out, w.w_in, w.w_out, s));
        x = w.x;
        w_in = w.w_in;
        w_out = w.w_out;
        y = w.y;
    }
    FREE_STEP(products_forward(z, x, w_in, w_out, act, y, gu, h, saved != nullptr, w.room, s));
    return z.padded ? fit(y, z.M, z.Dp, out, z.M, z.D, s) : FREE_OK;
}

template <typename T>
int32_t backward_of(const Sizes& z, const T* dout, const T* x, const T* w_in, const T* w_out, char* saved, int32_t act, T* dx, T* dw_in, T* dw_out,
                    char* ws, hipStream_t s) {
    if (z.M == 0) {                                      // empty sums
        FREE_STEP(fit(w_in, 0, 0, dw_in, 2 * z.F, z.D, s));
        return fit(w_out, 0, 0, dw_out, z.D, z.F, s);
    }
    const BackwardSpace<T> w(z, ws);
    const Saved<T> kept(z, saved);
    if (!z.padded) return products_backward(z, dout, x, w_in, w_out, kept, act, w, dx, dw_in, dw_out, s);
    FREE_STEP(fit(x, z.M, z.D, w.x, z.M, z.Dp, s));
    FREE_STEP(fit(dout, z.M, z.D, w.dy, z.M, z.Dp, s));
    FREE_STEP(pad_weights(z, w_in, w_out, w.w_in, w.w_out, s));
    FREE_STEP(products_backward(z, w.dy, w.x, w.w_in, w.w_out, kept, act, w, w.dx, w.dw_in, w.dw_out, s));
    FREE_STEP(fit(w.dx, z.M, z.Dp, dx, z.M, z.D, s));
    FREE_STEP(fit(w.dw_in, z.Fp, z.Dp, dw_in, z.F, z.D, s));
    FREE_STEP(fit(w.dw_in + static_cast<size_t>(z.Fp) * z.Dp, z.Fp, z.Dp, dw_in + static_cast<size_t>(z.F) * z.D, z.F, z.D, s));
    return fit(w.dw_out, z.Dp, z.Fp, dw_out, z.D, z.F, s);
}

}  // namespace

// 32-bit byte offsets inside a tile of 256 rows (fp32: 130 rows as long as all token rows, in the weights' gradients), 32-bit column numbers of [g | u], grids of less than 2^32 threads
bool ffn_covers(int32_t M, int32_t D, int32_t F, int32_t dtype) {
    constexpr int32_t kMost = 1 << 20;
    if (D > kMost || F > kMost || (dtype == FREE_FP32 && M > 4 * kMost - 65536)) return false;
    const int64_t m = (static_cast<int64_t>(M) + 127) / 128, d = (D + 127) / 128, f = (F + 63) / 64;
    return std::max({m * f, m * d, 2 * f * d}) <= 1 << 22;
}

size_t ffn_saved_bytes(int32_t M, int32_t D, int32_t F, int32_t dtype) {
    const Sizes z(M, D, F, dtype);
    return z.es == 2 ? Saved<bf16_t>(z, nullptr).bytes : Saved<float>(z, nullptr).bytes;
}

size_t ffn_workspace_bytes(int32_t M, int32_t D, int32_t F, int32_t dtype, bool backward) {
    const Sizes z(M, D, F, dtype);
    const size_t f = z.es == 2 ? ForwardSpace<bf16_t>(z, nullptr).bytes : ForwardSpace<float>(z, nullptr).bytes;
    const size_t b = z.es == 2 ? BackwardSpace<bf16_t>(z, nullptr).bytes : BackwardSpace<float>(z, nullptr).bytes;
    return backward ? std::max(f, b) : f;
}

int32_t launch_ffn_forward(const void* x, const void* w_in, const void* w_out, int32_t M, int32_t D, int32_t F, int32_t dtype, int32_t act,
                           void* out, void* saved, void* ws, hipStream_t s) {
    const Sizes z(M, D, F, dtype);
    const auto run = [&](auto t) {
        using T = decltype(t);
        return forward_of(z, static_cast<const T*>(x), static_cast<const T*>(w_in), static_cast<const T*>(w_out), act, static_cast<T*>(out),
                          static_cast<char*>(saved), static_cast<char*>(ws), s);
    };
    return dtype == FREE_BF16 ? run(bf16_t{}) : run(float{});
}

int32_t launch_ffn_backward(const void* dout, const void* x, const void* w_in, const void* w_out, const void* saved, int32_t M, int32_t D,
                            int32_t F, int32_t dtype, int32_t act, void* dx, void* dw_in, void* dw_out, void* ws, hipStream_t s) {
    const Sizes z(M, D, F, dtype);
    const auto run = [&](auto t) {
        using T = decltype(t);
        return backward_of(z, static_cast<const T*>(dout), static_cast<const T*>(x), static_cast<const T*>(w_in), static_cast<const T*>(w_out),
                           static_cast<char*>(const_cast<void*>(saved)), act, static_cast<T*>(dx), static_cast<T*>(dw_in), static_cast<T*>(dw_out),
                           static_cast<char*>(ws), s);
    };
    return dtype == FREE_BF16 ? run(bf16_t{}) : run(float{});
}

}  // namespace freemi
