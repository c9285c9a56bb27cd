// Gated feed-forward block of a token row x [D], with w_in [2 F, D] (gate rows, then up rows) and w_out [D, F]:
//   [g | u] = x w_in^T,   h = act(g) u,   y = h w_out^T
// and its gradient:
//   dh = dy w_out,  dg = dh u act'(g),  du = dh act(g),
//   dx = [dg | du] w_in,  dw_in = [dg | du]^T x,  dw_out = dy^T h.
// g and u stay fp32 from the sums to the activation and, for the gradient, in the saved state: rounded to bf16 there they would add an
// error of their own to dg and du, three roundings on the way to a gradient in place of two.  h, dg and du are rounded to the type of the
// block once, as operands of the next product (2-norm error of bf16 results against 64 bits: 2.4e-3, where the result's own rounding makes
// 1.7e-3).
//
// The products want widths that are multiples of 8 (bf16: 16-byte rows) or of 64 (fp32: whole slices of K).  Other widths go through
// zero-padded copies in the workspace, results through a cropping copy: zeros in D add nothing to a sum, zero rows of w_in give h = 0.
// (bf16, 1000 rows of 1152, forward and gradient, us: 2743 hidden values, padded, 177; 2736, not padded, 121; 2752 121.)
// bf16: ffn_mfma.hip; fp32: the products of three bf16 parts per value of gemm_f32.hip.  Both read operands in either layout.  Few rows:
// ffn_rows.hip.
#include <algorithm>

#include "ffn_mfma.h"
#include "free_internal.h"

namespace freemi {

namespace {

constexpr int kThreads = 256;

// dst [rows_to, cols_to] = src [rows, cols], cropped or filled with zeros; elements of 2 or 4 bytes.  A thread has 16 bytes of a row, at
// whatever address; rows over blockIdx.y.
template <typename T>
__global__ __launch_bounds__(kThreads) void ffn_fit_kernel(const T* src, int32_t rows, int32_t cols, T* dst, int32_t rows_to, int32_t cols_to) {
    constexpr int E = 16 / sizeof(T);
    const int c = (blockIdx.x * kThreads + threadIdx.x) * E;
    if (c >= cols_to) return;
    for (int64_t r = blockIdx.y; r < rows_to; r += gridDim.y) {
        const T* from = src + r * cols + c;
        T* to = dst + r * cols_to + c;
        const int n = r < rows ? cols - c : 0, m = cols_to - c;  // values there are, and are wanted, from c on
        T v[E];
        if (n >= E) {
            __builtin_memcpy(v, from, 16);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = e < n ? from[e] : T(0);
        }
        if (m >= E) {
            __builtin_memcpy(to, v, 16);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < m) to[e] = v[e];
        }
    }
}

template <typename T>
int32_t fit(const T* src, int32_t rows, int32_t cols, T* dst, int32_t rows_to, int32_t cols_to, hipStream_t s) {
    using U = typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type;
    const dim3 grid((cols_to + kThreads * 16 / sizeof(T) - 1) / (kThreads * 16 / sizeof(T)), std::min(rows_to, 65535));
    hipLaunchKernelGGL(ffn_fit_kernel<U>, grid, dim3(kThreads), 0, s, reinterpret_cast<const U*>(src), rows, cols, reinterpret_cast<U*>(dst), rows_to,
                       cols_to);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

int32_t up_to(int32_t v, int32_t step) { return (v + step - 1) / step * step; }

// The sizes of a block and where the parts of its saved state and of its workspaces lie
struct Sizes {
    int32_t M, D, F;                 // as given
    int32_t Dp, Fp;                  // as the products have them
    int32_t H;                       // values of a row of h, dg, du
    size_t es;
    bool padded;
    Sizes(int32_t m, int32_t d, int32_t f, int32_t dtype) : M(m), D(d), F(f), Dp(d), Fp(f), H(up_to(f, 64)), es(dtype == FREE_BF16 ? 2 : 4) {
        const int32_t step = es == 2 ? 8 : 64;
        padded = d % step != 0 || f % step != 0;
        if (padded) {
            Dp = up_to(d, 64);
            Fp = H;
        }
    }
    size_t gu_bytes() const { return static_cast<size_t>(up_to(M, 32)) * 2 * H * sizeof(float); }
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

// the products of the two passes
template <typename T>
struct ForwardProducts {
    FfnProduct<T> up, down;
    ForwardProducts(const Sizes& z, const T* x, const T* w_in, const T* w_out, int32_t act, T* y, float* gu, T* h, bool keep)
        : up{keep ? FFN_GATE_KEEP : FFN_GATE, x, w_in, z.Dp, z.Dp, z.M, z.Fp, z.Dp, h, z.H, gu, act, z.H},
          down{FFN_ROWS, h, w_out, z.H, z.Fp, z.M, z.Dp, z.Fp, y, z.Dp} {}
    size_t room() const { return std::max(ffn_products_part_bytes(&up, 1), ffn_products_part_bytes(&down, 1)); }
};

template <typename T>
struct BackwardProducts {
    FfnProduct<T> gate, rows, weights[2];
    BackwardProducts(const Sizes& z, const T* dy, const T* x, const T* w_in, const T* w_out, float* gu, const T* h, int32_t act, T* dgu, T* dx,
                     T* dw_in, T* dw_out)
        : gate{FFN_GATE_GRAD, dy, w_out, z.Dp, z.Fp, z.M, z.Fp, z.Dp, dgu, 2 * z.H, gu, act, z.H},
          rows{FFN_ROWS_BY_K, dgu, w_in, 2 * z.H, z.Dp, z.M, z.Dp, 2 * z.H, dx, z.Dp, nullptr, 0, 0, z.H, z.Fp},
          weights{{FFN_K_BY_K, dgu, x, 2 * z.H, z.Dp, 2 * z.H, z.Dp, z.M, dw_in, z.Dp, nullptr, 0, 0, z.H, z.Fp},
                  {FFN_K_BY_K, dy, h, z.Dp, z.H, z.Dp, z.Fp, z.M, dw_out, z.Fp}} {}
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
        h = c.take<T>(z.act_bytes(z.H));
        bytes = c.at + 256;
    }
};

template <typename T>
struct ForwardSpace {
    T *x, *w_in, *w_out, *y, *h;
    float* room;                     // parts of a product
    size_t bytes;
    ForwardSpace(const Sizes& z, char* base) {
        Carve c{base};
        h = c.take<T>(z.act_bytes(z.H));
        const auto room_of = [&](bool keep) { return ForwardProducts<T>(z, nullptr, nullptr, nullptr, 0, nullptr, nullptr, nullptr, keep).room(); };
        room = c.take<float>(std::max(room_of(false), room_of(true)));
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
    float* room;
    size_t bytes;
    BackwardSpace(const Sizes& z, char* base) {
        Carve c{base};
        dgu = c.take<T>(z.act_bytes(2 * z.H));
        room = c.take<float>(BackwardProducts<T>(z, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr, nullptr, nullptr, nullptr).room());
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

template <typename T>
int32_t products_backward(const Sizes& z, const T* dy, const T* x, const T* w_in, const T* w_out, const Saved<T>& kept, int32_t act,
                          const BackwardSpace<T>& w, T* dx, T* dw_in, T* dw_out, hipStream_t s) {
    const BackwardProducts<T> p(z, dy, x, w_in, w_out, kept.gu, kept.h, act, w.dgu, dx, dw_in, dw_out);
    FREE_STEP(launch_ffn_products(&p.gate, 1, w.room, s));
    FREE_STEP(launch_ffn_products(&p.rows, 1, w.room, s));
    return launch_ffn_products(p.weights, 2, w.room, s);
}

// the way of few rows, which keeps nothing and needs room for h alone
bool few_rows(const Sizes& z, bool keep) { return !keep && ffn_rows_pay(z.M, z.D, z.F, z.padded); }

template <typename T>
int32_t forward_of(const Sizes& z, const T* x, const T* w_in, const T* w_out, int32_t act, T* out, char* saved, char* ws, hipStream_t s) {
    if (few_rows(z, saved != nullptr)) return launch_ffn_rows(x, w_in, w_out, z.M, z.D, z.F, act, reinterpret_cast<T*>(ws), out, s);
    const ForwardSpace<T> w(z, ws);
    float* gu = nullptr;
    T* h = w.h;
    if (saved) {
        const Saved<T> k(z, saved);
        gu = k.gu;
        h = k.h;
    }
    T* y = out;
    if (z.padded) {
        FREE_STEP(fit(x, z.M, z.D, w.x, z.M, z.Dp, s));
        FREE_STEP(pad_weights(z, w_in, w_out, w.w_in, w.w_out, s));
        x = w.x;
        w_in = w.w_in;
        w_out = w.w_out;
        y = w.y;
    }
    const ForwardProducts<T> p(z, x, w_in, w_out, act, y, gu, h, saved != nullptr);
    FREE_STEP(launch_ffn_products(&p.up, 1, w.room, s));
    FREE_STEP(launch_ffn_products(&p.down, 1, w.room, s));
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

// 32-bit byte offsets inside a tile of 256 rows, 32-bit column numbers of [g | u], grids of less than 2^32 threads (fp32: of tiles a quarter
// as large)
bool ffn_covers(int32_t M, int32_t D, int32_t F, int32_t dtype) {
    if (D > 1 << 20 || F > 1 << 20) return false;
    const int64_t m = (static_cast<int64_t>(M) + 127) / 128, d = (D + 127) / 128, f = (F + 63) / 64;
    return std::max({m * f, m * d, 2 * f * d}) <= (dtype == FREE_FP32 ? 1 << 20 : 1 << 22);
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

size_t ffn_forward_bytes(int32_t M, int32_t D, int32_t F, int32_t dtype, bool keep) {
    const Sizes z(M, D, F, dtype);
    return few_rows(z, keep) ? z.act_bytes(z.F) : ffn_workspace_bytes(M, D, F, dtype, false);
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
