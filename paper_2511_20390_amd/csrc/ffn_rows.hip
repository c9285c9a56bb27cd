// The two products of the gated feed-forward block for few token rows (a token that is being sampled, a handful of states): bound by
// reading the weights once, 2 F D and D F values, whatever the rows are.
//
// A workgroup owns 16 weight rows (gated: 16 gate rows and the 16 up rows of the same hidden values) and its wavefronts share K: step
// s of 128 bytes per row goes to wavefront s % wavefronts, so that a workgroup reads runs of a kilobyte and more of every row.  Weights
// go from memory to the registers of the matrix instruction directly - they are used once, LDS would only delay them -: lane l holds 32
// bytes of weight row l % 16 at 32 (l / 16) of the step and the same k of token l % 16; which of a step's k meet in an instruction does
// not matter to the sum.  bf16: v_mfma_f32_16x16x32_bf16; fp32: v_mfma_f32_16x16x4_f32, exact products, fp32 sums.  The wavefronts' sums
// are added through LDS in order, and the activation is applied there.
// Any D, F and number of rows: rows past the end are read as the last one and not written, a row's last step is read value by value
// where it is not whole, and rows that are not 16-byte aligned cost the memory pipe more, no copies.
#include <algorithm>
#include <type_traits>

#include "ffn_mfma.h"
#include "gemm_tile.h"

namespace freemi {

namespace {

typedef float f32x4a_t __attribute__((ext_vector_type(4)));

constexpr int kRowsPerGroup = 16;
constexpr int kStepBytes = 128;
constexpr int kUnroll = 4;

struct RowArgs {
    const void *x, *w;
    void* out;
    int32_t M, N, K, act;
};

template <typename T>
__device__ __forceinline__ void load_piece(const T* p, int left, u32x4_t (&v)[2], bool whole) {
    constexpr int E = 16 / sizeof(T);
    if (whole) {
        __builtin_memcpy(&v[0], p, 16);
        __builtin_memcpy(&v[1], p + E, 16);
        return;
    }
    // (left: values of the row from p on, maybe none)
    T t[2 * E];
#pragma unroll
    for (int e = 0; e < 2 * E; ++e) t[e] = e < left ? p[e] : T{};
    __builtin_memcpy(&v[0], t, 16);
    __builtin_memcpy(&v[1], t + E, 16);
}

template <typename T>
__device__ __forceinline__ void multiply(const u32x4_t& w, const u32x4_t& x, f32x4a_t& acc) {
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[e]), __uint_as_float(x[e]), acc, 0, 0, 0);
    }
}

__device__ __forceinline__ float gate_of(float g, int act) {
    if (act == FREE_ACT_SILU) return g / (1.0f + expf(-g));
    return 0.5f * g * (1.0f + tanhf(0.7978845608028654f * (g + 0.044715f * g * g * g)));
}

// kEdge: rows or their ends may not be whole pieces
template <typename T, int MT, int WAVES, bool kGated, bool kEdge>
__global__ __launch_bounds__(WAVES * 64) void ffn_rows_kernel(RowArgs a) {
    constexpr int NB = kGated ? 2 : 1;                           // weight matrices
    constexpr int kStep = kStepBytes / sizeof(T);
    __shared__ f32x4a_t red[WAVES][NB * MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * kRowsPerGroup;
    const int r16 = lane & 15, part = (lane >> 4) * (kStep / 4);
    const int n = n0 + r16 < a.N ? n0 + r16 : a.N - 1;
    const T* w[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) w[b] = static_cast<const T*>(a.w) + (static_cast<int64_t>(b) * a.N + n) * a.K + part;
    const T* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = t * 16 + r16;
        x[t] = static_cast<const T*>(a.x) + static_cast<int64_t>(m < a.M ? m : a.M - 1) * a.K + part;
    }
    f32x4a_t acc[NB][MT];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[b][t] = f32x4a_t{0.f, 0.f, 0.f, 0.f};
    const int steps = (a.K + kStep - 1) / kStep;
    for (int s0 = wave; s0 < steps; s0 += WAVES * kUnroll) {
        u32x4_t wv[kUnroll][NB][2], xv[kUnroll][MT][2];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int s = s0 + u * WAVES;
            if (s >= steps) continue;
            const int64_t k = static_cast<int64_t>(s) * kStep;
            const bool whole = !kEdge || k + kStep <= a.K;
            const int left = static_cast<int>(a.K - k) - part;
#pragma unroll
            for (int b = 0; b < NB; ++b) load_piece(w[b] + k, left, wv[u][b], whole);
#pragma unroll
            for (int t = 0; t < MT; ++t) load_piece(x[t] + k, left, xv[u][t], whole);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (s0 + u * WAVES >= steps) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int t = 0; t < MT; ++t) multiply<T>(wv[u][b][h], xv[u][t][h], acc[b][t]);
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < MT; ++t) red[wave][b * MT + t][lane] = acc[b][t];
    __syncthreads();
    // value i of a tile: token i / 16, weight row i % 16; it stands in lane token + 16 (row / 4), register row % 4
    for (int i = threadIdx.x; i < MT * 256; i += WAVES * 64) {
        const int t = i >> 8, token = i >> 4 & 15, row = i & 15, from = token + 16 * (row >> 2);
        const int m = t * 16 + token;
        if (m >= a.M || n0 + row >= a.N) continue;
        float v[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            v[b] = red[0][b * MT + t][from][row & 3];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) v[b] += red[k][b * MT + t][from][row & 3];
        }
        if constexpr (kGated) v[0] = gate_of(v[0], a.act) * v[1];
        store_f(static_cast<T*>(a.out) + static_cast<int64_t>(m) * a.N + n0 + row, v[0]);
    }
}

template <typename T, int MT, int WAVES, bool kGated>
int32_t launch_edge(const RowArgs& a, hipStream_t s) {
    const dim3 grid((a.N + kRowsPerGroup - 1) / kRowsPerGroup), block(WAVES * 64);
    if (a.K % (kStepBytes / sizeof(T)) == 0) hipLaunchKernelGGL((ffn_rows_kernel<T, MT, WAVES, kGated, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ffn_rows_kernel<T, MT, WAVES, kGated, true>), grid, block, 0, s, a);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <typename T, bool kGated>
int32_t launch_rows(const RowArgs& a, hipStream_t s) {
    if (a.M <= 16) return launch_edge<T, 1, 8, kGated>(a, s);
    if (a.M <= 32) return launch_edge<T, 2, 8, kGated>(a, s);
    return launch_edge<T, 4, 8, kGated>(a, s);
}

}  // namespace

template <typename T>
int32_t launch_ffn_rows(const T* x, const T* w_in, const T* w_out, int32_t M, int32_t D, int32_t F, int32_t act, T* h, T* out, hipStream_t s) {
    const int32_t st = launch_rows<T, true>(RowArgs{x, w_in, h, M, F, D, act}, s);
    return st != FREE_OK ? st : launch_rows<T, false>(RowArgs{h, w_out, out, M, D, F, act}, s);
}
template int32_t launch_ffn_rows(const bf16_t*, const bf16_t*, const bf16_t*, int32_t, int32_t, int32_t, int32_t, bf16_t*, bf16_t*, hipStream_t);
template int32_t launch_ffn_rows(const float*, const float*, const float*, int32_t, int32_t, int32_t, int32_t, float*, float*, hipStream_t);

}  // namespace freemi
