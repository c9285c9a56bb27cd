// The two products of the gated feed-forward block for few token rows (a token that is being sampled, a handful of states): bound by
// reading the weights once, 2 F D and D F values, whatever the rows are.
//
// A workgroup owns R = 16 or 8 weight rows (gated: of either matrix, the same hidden values) and its 8 wavefronts share K, step by step of
// 128 bytes per row, so that a workgroup reads runs of a kilobyte of every row.  Weights go from memory to the registers of the matrix
// instruction directly: they are used once, LDS would only delay them.  A row's step is 8 pieces of 16 bytes, and 16 lanes meet two of
// them with their 16 tokens: with R = 16 lane l has both of weight row l % 16; with R = 8 it has one of row l % 8, and the instruction for the
// other finds its rows 8 lanes away.  Which of a step's k meet in an instruction does not matter to the sum.  bf16:
// v_mfma_f32_16x16x32_bf16; fp32: v_mfma_f32_16x16x4_f32, exact products, fp32 sums.  The wavefronts' sums are added through LDS in
// order, and the activation is applied there.
// R = 8 spreads the weights over twice the workgroups (a compute unit takes some 46 KB/us from memory) and reads 128 bytes of a row per
// instruction instead of 64, but loads the tokens once more per weight.  us with 16 rows in both launches, with 8 in both, with 8 for gate
// and up alone: bf16, one row, 1152 x 4608 15.7, 13.3, 15.2; 4096 x 10240 52.9, 46.4, 45.5; 16 rows 19.8, 18.2, 20.0; 60.9, 73.0, 64.5.
// Any D, F and number of rows: rows past the end are read as the last one and not written, a row's last step is read value by value
// where it is not whole, and rows that are not 16-byte aligned cost the memory pipe more, no copies.
#include <algorithm>
#include <type_traits>

#include "ffn_mfma.h"
#include "gemm_tile.h"

namespace freemi {

namespace {

typedef float f32x4a_t __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;

struct RowArgs {
    const void *x, *w;
    void* out;
    int32_t M, N, K, act;
};

// 16 bytes; left: values of the row from p on, maybe none
template <typename T>
__device__ __forceinline__ void load_piece(const T* p, int left, u32x4_t& v, bool whole) {
    constexpr int E = 16 / sizeof(T);
    if (whole || left >= E) {
        __builtin_memcpy(&v, p, 16);
        return;
    }
    T t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = e < left ? p[e] : T{};
    __builtin_memcpy(&v, t, 16);
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

// kEdge: rows' last steps may not be whole
template <typename T, int R, int MT, bool kGated, bool kEdge>
__global__ __launch_bounds__(kWaves * 64) void ffn_rows_kernel(RowArgs a) {
    constexpr int NB = kGated ? 2 : 1;                           // weight matrices
    constexpr int P = 2, H = R / 8;                              // pieces of a step for 16 lanes; of them in one lane
    constexpr int E = 16 / sizeof(T), kStep = 4 * P * E;         // values
    constexpr int U = 4;                                         // steps in flight per wavefront
    __shared__ f32x4a_t red[kWaves][NB * MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * R, quad = lane >> 4, r16 = lane & 15;
    const int n = n0 + r16 % R < a.N ? n0 + r16 % R : a.N - 1;
    const int w_at = (quad * P + r16 / R * H) * E, x_at = quad * P * E;
    const T* w[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) w[b] = static_cast<const T*>(a.w) + (static_cast<int64_t>(b) * a.N + n) * a.K + w_at;
    const T* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = t * 16 + r16;
        x[t] = static_cast<const T*>(a.x) + static_cast<int64_t>(m < a.M ? m : a.M - 1) * a.K + x_at;
    }
    f32x4a_t acc[NB][MT];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[b][t] = f32x4a_t{0.f, 0.f, 0.f, 0.f};
    const int steps = (a.K + kStep - 1) / kStep;
    for (int s0 = wave; s0 < steps; s0 += kWaves * U) {
        u32x4_t wv[U][NB][H], xv[U][MT][P];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * kWaves;
            if (s >= steps) continue;
            const int64_t k = static_cast<int64_t>(s) * kStep;
            const bool whole = !kEdge || k + kStep <= a.K;
            const int left = static_cast<int>(a.K - k);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int h = 0; h < H; ++h) load_piece(w[b] + k + h * E, left - w_at - h * E, wv[u][b][h], whole);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int p = 0; p < P; ++p) load_piece(x[t] + k + p * E, left - x_at - p * E, xv[u][t][p], whole);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u * kWaves >= steps) continue;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    const u32x4_t v = wv[u][b][h];
#pragma unroll
                    for (int t = 0; t < MT; ++t) multiply<T>(v, xv[u][t][h], acc[b][t]);
                    if constexpr (R == 8) {
                        u32x4_t other;
#pragma unroll
                        for (int e = 0; e < 4; ++e) other[e] = lane_xor<8>(static_cast<uint32_t>(v[e]));
#pragma unroll
                        for (int t = 0; t < MT; ++t) multiply<T>(other, xv[u][t][1], acc[b][t]);
                    }
                }
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < MT; ++t) red[wave][b * MT + t][lane] = acc[b][t];
    __syncthreads();
    // value i of a tile: token i / R, weight row i % R; it stands in lane token + 16 (row / 4), register row % 4
    for (int i = threadIdx.x; i < MT * 16 * R; i += kWaves * 64) {
        const int t = i / (16 * R), token = i / R % 16, row = i % R, from = token + 16 * (row >> 2);
        const int m = t * 16 + token;
        if (m >= a.M || n0 + row >= a.N) continue;
        float v[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            v[b] = red[0][b * MT + t][from][row & 3];
#pragma unroll
            for (int k = 1; k < kWaves; ++k) v[b] += red[k][b * MT + t][from][row & 3];
        }
        if constexpr (kGated) v[0] = gate_of(v[0], a.act) * v[1];
        store_f(static_cast<T*>(a.out) + static_cast<int64_t>(m) * a.N + n0 + row, v[0]);
    }
}

template <typename T, int R, int MT, bool kGated>
int32_t launch_edge(const RowArgs& a, hipStream_t s) {
    constexpr int kStep = 128 / sizeof(T);
    const dim3 grid((a.N + R - 1) / R), block(kWaves * 64);
    if (a.K % kStep == 0) hipLaunchKernelGGL((ffn_rows_kernel<T, R, MT, kGated, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ffn_rows_kernel<T, R, MT, kGated, true>), grid, block, 0, s, a);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <typename T, bool kGated>
int32_t launch_rows(const RowArgs& a, hipStream_t s) {
    // 8 weight rows where groups of 16 would leave compute units without one, and for gate and up of few tokens
    if (a.N < 16 * 256 || (kGated && a.M <= 8)) return a.M <= 16 ? launch_edge<T, 8, 1, kGated>(a, s) : launch_edge<T, 8, 2, kGated>(a, s);
    return a.M <= 16 ? launch_edge<T, 16, 1, kGated>(a, s) : launch_edge<T, 16, 2, kGated>(a, s);
}

}  // namespace

template <typename T>
int32_t launch_ffn_rows(const T* x, const T* w_in, const T* w_out, int32_t M, int32_t D, int32_t F, int32_t act, T* h, T* out, hipStream_t s) {
    const int32_t st = launch_rows<T, true>(RowArgs{x, w_in, h, M, F, D, act}, s);
    return st != FREE_OK ? st : launch_rows<T, false>(RowArgs{h, w_out, out, M, D, F, act}, s);
}
// Against the tiles of ffn_mfma.hip and gemm_f32.hip, us.  16 rows: bf16 384 x 1536 7.5 against 15, 1152 x 4608 18.3 against 26, 4096 x 10240
// 60.9 against 64.7; fp32 10.9 against 24, 31.9 against 38, 128 against 143.  32 rows: bf16 9.5 against 15.3, 27.0 against 26.9, 64.4 against 65.7
// (17 rows of 4096 x 10240 63.9 against 65.0); fp32 15.5 against 24, 49.8 against 38.8, 191 against 147.  Where the tiles would need
// padded copies of the weights, three times their bytes, 32 rows always.
bool ffn_rows_pay(int32_t M, int32_t D, int32_t F, bool tiles_padded) {
    return M <= 16 || (M <= 32 && (tiles_padded || static_cast<int64_t>(D) * F <= 1 << 22));
}

template int32_t launch_ffn_rows(const bf16_t*, const bf16_t*, const bf16_t*, int32_t, int32_t, int32_t, int32_t, bf16_t*, bf16_t*, hipStream_t);
template int32_t launch_ffn_rows(const float*, const float*, const float*, int32_t, int32_t, int32_t, int32_t, float*, float*, hipStream_t);

}  // namespace freemi
