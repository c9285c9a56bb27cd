// The matrix products of the gated feed-forward block (ffn_mfma.hip; fp32: gemm_f32.hip), for ffn.hip.  bf16: widths and leading
// dimensions are multiples of 8; fp32: of 64, and rows dense.  Pointers are 16-byte aligned.
#pragma once

#include "free_internal.h"

namespace freemi {

// what a product is: the layout of its operands and its epilogue
enum FfnKind {
    FFN_GATE,          // out = act(g) u of X [M, K] and W [2 N, K]
    FFN_GATE_KEEP,     // and g, u kept in gu
    FFN_GATE_GRAD,     // out [M, 2 N] = [dg | du] of dh = X [M, K] by W [K, N], with the kept gu
    FFN_ROWS,          // out = X [M, K] by W [N, K]
    FFN_ROWS_BY_K,     // out = X [M, K] by W [K, N]
    FFN_K_BY_K,        // out = X [K, M] by W [K, N]
    FFN_STORE,         // (epilogues of the kernel alone: plain, and parts of K)
    FFN_PART
};

template <typename T>                // bf16_t or float
struct FfnProduct {
    FfnKind kind;
    const T *X, *W;
    int64_t ldx, ldw;
    int32_t M, N, K;
    T* out;
    int64_t ldo;
    float* gu = nullptr;             // [g | u] as 32 x 32 blocks: [M / 32 rounded up][2 H / 32][4][lane][4]
    int32_t act = 0;
    // H, N rounded up to a multiple of 64, for the gated kinds: what `out` has columns for, zeros past N (the gradient: du at H)
    int32_t hidden = 0;
    // dg and du as rows of C (FFN_K_BY_K) or of W (FFN_ROWS_BY_K): index fold + i of [dg | du] is row fold_to + i, indexes from fold_to to
    // fold are none
    int32_t fold = 0, fold_to = 0;
    int32_t cols() const { return hidden > 0 ? hidden : N; }
    bool gated() const { return kind == FFN_GATE || kind == FFN_GATE_KEEP; }
};

// One launch for n products (1, or 2 FFN_K_BY_K), and one more for each whose sums over K are cut in parts, or, fp32, to which an activation is
// applied.  part: room of ffn_products_part_bytes (by the sizes alone).
size_t ffn_products_part_bytes(const FfnProduct<bf16_t>* p, int n);
size_t ffn_products_part_bytes(const FfnProduct<float>* p, int n);
int32_t launch_ffn_products(const FfnProduct<bf16_t>* p, int n, float* part, hipStream_t s);
int32_t launch_ffn_products(const FfnProduct<float>* p, int n, float* part, hipStream_t s);

// ffn_rows.hip: y of up to 32 token rows, any D and F, in two launches; h: room for [M, F].  ffn_rows_pay: where that is the faster way.
bool ffn_rows_pay(int32_t M, int32_t D, int32_t F, bool tiles_padded);
template <typename T>
int32_t launch_ffn_rows(const T* x, const T* w_in, const T* w_out, int32_t M, int32_t D, int32_t F, int32_t act, T* h, T* out, hipStream_t s);

}  // namespace freemi
