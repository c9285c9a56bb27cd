// What the rows of a linear layer get besides from the adapters of their requests, for the kernels that add it to the layer's sums.
#pragma once

#include <type_traits>

#include "free_internal.h"

namespace freemi {

// Row m, column n: the sum over ranks of t[m, rank] b_a[n, rank], a = adapter[m / rows_per_sample]; nothing where that is none of n_adapters.
// t: rows of t_row values, zeros past r, 16-byte aligned; b: [adapter][cols][b_row], any alignment.
struct AdapterTerm {
    const void *t, *b;
    const int32_t* adapter;
    const float* bias;               // few rows' kernel alone
    int32_t n_adapters, r, t_row, b_row, cols, rows_per_sample;
#if defined(__HIPCC__)
    __device__ __forceinline__ int of_row(int m) const {
        const int a = adapter[m / rows_per_sample];
        return a >= 0 && a < n_adapters ? a : -1;
    }
#endif
};

// epilogue code of the linear layers: FREE_EPI_BIAS of sums that begin with the rows' adapters
constexpr int FREE_EPI_ADAPT = 10;
struct NoAdapters {};
template <int EPI>
using AdaptersOf = std::conditional_t<EPI == FREE_EPI_ADAPT, AdapterTerm, NoAdapters>;

#if defined(__HIPCC__)
namespace {

// acc[i][j] += the term, for rows gm + 32 i and columns gn + 32 j of a wavefront whose lane has row and column lane % 32 (bf16, the
// accumulators' order of v_mfma_f32_32x32x16_bf16 with W's rows first).  The adapters of the wavefront's rows come one after the other as
// k-steps of 16 ranks.  Operands come straight from memory behind the loads of the first slices; a launch of its own over the finished result
// would read and write it once more, and round it twice.
// Zeros in the operands of rows with another adapter would not keep an infinite or NaN one out of them: where a wavefront's rows differ, such values
// of B count as zero, and the rows that have the adapter get NaN in their columns.
template <int TM, int TN, typename Acc>
__device__ __forceinline__ void add_adapters(const AdapterTerm& ad, int gm, int gn, int lhi, int M, Acc (&acc)[TM][TN]) {
    typedef uint32_t chunk_t __attribute__((ext_vector_type(4)));
    typedef __bf16 operand_t __attribute__((ext_vector_type(8)));
    int of[TM];                      // the adapters of this lane's rows that are still to be added
#pragma unroll
    for (int i = 0; i < TM; ++i) of[i] = gm + 32 * i < M ? ad.of_row(gm + 32 * i) : -1;
    const bool whole = ad.b_row % 8 == 0 && (reinterpret_cast<uintptr_t>(ad.b) & 15u) == 0;
    for (;;) {
        int which = -1;              // (of a row that has one)
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const uint64_t left = __ballot(of[i] >= 0);
            which = left != 0 ? __builtin_amdgcn_readlane(of[i], __builtin_ctzll(left)) : which;
        }
        if (which < 0) break;
        bool on[TM], all = true;     // (rows past the end do as the others do)
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            on[i] = of[i] == which;
            all = all && (on[i] || gm + 32 * i >= M);
            of[i] = on[i] ? -1 : of[i];
        }
        const bool mixed = __ballot(all) != ~0ull;
        uint32_t bad = 0;            // columns gn + 32 j with such values in this lane's ranks
        const bf16_t* const b = static_cast<const bf16_t*>(ad.b) + static_cast<int64_t>(which) * ad.cols * ad.b_row;
        for (int k0 = 0; k0 < ad.r; k0 += 16) {
            const int k = k0 + lhi * 8;
            chunk_t bv[TN], tv[TM];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int n = gn + 32 * j;
                const bf16_t* const p = b + static_cast<int64_t>(n < ad.cols ? n : ad.cols - 1) * ad.b_row + k;
                bv[j] = chunk_t{0, 0, 0, 0};
                if (whole) {
                    if (k < ad.r) bv[j] = *reinterpret_cast<const chunk_t*>(p);
                } else {
                    bf16_t v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = k + e < ad.r ? p[e] : bf16_t{0};
                    __builtin_memcpy(&bv[j], v, 16);
                }
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                tv[i] = chunk_t{0, 0, 0, 0};
                if (on[i]) tv[i] = *reinterpret_cast<const chunk_t*>(static_cast<const bf16_t*>(ad.t) + static_cast<int64_t>(gm + 32 * i) * ad.t_row + k);
            }
            if (mixed) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool lo = (bv[j][e] & 0x7f80u) == 0x7f80u, hi = (bv[j][e] & 0x7f800000u) == 0x7f800000u;
                        bv[j][e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
                        bad |= static_cast<uint32_t>(lo || hi) << j;
                    }
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(operand_t, bv[j]), __builtin_bit_cast(operand_t, tv[i]), acc[i][j], 0, 0, 0);
        }
        if (__builtin_expect(__ballot(bad != 0) != 0, 0)) {
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const uint64_t halves = __ballot(bad >> j & 1);
                const uint32_t columns = static_cast<uint32_t>(halves | halves >> 32) >> (4 * lhi);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        acc[i][j][e] = on[i] && (columns >> (8 * (e >> 2) + (e & 3)) & 1) ? __builtin_nanf("") : acc[i][j][e];
            }
        }
    }
}

}  // namespace
#endif

// bf16, K whole slices of 64: out = X W^T + bias and the term (gemm_mfma.hip chooses the tile as for free_op_linear)
int32_t launch_linear_adapters(const bf16_t* X, const bf16_t* W, const float* bias, int32_t M, int32_t N, int32_t K, bf16_t* out, const AdapterTerm& term,
                               hipStream_t s);
int32_t launch_linear_pipe_adapters(const bf16_t* X, const bf16_t* W, const float* bias, int32_t M, int32_t N, int32_t K, bf16_t* out, hipStream_t s,
                                    PipeTile tile, const AdapterTerm& term);
int32_t launch_linear_rows_adapters(const bf16_t* X, const bf16_t* W, const float* bias, int32_t M, int32_t N, int32_t K, bf16_t* out, hipStream_t s,
                                    RowsTile tile, const AdapterTerm& term);

}  // namespace freemi
