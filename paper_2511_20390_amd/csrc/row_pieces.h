// Operands of the matrix instructions on 16 rows straight from memory, for kernels on few rows or few columns.  Device code.
#pragma once

#include "ffn_mfma.h"
#include "gemm_tile.h"

namespace freemi {

namespace {

typedef float f32x4a_t __attribute__((ext_vector_type(4)));

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

// bias and adapter of one value of a product (AdapterTerm)
template <typename T>
__device__ __forceinline__ float adapter_value(const AdapterTerm& ad, int m, int n) {
    constexpr int E = 16 / sizeof(T);
    float v = ad.bias ? ad.bias[n] : 0.f;
    const int which = ad.of_row(m);
    if (which < 0) return v;
    const T* const t = static_cast<const T*>(ad.t) + static_cast<int64_t>(m) * ad.t_row;
    const T* const b = static_cast<const T*>(ad.b) + (static_cast<int64_t>(which) * ad.cols + n) * ad.b_row;
    for (int k = 0; k < ad.r; k += E) {
        u32x4_t tv, bv;
        load_piece(t + k, ad.r - k, tv, false);
        load_piece(b + k, ad.r - k, bv, false);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) {
                v = fmaf(__uint_as_float(tv[e] << 16), __uint_as_float(bv[e] << 16), v);
                v = fmaf(__uint_as_float(tv[e] & 0xffff0000u), __uint_as_float(bv[e] & 0xffff0000u), v);
            } else {
                v = fmaf(__uint_as_float(tv[e]), __uint_as_float(bv[e]), v);
            }
        }
    }
    return v;
}

}  // namespace
}  // namespace freemi
