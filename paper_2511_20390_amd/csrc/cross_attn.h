// What the kernels of cross attention and of its gradient share (cross_attn.hip, cross_attn_grad.hip).  Device code, bf16 and fp32.
//
// Formulation of both: a tile of scores is computed so that in the accumulator layout of the 32 x 32 matrix instructions a lane owns one
// column (its queries, or in the keys' gradient its keys) and half of the tile's rows.  What is computed from the scores then already is
// the B operand of the next product, whose A operand is the tile the rows came from, read column-wise: bf16 by the transposing LDS read
// (8 consecutive rows of a column per lane; the rows of a 32-row block are taken with bits 2 and 3 of their number swapped, which makes the
// 8 registers of an instruction 8 consecutive rows), fp32 by one value per register (v_mfma_f32_32x32x2_f32 contracts over the two rows
// that the half-waves hold in a register).  A 16-byte chunk of a row is 8 values or 4, one instruction or four: the loops are the same.
#pragma once

#include "buffer_range.h"
#include "free_internal.h"
#include "lanes.h"

namespace freemi {

struct CrossArgs {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;        // values from row to row
    const int32_t* key_len;                      // nullable
    const uint8_t* key_mask;                     // nullable, [B, Nk]
    int32_t B, Nq, Nk, heads, kv_heads, dh;
    float scale;
    // forward
    void* out;
    int64_t out_stride;
    float* lse;                                  // nullable; the gradient: an input
    // gradient
    const void* dout;
    int64_t dout_stride;
    void *dq, *dk, *dv;
    int64_t dq_stride, dk_stride, dv_stride;
};

namespace {

typedef __bf16 xbf16x8_t __attribute__((ext_vector_type(8)));
typedef short xs16x4_t __attribute__((ext_vector_type(4)));
typedef short xs16x8_t __attribute__((ext_vector_type(8)));
typedef float xf32x4_t __attribute__((ext_vector_type(4)));
typedef float xf32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t xu32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t xu32x2_t __attribute__((ext_vector_type(2)));

constexpr int kXcds = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// DP: the head dimension, rounded up to one there is an instance of
template <typename T, int DP>
struct HeadShape {
    static constexpr int E = 16 / sizeof(T);                     // values of a chunk
    static constexpr int CH = DP / E;                            // chunks of a row
    static constexpr int KSTEPS = CH / 2;                        // the half-waves take one chunk each
    static constexpr int DT = (DP + 31) / 32;                    // 32-row tiles of a result with the head dimension as rows
};

__device__ __forceinline__ int swapped_bits_2_3(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// the row of a 32-row block that stands in row i of a tile of scores
template <typename T>
__device__ __forceinline__ int block_row(int i) {
    return sizeof(T) == 2 ? swapped_bits_2_3(i) : i;
}
// ... and which of the block's rows register e of half-wave g holds
template <typename T>
__device__ __forceinline__ constexpr int register_row(int e, int g) {
    return sizeof(T) == 2 ? 16 * (e >> 3) + 8 * g + 4 * ((e >> 2) & 1) + (e & 3) : 8 * (e >> 2) + 4 * g + (e & 3);
}

// acc += a b over one chunk of each half-wave
template <typename T>
__device__ __forceinline__ void chunk_product(const xu32x4_t& a, const xu32x4_t& b, xf32x16_t& acc) {
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(xbf16x8_t, a), __builtin_bit_cast(xbf16x8_t, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
    }
}

__device__ __forceinline__ void clear_tile(xf32x16_t& v) {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = 0.f;
}

// a row's chunk c, at p + c E; kVec: rows are 16-byte aligned and dh whole chunks, else value by value.  Behind dh: zeros.
template <typename T, bool kVec>
__device__ __forceinline__ xu32x4_t row_chunk(const T* p, int c, int dh) {
    constexpr int E = 16 / sizeof(T);
    xu32x4_t v = {0, 0, 0, 0};
    if constexpr (kVec) {
        if (c * E < dh) v = *reinterpret_cast<const xu32x4_t*>(p + c * E);
    } else {
        T t[E];
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = c * E + e < dh ? p[c * E + e] : T{};
        __builtin_memcpy(&v, t, 16);
    }
    return v;
}

// the same out of a buffer that ends where the rows do: voff (bytes) is the chunk's place for this lane
template <typename T, bool kVec>
__device__ __forceinline__ xu32x4_t buffer_chunk(__amdgpu_buffer_rsrc_t rsrc, int voff, int c, int dh) {
    constexpr int E = 16 / sizeof(T);
    if constexpr (kVec) {
        return __builtin_bit_cast(xu32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rsrc, c * E < dh ? voff : 0x7fffffff, 0, 0));
    } else {
        T t[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int at = c * E + e < dh ? voff + e * static_cast<int>(sizeof(T)) : 0x7fffffff;
            if constexpr (sizeof(T) == 2) t[e].v = static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(rsrc, at, 0, 0));
            else t[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rsrc, at, 0, 0));
        }
        xu32x4_t v;
        __builtin_memcpy(&v, t, 16);
        return v;
    }
}

// buffer over `rows` rows of dh values from p on (none: everything reads as zero)
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const T* p, int64_t rows, int64_t stride, int dh) {
    const int64_t bytes = rows > 0 ? ((rows - 1) * stride + dh) * static_cast<int64_t>(sizeof(T)) : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p), 0, static_cast<int>(range_bytes(bytes)), 0x00020000);
}

// four consecutive values of a row to memory, those before dh
template <typename T, bool kVec>
__device__ __forceinline__ void store4(T* row, int d, int dh, float a, float b, float c, float e) {
    if constexpr (kVec) {
        if (d >= dh) return;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<xu32x2_t*>(row + d) = xu32x2_t{pack_bf16_pair(a, b), pack_bf16_pair(c, e)};
        else *reinterpret_cast<xf32x4_t*>(row + d) = xf32x4_t{a, b, c, e};
    } else {
        const float v[4] = {a, b, c, e};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d + i < dh) store_f(row + d + i, v[i]);
    }
}

// 8 registers of a tile of scores' row order as operands of the next product; fp32 uses the registers as they are
__device__ __forceinline__ xu32x4_t pack8(const float (&p)[8]) {
    return xu32x4_t{pack_bf16_pair(p[0], p[1]), pack_bf16_pair(p[2], p[3]), pack_bf16_pair(p[4], p[5]), pack_bf16_pair(p[6], p[7])};
}

__device__ __forceinline__ xs16x4_t read_transposed(const char* at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) xs16x4_t*)(at));
}

__device__ __forceinline__ xu32x4_t transposed_chunk(const char* lo, const char* hi) {
    const xs16x8_t v = __builtin_shufflevector(read_transposed(lo), read_transposed(hi), 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(xu32x4_t, v);
}

// which of the 64 (or, with 32 keys per tile, low 32) keys from kv0 on count
__device__ __forceinline__ uint64_t keys_below(int left) { return left >= 64 ? ~0ull : left <= 0 ? 0ull : (1ull << left) - 1; }

}  // namespace

// cross_attn.hip, cross_attn_grad.hip; arguments checked in cross_abi.hip
size_t cross_forward_bytes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype);
size_t cross_backward_bytes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype);
int32_t launch_cross_forward(const CrossArgs& a, int32_t dtype, void* ws, hipStream_t s);
int32_t launch_cross_backward(const CrossArgs& a, int32_t dtype, void* ws, hipStream_t s);

}  // namespace freemi
