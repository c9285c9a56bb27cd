// What the kernels of cross attention and of its gradient share (cross_attn.hip, cross_attn_grad.hip).  Device code, bf16 and fp32.
//
// Formulation of both: a tile of scores is computed so that in the accumulator layout of the 32 x 32 matrix instructions a lane owns one
// column (its queries, or in the keys' gradient its keys) and half of the tile's rows.  What is computed from the scores then already is
// the B operand of the next product, whose A operand is the tile the rows came from, read column-wise: bf16 by the transposing LDS read
// (8 consecutive rows of a column per lane; the rows of a 32-row block are taken with bits 2 and 3 of their number swapped, which makes the
// 8 registers of an instruction 8 consecutive rows), fp32 by one value per register (v_mfma_f32_32x32x2_f32 contracts over the two rows
// that the half-waves hold in a register).  A 16-byte chunk of a row is 8 values or 4, one instruction or four: the loops are the same.
#pragma once

#include <algorithm>
#include <type_traits>

#include "gemm_dma.h"
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

// A lane's column of 32 DT values (register e of tile dt: value 32 dt + 8 (e / 4) + 4 (lane / 32) + e % 4) times `factor` to its row, those before dh.
// bf16: the half-waves, which have four values of eight each, exchange them, so that a store is 16 bytes per lane and 32 next to each other: the memory
// pipe takes as long for 8 bytes of 32 rows.
template <typename T, bool kVec, int DT>
__device__ __forceinline__ void store_column(T* row, int dh, int g, const xf32x16_t (&v)[DT], float factor, bool on) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        if constexpr (sizeof(T) == 2 && kVec) {
#pragma unroll
            for (int e8 = 0; e8 < 2; ++e8) {
                const auto pair = [&](int e) { return pack_bf16_pair(v[dt][8 * e8 + e] * factor, v[dt][8 * e8 + e + 1] * factor); };
                const xu32x2_t s0 = __builtin_amdgcn_permlane32_swap(pair(0), pair(4), false, false), s1 = __builtin_amdgcn_permlane32_swap(pair(2), pair(6), false, false);
                const int d = 32 * dt + 16 * e8 + 8 * g;
                if (on && d < dh) *reinterpret_cast<xu32x4_t*>(row + d) = xu32x4_t{s0[0], s1[0], s0[1], s1[1]};
            }
        } else if (on) {
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                store4<T, kVec>(row, 32 * dt + 8 * e4 + 4 * g, dh, v[dt][4 * e4] * factor, v[dt][4 * e4 + 1] * factor, v[dt][4 * e4 + 2] * factor, v[dt][4 * e4 + 3] * factor);
        }
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

// Loads that a loop's products use have arrived: without this the compiler waits for them in the loop, and there for every load that the loop
// itself has requested since.
template <int N>
__device__ __forceinline__ void arrived(xu32x4_t (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

__device__ __forceinline__ int over_group(int row, int group) { return group == 1 ? row : row / group; }

// which of the 64 (or, with 32 keys per tile, low 32) keys from kv0 on count
__device__ __forceinline__ uint64_t keys_below(int left) { return left >= 64 ? ~0ull : left <= 0 ? 0ull : (1ull << left) - 1; }

// ---- tiles of streamed rows in LDS.  A tile is read by rows (16 bytes of 32 rows: scores) and by columns (transposing reads of 4 rows x 64 bytes; fp32
// 32 values of a row), and its chunks are at places that keep the lanes of either off each other's banks (64 banks, 16 chunks):
//   rows of 4 or 12 chunks: 16 rows of one chunk c, four next to each other on every fourth place -> c ^ (row / 4 % 4)
//   rows of 10: every second place, eight rows of them -> c ^ (row / 8 % 2)      rows of 8 and 16: likewise, and the four rows of a
//   transposing read, which start at the same bank, on different groups of four places
// fp32: rows of an odd number of chunks.
constexpr int kOverRead = 128;                   // bytes behind a tile that its last rows' columns may reach (they are read, and dropped)

template <typename T, int DP>
struct Tile {
    using H = HeadShape<T, DP>;
    static constexpr int kRows = sizeof(T) == 2 ? 64 : 32;
    static constexpr int CHP = sizeof(T) == 2 ? H::CH : H::CH | 1;                // chunks from row to row
    static constexpr int kPitch = CHP * 16;
    static constexpr int kBytes = kRows * kPitch + kOverRead;
    static_assert(sizeof(T) == 4 || CHP == 4 || CHP == 8 || CHP == 10 || CHP == 12 || CHP == 16, "a place for every chunk");
    static __host__ __device__ __forceinline__ constexpr int turn(int row) {
        if constexpr (sizeof(T) == 4) return 0;
        else if constexpr (CHP == 16) return (row & 3) << 2 | (row >> 2 & 3);
        else if constexpr (CHP == 8) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
        else if constexpr (CHP == 10) return row >> 3 & 1;
        else return row >> 2 & 3;
    }
    static __host__ __device__ __forceinline__ constexpr int at(int row, int c) { return row * kPitch + ((c ^ turn(row)) << 4); }
    // behind the last byte that reading the tile's columns touches: all 32 of the last block of them
    static constexpr int columns_end() {
        if (sizeof(T) == 4) return (kRows - 1) * kPitch + H::DT * 128;
        int end = 0;
        for (int row = 0; row < kRows; ++row)
            for (int c = 0; c < 4 * H::DT; ++c) end = std::max(end, at(row, c) + 16);
        return end;
    }
};

constexpr int kStreamThreads = 256, kNowhere = 0x7fffffff;       // a byte offset behind every buffer: reads as zero

// Brings tiles of one tensor's rows into LDS.  bf16 rows of whole chunks go there without registers in between (a lane's place in LDS is given,
// so it fetches the chunk that belongs there); others through registers: request() ahead of a tile's products, deliver() behind them.
template <typename T, int DP, bool kVec>
struct TileStream {
    using TL = Tile<T, DP>;
    static constexpr bool kDirect = sizeof(T) == 2 && kVec;
    static constexpr int E = TL::H::E, CH = TL::H::CH, kBlocks = TL::kRows * TL::kPitch / 1024, kWaves = kStreamThreads / 64;
    static constexpr int N = kDirect ? (kBlocks + kWaves - 1) / kWaves : (TL::kRows * CH + kStreamThreads - 1) / kStreamThreads;
    static_assert(!kDirect || TL::kRows * TL::kPitch % 1024 == 0, "whole blocks");
    xu32x4_t reg[kDirect ? 1 : N];

    // Row r of the tile is place(r) bytes behind base, whose buffer ends with the last row that there is.  valid: the rows that count, where
    // `masked` (others read as zero).  lds: the tile.
    template <typename Place>
    __device__ __forceinline__ void request(const T* base, int64_t bytes, uint32_t lds, int wave, int lane, int dh, bool masked, uint64_t valid, Place&& place) {
        if constexpr (kDirect) {
            const u32x4_t rsrc = make_rsrc(base, bytes);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int block = wave + kWaves * i;
                if (kBlocks % kWaves != 0 && block >= kBlocks) break;
                const int slot = block * 64 + lane, row = slot / TL::CHP, c = (slot % TL::CHP) ^ TL::turn(row);
                int off = c * E < dh ? place(row) + c * 16 : kNowhere;
                if (masked) off = valid >> row & 1 ? off : kNowhere;
                dma_1k(lds + block * 1024, off, rsrc, 0);
            }
        } else {
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, static_cast<int>(range_bytes(bytes)), 0x00020000);
            const int tid = wave * 64 + lane;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int idx = tid + kStreamThreads * i, row = idx / CH, c = idx % CH;
                if (idx < TL::kRows * CH) reg[i] = buffer_chunk<T, kVec>(rsrc, place(row) + c * 16, c, dh);
            }
        }
    }
    __device__ __forceinline__ void deliver(char* tile, int tid, bool masked, uint64_t valid) {
        if constexpr (!kDirect) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int idx = tid + kStreamThreads * i, row = idx / CH, c = idx % CH;
                if (idx < TL::kRows * CH) {
                    if (masked && !(valid >> row & 1)) reg[i] = xu32x4_t{0, 0, 0, 0};
                    *reinterpret_cast<xu32x4_t*>(tile + TL::at(row, c)) = reg[i];
                }
            }
        }
    }
    // everything requested and delivered is in LDS, for the whole workgroup
    static __device__ __forceinline__ void settle() {
        if constexpr (kDirect) wait_vm_barrier<0>();
        else __syncthreads();
    }
};

// The operands of a product are read from LDS ahead of the products before it: a wavefront that reads, waits and multiplies in turn spends
// its time on the latency of LDS (dk and dv of 32760 queries to 512 keys of 16 heads of 128, 530 -> 385 us).  `fence` keeps the compiler from putting
// the reads back behind the products.
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// chunks of a row that are read together (fp32: its products take eight times as long per chunk)
template <typename T, int DP>
constexpr int kRowGroup = sizeof(T) == 4 ? 4 : HeadShape<T, DP>::KSTEPS <= 5 ? HeadShape<T, DP>::KSTEPS : HeadShape<T, DP>::KSTEPS / 2;

// the row operands of the block of 32 rows from row0 on: a group of chunks from `first` on
template <typename T, int DP>
__device__ __forceinline__ void read_rows(const char* tile, int row0, int lane, int first, xu32x4_t (&f)[kRowGroup<T, DP>]) {
    const int row = block_row<T>(lane & 31), g = lane >> 5;
    const char* const base = tile + row0 * Tile<T, DP>::kPitch;
#pragma unroll
    for (int k = 0; k < kRowGroup<T, DP>; ++k)
        if (first + k < HeadShape<T, DP>::KSTEPS) f[k] = *reinterpret_cast<const xu32x4_t*>(base + Tile<T, DP>::at(row, 2 * (first + k) + g));
}

// acc += block . own, with the first group of the block's rows in f.  kAhead: see fence; without it the compiler orders reads and products.
template <typename T, int DP, bool kAhead = true>
__device__ __forceinline__ void row_products(const char* tile, int row0, int lane, xu32x4_t (&f)[kRowGroup<T, DP>],
                                             const xu32x4_t (&own)[HeadShape<T, DP>::KSTEPS], xf32x16_t& acc) {
    constexpr int G = kRowGroup<T, DP>, KSTEPS = HeadShape<T, DP>::KSTEPS;
#pragma unroll
    for (int first = 0; first < KSTEPS; first += G) {
        xu32x4_t next[G];
        if (first + G < KSTEPS) {
            read_rows<T, DP>(tile, row0, lane, first + G, next);
            if constexpr (kAhead) fence();
        }
#pragma unroll
        for (int k = 0; k < G; ++k)
            if (first + k < KSTEPS) chunk_product<T>(f[k], own[first + k], acc);
#pragma unroll
        for (int k = 0; k < G; ++k) f[k] = next[k];
    }
}

// Column operands of a block: bf16, for 16 of its rows and all columns; fp32, for two registers (two rows each)
template <typename T, int DP>
struct Columns {
    using TL = Tile<T, DP>;
    static constexpr int DT = HeadShape<T, DP>::DT;
    static constexpr int kSteps = sizeof(T) == 2 ? 2 : 8;        // parts of a block
    using Operand = std::conditional_t<sizeof(T) == 2, xu32x4_t, xu32x2_t>;
    Operand f[DT];
    __device__ __forceinline__ void read(const char* tile, int row0, int lane, int step) {
        const int l32 = lane & 31, g = lane >> 5;
        const char* const base = tile + row0 * TL::kPitch;
        if constexpr (sizeof(T) == 2) {
            const int row = 8 * g + ((lane & 15) >> 2), c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), in = 8 * (lane & 1);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                f[dt] = transposed_chunk(base + step * 16 * TL::kPitch + TL::at(row, 4 * dt + c) + in, base + step * 16 * TL::kPitch + TL::at(row + 4, 4 * dt + c) + in);
        } else {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    f[dt][e] = *reinterpret_cast<const uint32_t*>(base + register_row<T>(2 * step + e, g) * TL::kPitch + (32 * dt + l32) * 4);
        }
    }
    // o[d, column] += the part's rows times s, whose registers the part has
    __device__ __forceinline__ void multiply(const xf32x16_t& s, int step, xf32x16_t (&o)[DT]) const {
        if constexpr (sizeof(T) == 2) {
            const int h = 8 * step;
            const xu32x4_t pk = pack8({s[h], s[h + 1], s[h + 2], s[h + 3], s[h + 4], s[h + 5], s[h + 6], s[h + 7]});
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) chunk_product<T>(f[dt], pk, o[dt]);
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(f[dt][e]), s[2 * step + e], o[dt], 0, 0, 0);
        }
    }
};

// o[d, column] += sum over the 32 rows from row0 on of tile[row, d] s[row, column], the first part's operands in c
template <typename T, int DP, bool kAhead = true>
__device__ __forceinline__ void column_products(const char* tile, int row0, int lane, Columns<T, DP>& c, const xf32x16_t& s,
                                                xf32x16_t (&o)[HeadShape<T, DP>::DT]) {
#pragma unroll
    for (int step = 0; step < Columns<T, DP>::kSteps; ++step) {
        Columns<T, DP> next;
        if (step + 1 < Columns<T, DP>::kSteps) {
            next.read(tile, row0, lane, step + 1);
            if constexpr (kAhead) fence();
        }
        c.multiply(s, step, o);
        c = next;
    }
}

// Tiles of two tensors' rows (keys and values; queries and their gradients) one after the other in LDS, bf16 rows of whole chunks, NW wavefronts: block
// of 1 KB w, w + NW, ... of both is wavefront w's, so that every wavefront has as many loads in flight and a wait counts tiles.
template <int DP, int NW>
struct PairRing {
    using TL = Tile<bf16_t, DP>;
    static constexpr int kBlocks = TL::kRows * TL::kPitch / 1024, kSecond = kBlocks * 1024, N = (2 * kBlocks + NW - 1) / NW, kTileBytes = N * NW * 1024;
    int off[N];                      // of this lane's chunks in a tile, bytes behind the tile's first row
    // place(second, r): where row r of a tile is
    template <typename Place>
    __device__ __forceinline__ void aim(int wave, int lane, int dh, Place&& place) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int block = wave + NW * i, second = block >= kBlocks ? 1 : 0, slot = (block - second * kBlocks) * 64 + lane;
            const int row = slot / TL::CHP, c = (slot % TL::CHP) ^ TL::turn(row);
            off[i] = block < 2 * kBlocks && c * 8 < dh ? place(second, row) + c * 16 : kNowhere;
            asm volatile("" : "+v"(off[i]));     // (kept, not computed again for every tile)
        }
    }
    __device__ __forceinline__ void request(const u32x4_t& first, const u32x4_t& second, uint32_t tile, int wave) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int block = wave + NW * i;
            dma_1k(tile + block * 1024, off[i], block >= kBlocks ? second : first, 0);
        }
    }
};

// Kernels with a PairRing: as many wavefronts, and tiles under way while one is multiplied: requested one ahead, a tile arrives later than the products of
// another take.
constexpr int kRing = 3, kRingWaves = 8, kMaxTiles = 16;
constexpr int kLdsBytes = 160 * 1024 - 256;
// Two workgroups of kPassWaves share a compute unit where tiles pass through: one is busy while the other brings or stores its rows.  Tiles of each in LDS
// (with two, one is under way while one is multiplied).
constexpr int kPassWaves = 4;
template <int DP>
constexpr int kPassTiles = (kLdsBytes / 2 - kOverRead) / PairRing<DP, kPassWaves>::kTileBytes >= 3 ? 3 : 2;

// 64 floats, one per lane, to LDS (dma_1k's comment)
__device__ __forceinline__ void dma_floats(uint32_t lds_addr, int voff, u32x4_t rsrc) {
    asm volatile("s_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "{m0}"(lds_addr), "v"(voff), "s"(rsrc));
}

// rows [first, first + rows) of a tensor as a buffer
__device__ __forceinline__ u32x4_t rows_rsrc(const bf16_t* p, int64_t first, int64_t rows, int64_t stride, int width) {
    return make_rsrc(p + first * stride, rows > 0 ? ((rows - 1) * stride + width) * 2 : 0);
}

// the keys of sample b that can count
__device__ __forceinline__ int attended(const CrossArgs& a, int b) {
    if (!a.key_len) return a.Nk;
    const int n = a.key_len[b];
    return n < 0 ? 0 : n < a.Nk ? n : a.Nk;
}

// Keys and values of a (sample, key head) for the kernels with a PairRing
template <int DP, int NW = kRingWaves>
struct RingKeys {
    using TL = Tile<bf16_t, DP>;
    using Ring = PairRing<DP, NW>;
    const bf16_t *kp, *vp;
    const uint8_t* mask;
    int64_t k_stride, v_stride;
    int len, dh;
    Ring ring;
    __device__ __forceinline__ RingKeys(const CrossArgs& a, int b, int kvh, int wave, int lane)
        : kp(static_cast<const bf16_t*>(a.k) + static_cast<int64_t>(b) * a.Nk * a.k_stride + static_cast<int64_t>(kvh) * a.dh),
          vp(static_cast<const bf16_t*>(a.v) + static_cast<int64_t>(b) * a.Nk * a.v_stride + static_cast<int64_t>(kvh) * a.dh),
          mask(a.key_mask ? a.key_mask + static_cast<int64_t>(b) * a.Nk : nullptr), k_stride(a.k_stride), v_stride(a.v_stride), len(attended(a, b)), dh(a.dh) {
        ring.aim(wave, lane, dh, [&](int second, int r) { return r * static_cast<int>(second ? v_stride : k_stride) * 2; });
    }
    __device__ __forceinline__ int tiles() const { return (len + TL::kRows - 1) / TL::kRows; }
    __device__ __forceinline__ void request(int t, uint32_t tile, int wave) const {
        const int64_t first = static_cast<int64_t>(t) * TL::kRows;
        ring.request(rows_rsrc(kp, first, len - first, k_stride, dh), rows_rsrc(vp, first, len - first, v_stride, dh), tile, wave);
    }
    // which of tile t's keys count; with a mask it waits for memory
    __device__ __forceinline__ uint64_t valid(int t, int lane) const {
        const int key = t * TL::kRows + lane;
        return mask ? __ballot(key < len && mask[key] != 0) : keys_below(len - t * TL::kRows);
    }
    // rows of keys that do not count are replaced, in LDS, where they are multiplied by zeros and may be NaN: the keys' (second 0) or the values'
    static __device__ __forceinline__ void drop(char* tile, int second, uint64_t valid, int wave, int lane) {
        if (valid == ~0ull) return;
        for (int r = wave; r < TL::kRows; r += NW)
            if (!(valid >> r & 1) && lane < TL::CHP) *reinterpret_cast<xu32x4_t*>(tile + second * Ring::kSecond + r * TL::kPitch + lane * 16) = xu32x4_t{0, 0, 0, 0};
    }
};

// Resident keys: all tiles to LDS, masks[t] their bits; whether any key counts.  Ends with a barrier.
template <int DP>
__device__ __forceinline__ bool bring_keys(const RingKeys<DP>& keys, char* lds, uint64_t (&masks)[kMaxTiles], int drop_second, int wave, int lane) {
    using Ring = typename RingKeys<DP>::Ring;
    const int tiles = keys.tiles();
    bool any = tiles > 0;
    if (keys.mask) {
        for (int t = wave; t < tiles; t += kRingWaves) {
            const uint64_t bits = keys.valid(t, lane);
            if (lane == 0) masks[t] = bits;
        }
    }
    wait_vm_barrier<0>();
    if (keys.mask) {
        any = false;
        for (int t = 0; t < tiles; ++t) {
            const uint64_t valid = masks[t];
            any |= valid != 0;
            keys.drop(lds + t * Ring::kTileBytes, drop_second, valid, wave, lane);
        }
        __syncthreads();
    }
    return any;
}

template <int DP>
constexpr int ring_tiles() { return (kLdsBytes - kOverRead) / PairRing<DP, kRingWaves>::kTileBytes; }

// LDS of a kernel with `tiles` tiles of a PairRing, whose last one ends with the second tensor's rows
template <int DP, int NW>
constexpr size_t ring_bytes(int tiles) {
    using Ring = PairRing<DP, NW>;
    static_assert(Ring::kSecond + Tile<bf16_t, DP>::columns_end() <= Ring::kTileBytes + kOverRead, "columns of the last tile's second tensor");
    return static_cast<size_t>(tiles) * Ring::kTileBytes + kOverRead;
}
inline int tiles_that_fit(int32_t dh) {
    return std::min(kMaxTiles, dh <= 32 ? ring_tiles<32>() : dh <= 64 ? ring_tiles<64>() : dh <= 80 ? ring_tiles<80>() : dh <= 96 ? ring_tiles<96>() : ring_tiles<128>());
}

// (sample, key head) and place in it of a workgroup: an XCD has heads that are next to each other, and the same place of them at a time - rows of 144 bytes
// share lines
struct WorkPlace {
    int pair, place;
    __device__ __forceinline__ WorkPlace(int id, int pairs) {
        const bool by_xcd = pairs % kXcds == 0;
        const int per = by_xcd ? pairs / kXcds : pairs, at = by_xcd ? id / kXcds : id;
        pair = (by_xcd ? id % kXcds * per : 0) + at % per;
        place = at / per;
    }
};

// Keys and values of a (sample, key head), tile by tile, and which of a tile's keys count.  The mask of a tile is requested a tile ahead of its rows.
template <typename T, int DP, bool kVec>
struct KeyStream {
    using TL = Tile<T, DP>;
    TileStream<T, DP, kVec> k, v;
    const T *kp, *vp;
    const uint8_t* mask;
    int k_row, v_row, len, dh;
    uint32_t mask_byte = 1;
    __device__ __forceinline__ KeyStream(const CrossArgs& a, int b, int kvh)
        : kp(static_cast<const T*>(a.k) + static_cast<int64_t>(b) * a.Nk * a.k_stride + static_cast<int64_t>(kvh) * a.dh),
          vp(static_cast<const T*>(a.v) + static_cast<int64_t>(b) * a.Nk * a.v_stride + static_cast<int64_t>(kvh) * a.dh),
          mask(a.key_mask ? a.key_mask + static_cast<int64_t>(b) * a.Nk : nullptr),
          k_row(static_cast<int>(a.k_stride)), v_row(static_cast<int>(a.v_stride)), len(attended(a, b)), dh(a.dh) {}
    __device__ __forceinline__ int tiles() const { return (len + TL::kRows - 1) / TL::kRows; }
    __device__ __forceinline__ void request_mask(int t, int lane) {
        if (mask) mask_byte = lane < len - t * TL::kRows ? mask[t * TL::kRows + lane] : 0;
    }
    // of the tile whose mask was requested last
    __device__ __forceinline__ uint64_t valid_of(int t) const {
        const uint64_t v = keys_below(min(len - t * TL::kRows, TL::kRows));
        return mask ? v & __ballot(mask_byte != 0) : v;
    }
    __device__ __forceinline__ void request(int t, uint32_t tile_k, uint32_t tile_v, int wave, int lane, uint64_t valid) {
        constexpr int ES = static_cast<int>(sizeof(T));
        const int64_t first = static_cast<int64_t>(t) * TL::kRows, rows = len - first;
        k.request(kp + first * k_row, ((rows - 1) * k_row + dh) * ES, tile_k, wave, lane, dh, mask != nullptr, valid, [&](int r) { return r * k_row * ES; });
        v.request(vp + first * v_row, ((rows - 1) * v_row + dh) * ES, tile_v, wave, lane, dh, mask != nullptr, valid, [&](int r) { return r * v_row * ES; });
    }
    __device__ __forceinline__ void deliver(char* tile_k, char* tile_v, int tid, uint64_t valid) {
        k.deliver(tile_k, tid, mask != nullptr, valid);
        v.deliver(tile_v, tid, mask != nullptr, valid);
    }
};

}  // namespace

// cross_attn.hip, cross_attn_grad.hip; arguments checked in cond_abi.hip
size_t cross_forward_bytes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype);
size_t cross_backward_bytes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype);
int32_t launch_cross_forward(const CrossArgs& a, int32_t dtype, void* ws, hipStream_t s);
int32_t launch_cross_backward(const CrossArgs& a, int32_t dtype, void* ws, hipStream_t s);

}  // namespace freemi
