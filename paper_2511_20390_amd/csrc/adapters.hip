// A shared projection with the low-rank adapters of many requests beside it, and the gradient that fits adapters.  Row m belongs to request
// m / rows_per_sample, which has adapter a of n (or none):
//   t = s_a x A_a^T [M, r],   out = x W^T + bias + t B_a^T
//   u = s_a dout B_a [M, r],  dx = dout W + u A_a,   dA_a = sum over the adapter's rows of u^T x,   dB_a = sum of dout^T t
// (s: a scale per adapter; W is shared and keeps still).  Requests come in any order: wherever a kernel has a block of rows, it takes the
// adapters of these rows one after the other, with the other rows masked.
//  * t and u: x (dout) is read once, 16 or 32 rows per workgroup whose wavefronts share K; rounded to the type of the product they are
//    operands of, like the hidden values of the gated block.  Bound by reading x and, for each block of rows, its adapter again from the L2: 12288 x 1152,
//    rank 16, 8.6 us (3.3 TB/s); 4100 x 4096, rank 64, 26.
//  * out and dx: the kernels and tiles of the linear layers, whose sums begin with the adapters' (bf16, adapter_term.h: 12288 rows of 1152 to 1152, 34 us; 8192
//    of 1152 to 4608, 86 and back 95, 1.01 and 0.92 PFLOP/s; what bounds them is in gemm_pipe.hip), or a second pass over the result (fp32: 1000 rows of
//    384 to 1536, 17 and 8.4 us); few rows ffn_rows.hip (8 rows of 4096 to 4096: 7.6, 4.4 TB/s).  The tiles
//    of the gated block, which read W by its columns as well, took 489 against 345 for both passes of 4100 rows of 4096 to 4096.
//  * dA and dB: 128 columns of x or dout by all ranks per workgroup, over the rows of one adapter, in parts that a second launch adds in
//    order.  Rows of other adapters are not read, but every (columns, adapter, part) stores its part, zeros where no row is the adapter's.  8192 rows of
//    1152 and 4608, rank 32, 3 adapters: 27 us, the reading of x and dout at 3.5 TB/s, and 5.6 for the parts; 4100 of 4096 and 4096, rank 64, 6 adapters: 34
//    and 10, 67 MB read at 2 TB/s beside 38 MB of parts.
// For the gradient W, B and A are needed the other way round ([K][N], [rank][N], [K][rank]): copies of that layout go into the workspace, filled
// up with zeros to whole slices (4096 x 4096 of 6 adapters of rank 64: 17 us).
#include <algorithm>

#include "adapter_term.h"
#include "cross_attn.h"
#include "ffn_mfma.h"
#include "free_internal.h"
#include "row_pieces.h"

namespace freemi {

namespace {

constexpr int kThreads = 256;
constexpr int kDownWaves = 8;
constexpr int kTileRows = 64;                    // token rows of a tile of the weights' gradients
constexpr int kMasks = 512;                      // tiles whose rows are looked over at once

int32_t up_to(int32_t v, int32_t step) { return (v + step - 1) / step * step; }

// ---- t, u
struct DownArgs {
    const void *x, *w;                           // x [M, K]; w [adapter][w_rows][K]
    const int32_t* adapter;
    const float* scale;                          // nullable
    void* out;                                   // [M][t_row], zeros from r on
    int32_t M, K, n_adapters, w_rows, r, t_row, rows_per_sample;
    float* zeros = nullptr;                      // nullable: zero_n values to clear, a bias for the product behind
    int32_t zero_n = 0;
};

// Workgroup (block of 16 MT rows, j, 16 RT ranks): the j-th adapter of the block's rows, in the order they come.  A workgroup more than the block has
// adapters ends at once: how many it has is on the device.
template <typename T, int MT, int RT, bool kEdge>
__global__ __launch_bounds__(kDownWaves * 64) void adapter_down_kernel(DownArgs a) {
    constexpr int P = 2, E = 16 / sizeof(T), kStep = 4 * P * E, U = MT * RT == 1 ? 8 : MT * RT == 2 ? 4 : 2;      // steps in flight
    __shared__ f32x4a_t red[kDownWaves][RT * MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // blocks of rows next to each other on one XCD: its L2 has the adapters of few requests to hold
    const int m0 = xcd_tile(blockIdx.x, gridDim.x) * 16 * MT, rank0 = blockIdx.z * 16 * RT, quad = lane >> 4, r16 = lane & 15;
    if (a.zeros && blockIdx.y == 0 && blockIdx.z == 0)       // (a grid of 2^22 workgroups has 2^31 threads)
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * kDownWaves * 64 + threadIdx.x; i < a.zero_n; i += static_cast<int64_t>(gridDim.x) * kDownWaves * 64) a.zeros[i] = 0.f;
    int of = -1;                                 // lane: row m0 + lane's adapter
    if (lane < 16 * MT && m0 + lane < a.M) {
        const int id = a.adapter[(m0 + lane) / a.rows_per_sample];
        of = id >= 0 && id < a.n_adapters ? id : -1;
    }
    int which = -1;
    uint64_t left = __ballot(of >= 0);
    for (int j = 0; left != 0; ++j) {
        which = __builtin_amdgcn_readlane(of, __builtin_ctzll(left));
        if (j == static_cast<int>(blockIdx.y)) break;
        left &= ~__ballot(of == which);
    }
    if (left == 0) return;
    const uint64_t mine = __ballot(of == which);
    const float scale = a.scale ? a.scale[which] : 1.0f;
    const int at = quad * E;                     // of a step's 128 bytes: piece p is 64 p bytes on, so that 4 lanes read 64 bytes
    const T* w[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int rank = rank0 + t * 16 + r16;
        w[t] = static_cast<const T*>(a.w) + (static_cast<int64_t>(which) * a.w_rows + (rank < a.r ? rank : a.r - 1)) * a.K + at;
    }
    const T* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int row = mine >> (t * 16 + r16) & 1 ? t * 16 + r16 : __builtin_ctzll(mine);      // (other adapters' rows are not read)
        x[t] = static_cast<const T*>(a.x) + static_cast<int64_t>(m0 + row) * a.K + at;
    }
    f32x4a_t acc[RT][MT];
#pragma unroll
    for (int b = 0; b < RT; ++b)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[b][t] = f32x4a_t{0.f, 0.f, 0.f, 0.f};
    const int steps = (a.K + kStep - 1) / kStep;
    for (int s0 = wave; s0 < steps; s0 += kDownWaves * U) {
        u32x4_t wv[U][RT][P], xv[U][MT][P];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * kDownWaves;
            if (s >= steps) continue;
            const int64_t k = static_cast<int64_t>(s) * kStep;
            const bool whole = !kEdge || k + kStep <= a.K;
            const int rest = static_cast<int>(a.K - k) - at;
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int p = 0; p < P; ++p) load_piece(x[t] + k + p * 4 * E, rest - p * 4 * E, xv[u][t][p], whole);
#pragma unroll
            for (int b = 0; b < RT; ++b)
#pragma unroll
                for (int p = 0; p < P; ++p) load_piece(w[b] + k + p * 4 * E, rest - p * 4 * E, wv[u][b][p], whole);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u * kDownWaves >= steps) continue;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int b = 0; b < RT; ++b)
#pragma unroll
                    for (int t = 0; t < MT; ++t) multiply<T>(wv[u][b][p], xv[u][t][p], acc[b][t]);
        }
    }
#pragma unroll
    for (int b = 0; b < RT; ++b)
#pragma unroll
        for (int t = 0; t < MT; ++t) red[wave][b * MT + t][lane] = acc[b][t];
    __syncthreads();
    // value i: token i / (16 RT), rank i % (16 RT); it stands in lane token + 16 (rank / 4), register rank % 4
    for (int i = threadIdx.x; i < MT * 16 * RT * 16; i += kDownWaves * 64) {
        const int row = i / (16 * RT), c = i % (16 * RT), t = row / 16, b = c / 16, from = row % 16 + 16 * (c % 16 / 4);
        if (!(mine >> row & 1) || rank0 + c >= a.t_row) continue;
        float v = red[0][b * MT + t][from][c & 3];
#pragma unroll
        for (int k = 1; k < kDownWaves; ++k) v += red[k][b * MT + t][from][c & 3];
        store_f(static_cast<T*>(a.out) + static_cast<int64_t>(m0 + row) * a.t_row + rank0 + c, rank0 + c < a.r ? v * scale : 0.f);
    }
}

template <typename T, int MT, int RT>
int32_t launch_down_shape(const DownArgs& a, hipStream_t s) {
    const int32_t block = 16 * MT, rows = std::min(block, a.M);
    // adapters that a block of rows can have
    int32_t most = a.rows_per_sample >= a.M || a.rows_per_sample % block == 0 ? 1 : std::min(rows, (rows - 1) / a.rows_per_sample + 2);
    most = std::min(most, a.n_adapters);
    const dim3 grid((a.M + block - 1) / block, most, (a.t_row + 16 * RT - 1) / (16 * RT));
    constexpr int kStep = 128 / sizeof(T);
    if (a.K % kStep == 0) hipLaunchKernelGGL((adapter_down_kernel<T, MT, RT, false>), grid, dim3(kDownWaves * 64), 0, s, a);
    else hipLaunchKernelGGL((adapter_down_kernel<T, MT, RT, true>), grid, dim3(kDownWaves * 64), 0, s, a);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <typename T, int MT>
int32_t launch_down_ranks(const DownArgs& a, hipStream_t s) {
    // more ranks per workgroup read x less often, but few workgroups leave compute units without work: 7 rows of 4096 in fp32, rank 62, 34 us with 64
    // ranks and 13 with 16; 244 in bf16, rank 64, 20.6 and 9.1 (1 and 16 blocks; from where on 32 and 64 ranks pay is not measured closer)
    const int32_t blocks = (a.M + 16 * MT - 1) / (16 * MT);
    if (a.t_row <= 16 || blocks < 64) return launch_down_shape<T, MT, 1>(a, s);
    if (a.t_row <= 32 || blocks < 128) return launch_down_shape<T, MT, 2>(a, s);
    return launch_down_shape<T, MT, 4>(a, s);
}

template <typename T>
int32_t launch_down(const DownArgs& a, hipStream_t s) {
    // 32 rows read an adapter half as often: 4100 x 4096, rank 64, 26 us against 38 with 16
    return a.M <= 16 * 128 ? launch_down_ranks<T, 1>(a, s) : launch_down_ranks<T, 2>(a, s);
}

// ---- W, B and A the other way round
struct TurnJob {
    const void* src;                             // [n][rows][cols]
    void* dst;                                   // [n][cols_to][rows_to], zeros past cols and rows
    int32_t rows, cols, rows_to, cols_to, n;
    int32_t tiles;                               // of 64 x 64, of all n
};
struct TurnJobs {
    TurnJob job[3];
};

// A tile of 64 x 64 values through LDS, 16 bytes per thread in and out, at any address
template <typename T>
__global__ __launch_bounds__(kThreads) void adapter_turn_kernel(TurnJobs jobs) {
    constexpr int E = 16 / sizeof(T), C = 64 / E;
    __shared__ T tile[64][64 + 2];
    int id = blockIdx.x, k = 0;
    while (k < 2 && id >= jobs.job[k].tiles) id -= jobs.job[k++].tiles;
    const TurnJob& j = jobs.job[k];
    const int tiles_r = (j.rows_to + 63) / 64, tiles_c = (j.cols_to + 63) / 64, which = id / (tiles_r * tiles_c), at = id % (tiles_r * tiles_c);
    const int r0 = at / tiles_c * 64, c0 = at % tiles_c * 64;
    const T* const src = static_cast<const T*>(j.src) + static_cast<int64_t>(which) * j.rows * j.cols;
    T* const dst = static_cast<T*>(j.dst) + static_cast<int64_t>(which) * j.rows_to * j.cols_to;
#pragma unroll
    for (int i = threadIdx.x; i < 64 * C; i += kThreads) {
        const int r = r0 + i / C, c = c0 + i % C * E;
        u32x4_t v = {0, 0, 0, 0};
        if (r < j.rows) load_piece(src + static_cast<int64_t>(r) * j.cols + c, j.cols - c, v, false);
        T t[E];
        __builtin_memcpy(t, &v, 16);
#pragma unroll
        for (int e = 0; e < E; ++e) tile[i / C][i % C * E + e] = t[e];
    }
    __syncthreads();
#pragma unroll
    for (int i = threadIdx.x; i < 64 * C; i += kThreads) {
        const int c = c0 + i / C, r = r0 + i % C * E;
        if (c >= j.cols_to || r >= j.rows_to) continue;
        T t[E];
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = tile[i % C * E + e][i / C];
        T* const to = dst + static_cast<int64_t>(c) * j.rows_to + r;
        if (r + E <= j.rows_to) {
            __builtin_memcpy(to, t, 16);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (r + e < j.rows_to) to[e] = t[e];
        }
    }
}

// ---- fp32: out += t B^T; a wavefront has 32 x 32 values
__global__ __launch_bounds__(kThreads) void adapter_up_kernel(AdapterTerm ad, int32_t M, float* out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, g = lane >> 5;
    const int n0 = (blockIdx.x * 4 + wave) * 32, N = ad.cols;
    if (n0 >= N) return;
    const bool whole = ad.b_row % 4 == 0 && (reinterpret_cast<uintptr_t>(ad.b) & 15u) == 0;
    for (int64_t m0 = static_cast<int64_t>(blockIdx.y) * 32; m0 < M; m0 += static_cast<int64_t>(gridDim.y) * 32) {
        const int m = static_cast<int>(m0) + l32;
        xf32x16_t acc;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int n = n0 + 8 * (e >> 2) + 4 * g + (e & 3);
            acc[e] = m < M && n < N ? out[static_cast<int64_t>(m) * N + n] : 0.f;
        }
        int of = m < M ? ad.of_row(m) : -1;
        for (uint64_t left = __ballot(of >= 0); left != 0; left = __ballot(of >= 0)) {
            const int which = __builtin_amdgcn_readlane(of, __builtin_ctzll(left));
            const int n = n0 + l32 < N ? n0 + l32 : N - 1;
            const float* const b = static_cast<const float*>(ad.b) + (static_cast<int64_t>(which) * N + n) * ad.b_row;
            const float* const t = static_cast<const float*>(ad.t) + static_cast<int64_t>(m < M ? m : M - 1) * ad.t_row;
            xf32x16_t sum;               // (of its own: an infinite or NaN adapter stays out of the other rows)
            clear_tile(sum);
            for (int k0 = 0; k0 < ad.r; k0 += 8) {
                const int k = k0 + 4 * g;
                xu32x4_t tv = {0, 0, 0, 0}, bv = {0, 0, 0, 0};
                if (of == which) tv = *reinterpret_cast<const xu32x4_t*>(t + k);
                if (whole) {
                    if (k < ad.r) bv = *reinterpret_cast<const xu32x4_t*>(b + k);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) bv[e] = k + e < ad.r ? __float_as_uint(b[k + e]) : 0u;
                }
                chunk_product<float>(bv, tv, sum);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] += of == which ? sum[e] : 0.f;
            of = of == which ? -1 : of;
        }
        if (m < M) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int n = n0 + 8 * (e >> 2) + 4 * g + (e & 3);
                if (n < N) out[static_cast<int64_t>(m) * N + n] = acc[e];
            }
        }
    }
}

// ---- dA, dB
struct SumArgs {
    const void* wide[2];                         // x, dout: [M][ld]
    const void* thin[2];                         // u, t: [M][t_row]
    int64_t ld[2];
    int32_t cols[2];                             // K, N
    int32_t tiles[2];                            // of 128 columns
    void* out[2];                                // dA [n][r][K], dB [n][N][r]
    float* part;                                 // parts > 1: per part the values of both results, in their order
    const int32_t* adapter;
    int32_t M, n_adapters, r, t_row, rows_per_sample, parts, part_tiles;
};

// Where chunk c of a row is, so that neither the stores nor the transposing reads of 4 rows x 64 bytes share banks.  Rows of 256, 128 or 64
// bytes (whose four rows are next to each other).
template <int kPitch>
__device__ __forceinline__ int chunk_place(int row, int c) {
    const int turn = kPitch == 256 ? (row & 3) << 2 | (row >> 2 & 3) : kPitch == 128 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : 0;
    return row * kPitch + ((c ^ turn) << 4);
}

// bytes of a stage of adapter_sum_kernel: tiles of 64 rows of 128 columns, and of the ranks
constexpr int sum_stage(int rb) { return kTileRows * (256 + rb * 64); }

// RB: blocks of 32 ranks.  Workgroup (columns, adapter, part): a wavefront has 32 columns.
template <typename T, int RB>
__global__ __launch_bounds__(kThreads) void adapter_sum_kernel(SumArgs a) {
    constexpr int kThinPitch = RB * 64, kThinChunks = RB * 4, kLoads = kTileRows * 16 / kThreads, kThinLoads = kTileRows * kThinChunks / kThreads;
    __shared__ uint64_t masks[kMasks];
    extern __shared__ __attribute__((aligned(16))) char lds[];          // bf16: [stage][wide, thin]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, g = lane >> 5;
    const int col_tiles = a.tiles[0] + a.tiles[1];
    const int ct = blockIdx.x % col_tiles, which = blockIdx.x / col_tiles % a.n_adapters, part = blockIdx.x / col_tiles / a.n_adapters;
    const bool second = ct >= a.tiles[0];
    const T* const wide = static_cast<const T*>(second ? a.wide[1] : a.wide[0]);
    const T* const thin = static_cast<const T*>(second ? a.thin[1] : a.thin[0]);
    const int64_t ld = second ? a.ld[1] : a.ld[0];
    const int cols = second ? a.cols[1] : a.cols[0], c0 = (second ? ct - a.tiles[0] : ct) * 128;
    const int tiles = (a.M + kTileRows - 1) / kTileRows, first = part * a.part_tiles, last = min(first + a.part_tiles, tiles);
    xf32x16_t acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) clear_tile(acc[b]);
    for (int base = first; base < last; base += kMasks) {
        // which rows of the tiles are this adapter's
        const int count = min(last - base, kMasks);
        if (base > first) __syncthreads();
        for (int i = wave; i < count; i += 4) {
            const int64_t m = static_cast<int64_t>(base + i) * kTileRows + lane;
            const uint64_t bits = __ballot(m < a.M && a.adapter[(m < a.M ? m : 0) / a.rows_per_sample] == which);
            if (lane == 0) masks[i] = bits;
        }
        __syncthreads();
        const auto next = [&](int i) {
            while (i < count && masks[i] == 0) ++i;
            return i;
        };
        if constexpr (sizeof(T) == 2) {
            u32x4_t wv[kLoads], tv[kThinLoads];
            const auto fetch = [&](int i) {
                const uint64_t bits = masks[i];
                const int64_t m0 = static_cast<int64_t>(base + i) * kTileRows;
#pragma unroll
                for (int k = 0; k < kLoads; ++k) {
                    const int row = (tid + k * kThreads) / 16, c = (tid + k * kThreads) % 16;
                    wv[k] = u32x4_t{0, 0, 0, 0};
                    if ((bits >> row & 1) && c0 + c * 8 < cols) wv[k] = *reinterpret_cast<const u32x4_t*>(wide + (m0 + row) * ld + c0 + c * 8);
                }
#pragma unroll
                for (int k = 0; k < kThinLoads; ++k) {
                    const int row = (tid + k * kThreads) / kThinChunks, c = (tid + k * kThreads) % kThinChunks;
                    tv[k] = u32x4_t{0, 0, 0, 0};
                    if ((bits >> row & 1) && c * 8 < a.t_row) tv[k] = *reinterpret_cast<const u32x4_t*>(thin + (m0 + row) * a.t_row + c * 8);
                }
            };
            const auto stash = [&](int stage) {
                char* const to = lds + stage * sum_stage(RB);
#pragma unroll
                for (int k = 0; k < kLoads; ++k)
                    *reinterpret_cast<u32x4_t*>(to + chunk_place<256>((tid + k * kThreads) / 16, (tid + k * kThreads) % 16)) = wv[k];
#pragma unroll
                for (int k = 0; k < kThinLoads; ++k)
                    *reinterpret_cast<u32x4_t*>(to + kTileRows * 256 + chunk_place<kThinPitch>((tid + k * kThreads) / kThinChunks, (tid + k * kThreads) % kThinChunks)) = tv[k];
            };
            // transposing reads: 8 consecutive rows of a column per lane (cross_attn.h)
            const int row = 8 * g + ((lane & 15) >> 2), in_c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), in = 8 * (lane & 1);
            const auto column = [&](const char* tile, auto pitch, int ks, int block) {
                constexpr int kPitch = decltype(pitch)::value;
                const char* const p = tile + ks * 16 * kPitch + in;
                return transposed_chunk(p + chunk_place<kPitch>(row, 4 * block + in_c), p + chunk_place<kPitch>(row + 4, 4 * block + in_c));
            };
            int i = next(0), stage = 0;
            if (i < count) fetch(i);
            while (i < count) {
                stash(stage);
                i = next(i + 1);
                if (i < count) fetch(i);
                __syncthreads();
                const char* const tile = lds + stage * sum_stage(RB);
                const std::integral_constant<int, 256> wide_pitch{};
                const std::integral_constant<int, kThinPitch> thin_pitch{};
#pragma unroll
                for (int ks = 0; ks < kTileRows / 16; ++ks) {
                    const xu32x4_t w = column(tile, wide_pitch, ks, wave);
#pragma unroll
                    for (int b = 0; b < RB; ++b) chunk_product<T>(w, column(tile + kTileRows * 256, thin_pitch, ks, b), acc[b]);
                }
                stage ^= 1;
            }
        } else {
            constexpr int kPairs = RB == 1 ? 32 : RB == 2 ? 16 : 8;        // row pairs whose loads are in flight together
            const int col = min(c0 + wave * 32 + l32, cols - 1);
            int rank[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) rank[b] = min(b * 32 + l32, a.t_row - 1);
            for (int i = next(0); i < count; i = next(i + 1)) {
                const uint64_t bits = masks[i];
                const int own = __builtin_ctzll(bits);
                const int64_t m0 = static_cast<int64_t>(base + i) * kTileRows;
                // (rows of other adapters: one of this adapter's is read again and zeros multiply)
#pragma unroll
                for (int k0 = 0; k0 < kTileRows / 2; k0 += kPairs) {
                    float wv[kPairs], tv[RB][kPairs];
#pragma unroll
                    for (int k = 0; k < kPairs; ++k) {
                        const int row = 2 * (k0 + k) + g, from = bits >> row & 1 ? row : own;
                        wv[k] = wide[(m0 + from) * ld + col];
#pragma unroll
                        for (int b = 0; b < RB; ++b) tv[b][k] = thin[(m0 + from) * a.t_row + rank[b]];
                    }
#pragma unroll
                    for (int k = 0; k < kPairs; ++k) {
                        const bool on = bits >> (2 * (k0 + k) + g) & 1;
#pragma unroll
                        for (int b = 0; b < RB; ++b)
                            acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(on ? wv[k] : 0.f, on ? tv[b][k] : 0.f, acc[b], 0, 0, 0);
                    }
                }
            }
        }
    }
    // register e: column 8 (e / 4) + 4 g + e % 4 of the wavefront's, rank 32 b + l32
    const int64_t values = static_cast<int64_t>(a.cols[0] + a.cols[1]) * a.r * a.n_adapters;
    const int64_t first_value = second ? static_cast<int64_t>(a.cols[0]) * a.r * a.n_adapters : 0;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int rank = b * 32 + l32;
        if (rank >= a.r) continue;
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const int col = c0 + wave * 32 + 8 * e4 + 4 * g;
            const float v[4] = {acc[b][4 * e4], acc[b][4 * e4 + 1], acc[b][4 * e4 + 2], acc[b][4 * e4 + 3]};
            const int64_t at = second ? (static_cast<int64_t>(which) * cols + col) * a.r + rank : (static_cast<int64_t>(which) * a.r + rank) * cols + col;
            const int64_t step = second ? a.r : 1;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (col + c >= cols) continue;
                if (a.parts > 1) a.part[part * values + first_value + at + c * step] = v[c];
                else store_f(static_cast<T*>(second ? a.out[1] : a.out[0]) + at + c * step, v[c]);
            }
        }
    }
}

// the parts, added in order: a thread per value
template <typename T>
__global__ __launch_bounds__(kThreads) void adapter_join_kernel(SumArgs a) {
    const int64_t values = static_cast<int64_t>(a.cols[0] + a.cols[1]) * a.r * a.n_adapters, first = static_cast<int64_t>(a.cols[0]) * a.r * a.n_adapters;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= values) return;
    float v = a.part[i];
#pragma unroll 4
    for (int k = 1; k < a.parts; ++k) v += a.part[k * values + i];
    store_f(i < first ? static_cast<T*>(a.out[0]) + i : static_cast<T*>(a.out[1]) + (i - first), v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void adapter_clear_kernel(T* p, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) p[i] = T{};
}

// ---- sizes, workspaces, launches
struct Sizes {
    int32_t M, K, N, r, n;
    int32_t Kp, Np;                              // K and N in whole slices of a sum
    int32_t t_row;
    size_t es;
    Sizes(int32_t m, int32_t k, int32_t nn, int32_t rank, int32_t adapters, int32_t dtype)
        : M(m), K(k), N(nn), r(rank), n(adapters), t_row(up_to(rank, 16)), es(dtype == FREE_BF16 ? 2 : 4) {
        const int32_t slice = es == 2 ? 64 : 32;
        Kp = up_to(k, slice);
        Np = up_to(nn, slice);
    }
    // few rows' kernel: as for the gated block, and all it takes in fp32, where tiles of 64 rows spend their time on empty ones (28 rows of 4096 to 4096
    // with 64 ranks: 73 -> 32 us)
    bool few() const { return ffn_rows_pay(M, K, N, K != Kp) || (es == 4 && M <= 32); }
    bool few_back() const { return ffn_rows_pay(M, Np, K, false) || (es == 4 && M <= 32); }
    size_t thin_bytes() const { return static_cast<size_t>(M) * t_row * es; }
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

template <typename T>
struct ForwardSpace {
    T *t, *x, *w;
    float* zeros;                                // in place of a bias
    size_t bytes;
    ForwardSpace(const Sizes& z, char* base) {
        Carve c{base};
        t = c.take<T>(z.thin_bytes());
        zeros = c.take<float>(static_cast<size_t>(z.N) * sizeof(float));
        x = w = nullptr;
        if (!z.few() && z.K != z.Kp) {
            x = c.take<T>(static_cast<size_t>(z.M) * z.Kp * sizeof(T));
            w = c.take<T>(static_cast<size_t>(z.N) * z.Kp * sizeof(T));
        }
        bytes = c.at + 256;
    }
};

// Parts of the rows of the weights' gradients: workgroups for the chip, at least 4 tiles of 64 rows each (fp32, whose rows take longer: 2).
struct SumPlan {
    int32_t parts, part_tiles;
    explicit SumPlan(const Sizes& z) {
        const int64_t tiles = std::max<int64_t>(1, (static_cast<int64_t>(z.M) + kTileRows - 1) / kTileRows);
        const int64_t groups = (static_cast<int64_t>(z.K + 127) / 128 + (z.N + 127) / 128) * z.n;
        const int64_t want = std::max<int64_t>(1, std::min({(1024 + groups - 1) / groups, tiles / (z.es == 2 ? 4 : 2), static_cast<int64_t>(64)}));
        part_tiles = static_cast<int32_t>((tiles + want - 1) / want);
        parts = static_cast<int32_t>((tiles + part_tiles - 1) / part_tiles);
    }
};

template <typename T>
struct BackwardSpace {
    T *u, *wt, *bt, *at, *x, *dout;
    float *zeros, *part;
    size_t bytes;
    BackwardSpace(const Sizes& z, char* base) {
        Carve c{base};
        u = c.take<T>(z.thin_bytes());
        wt = c.take<T>(static_cast<size_t>(z.K) * z.Np * sizeof(T));
        bt = c.take<T>(static_cast<size_t>(z.n) * z.t_row * z.Np * sizeof(T));
        at = c.take<T>(static_cast<size_t>(z.n) * z.K * z.t_row * sizeof(T));
        zeros = c.take<float>(static_cast<size_t>(z.K) * sizeof(float));
        const SumPlan sum(z);
        part = c.take<float>(sum.parts > 1 ? static_cast<size_t>(sum.parts) * z.n * (z.K + z.N) * z.r * sizeof(float) : 0);
        x = dout = nullptr;
        // (rows of x in 16-byte pieces for dA; rows of dout in whole slices for dx)
        if (z.K % (16 / sizeof(T)) != 0) x = c.take<T>(static_cast<size_t>(z.M) * z.Kp * sizeof(T));
        if (z.N != z.Np) dout = c.take<T>(static_cast<size_t>(z.M) * z.Np * sizeof(T));
        bytes = c.at + 256;
    }
};

#define FREE_STEP(call)                     \
    do {                                    \
        const int32_t st_ = (call);         \
        if (st_ != FREE_OK) return st_;     \
    } while (0)

// out [M, term.cols] = x w^T + bias and the adapters', K whole slices
template <typename T>
int32_t linear_with(const T* x, const T* w, const float* bias, int32_t M, int32_t K, const AdapterTerm& term, T* out, hipStream_t s) {
    if constexpr (sizeof(T) == 2) {
        return launch_linear_adapters(x, w, bias, M, term.cols, K, out, term, s);
    } else {
        FREE_STEP(launch_linear_f32(x, w, bias, M, term.cols, K, FREE_EPI_BIAS, out, nullptr, RowVec{nullptr, 0, 1}, s));
        const dim3 grid((term.cols + 127) / 128, std::min((M + 31) / 32, 65535));
        hipLaunchKernelGGL(adapter_up_kernel, grid, dim3(kThreads), 0, s, term, M, out);
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;
    }
}

template <typename T>
int32_t forward_of(const Sizes& z, const AdapterArgs& a, char* ws, hipStream_t s) {
    const ForwardSpace<T> w(z, ws);
    T* const t = a.saved ? static_cast<T*>(a.saved) : w.t;
    const T *x = static_cast<const T*>(a.x), *weight = static_cast<const T*>(a.w);
    T* const out = static_cast<T*>(a.out);
    DownArgs down{x, a.a, a.adapter, a.scale, t, z.M, z.K, z.n, z.r, z.r, z.t_row, a.rows_per_sample};
    if (!a.bias && !z.few()) {
        down.zeros = w.zeros;
        down.zero_n = z.N;
    }
    FREE_STEP(launch_down<T>(down, s));
    const AdapterTerm term{t, a.b, a.adapter, a.bias, z.n, z.r, z.t_row, z.r, z.N, a.rows_per_sample};
    if (z.few()) return launch_adapter_rows<T>(x, weight, z.M, z.N, z.K, term, out, s);
    if (z.K != z.Kp) {
        FREE_STEP(launch_fit<T>(x, z.M, z.K, w.x, z.M, z.Kp, s));
        FREE_STEP(launch_fit<T>(weight, z.N, z.K, w.w, z.N, z.Kp, s));
        x = w.x;
        weight = w.w;
    }
    return linear_with<T>(x, weight, a.bias ? a.bias : w.zeros, z.M, z.Kp, term, out, s);
}

template <typename T, int RB>
int32_t launch_sum(const SumArgs& a, hipStream_t s) {
    const int64_t blocks = static_cast<int64_t>(a.tiles[0] + a.tiles[1]) * a.n_adapters * a.parts;
    if (blocks > 0x7fffffff) return FREE_ERR_LIMIT;
    const size_t lds = sizeof(T) == 2 ? 2 * sum_stage(RB) : 0;
    auto kern = adapter_sum_kernel<T, RB>;
    static LdsLimit limit;
    if (!limit.allow(reinterpret_cast<const void*>(kern), lds)) return FREE_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), lds, s, a);
    if (!launch_ok()) return FREE_ERR_HIP;
    if (a.parts == 1) return FREE_OK;
    const int64_t values = static_cast<int64_t>(a.cols[0] + a.cols[1]) * a.r * a.n_adapters;
    hipLaunchKernelGGL(adapter_join_kernel<T>, dim3(static_cast<uint32_t>((values + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, a);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <typename T>
int32_t clear(void* p, int64_t n, hipStream_t s) {
    const int64_t blocks = std::min<int64_t>((n + kThreads - 1) / kThreads, 4096);
    hipLaunchKernelGGL(adapter_clear_kernel<T>, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, s, static_cast<T*>(p), n);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <typename T>
int32_t backward_of(const Sizes& z, const AdapterArgs& a, char* ws, hipStream_t s) {
    if (z.M == 0) {                                      // empty sums
        FREE_STEP(clear<T>(a.da, static_cast<int64_t>(z.n) * z.r * z.K, s));
        return clear<T>(a.db, static_cast<int64_t>(z.n) * z.r * z.N, s);
    }
    const BackwardSpace<T> w(z, ws);
    const T *x = static_cast<const T*>(a.x), *dout = static_cast<const T*>(a.dout);
    if (w.x) {
        FREE_STEP(launch_fit<T>(x, z.M, z.K, w.x, z.M, z.Kp, s));
        x = w.x;
    }
    if (w.dout) {
        FREE_STEP(launch_fit<T>(dout, z.M, z.N, w.dout, z.M, z.Np, s));
        dout = w.dout;
    }
    TurnJobs jobs{{{a.w, w.wt, z.N, z.K, z.Np, z.K, 1, 0}, {a.b, w.bt, z.N, z.r, z.Np, z.t_row, z.n, 0}, {a.a, w.at, z.r, z.K, z.t_row, z.K, z.n, 0}}};
    int64_t tiles = 0;
    for (TurnJob& j : jobs.job) {
        const int64_t n = static_cast<int64_t>((j.rows_to + 63) / 64) * ((j.cols_to + 63) / 64) * j.n;
        tiles += n;
        if (tiles > 0x7fffffff) return FREE_ERR_LIMIT;
        j.tiles = static_cast<int32_t>(n);
    }
    hipLaunchKernelGGL(adapter_turn_kernel<T>, dim3(static_cast<uint32_t>(tiles)), dim3(kThreads), 0, s, jobs);
    if (!launch_ok()) return FREE_ERR_HIP;
    DownArgs down{dout, w.bt, a.adapter, a.scale, w.u, z.M, z.Np, z.n, z.t_row, z.r, z.t_row, a.rows_per_sample, w.zeros, z.K};
    FREE_STEP(launch_down<T>(down, s));
    const AdapterTerm term{w.u, w.at, a.adapter, nullptr, z.n, z.t_row, z.t_row, z.t_row, z.K, a.rows_per_sample};
    if (z.few_back()) FREE_STEP(launch_adapter_rows<T>(dout, w.wt, z.M, z.K, z.Np, term, static_cast<T*>(a.dx), s));
    else FREE_STEP(linear_with<T>(dout, w.wt, w.zeros, z.M, z.Np, term, static_cast<T*>(a.dx), s));
    const SumPlan plan(z);
    const SumArgs sum{{x, dout}, {w.u, a.saved}, {w.x ? z.Kp : z.K, z.Np}, {z.K, z.N}, {(z.K + 127) / 128, (z.N + 127) / 128}, {a.da, a.db}, w.part, a.adapter, z.M,
                      z.n, z.r, z.t_row, a.rows_per_sample, plan.parts, plan.part_tiles};
    if (z.t_row <= 32) return launch_sum<T, 1>(sum, s);
    if (z.t_row <= 64) return launch_sum<T, 2>(sum, s);
    return launch_sum<T, 4>(sum, s);
}

}  // namespace

// 32-bit byte offsets inside a tile of 384 rows, grids of less than 2^32 threads
bool adapters_cover(int32_t M, int32_t K, int32_t N, int32_t r, int32_t n, int32_t dtype) {
    if (M > 1 << 27 || K > 1 << 20 || N > 1 << 20 || r > 128 || n > 16384) return false;
    if (static_cast<int64_t>(K) * N > int64_t{1} << 34 || (static_cast<int64_t>(K) + N + 128) * n > 1 << 28) return false;
    const int64_t m = (static_cast<int64_t>(M) + 127) / 128, k = (K + 127) / 128, c = (N + 127) / 128;
    return std::max(m * k, m * c) <= (dtype == FREE_FP32 ? 1 << 20 : 1 << 22) && (static_cast<int64_t>(K) + N) * r * n <= int64_t{1} << 36;
}

size_t adapters_saved_bytes(int32_t M, int32_t r, int32_t dtype) { return static_cast<size_t>(M) * up_to(r, 16) * (dtype == FREE_BF16 ? 2 : 4) + 256; }

size_t adapters_workspace_bytes(int32_t M, int32_t K, int32_t N, int32_t r, int32_t n, int32_t dtype, bool backward) {
    const Sizes z(M, K, N, r, n, dtype);
    const size_t f = z.es == 2 ? ForwardSpace<bf16_t>(z, nullptr).bytes : ForwardSpace<float>(z, nullptr).bytes;
    const size_t b = z.es == 2 ? BackwardSpace<bf16_t>(z, nullptr).bytes : BackwardSpace<float>(z, nullptr).bytes;
    return (backward ? std::max(f, b) : f) / 256 * 256 + 256;
}

int32_t launch_adapters_forward(const AdapterArgs& a, int32_t M, int32_t K, int32_t N, int32_t r, int32_t n, int32_t dtype, void* ws, hipStream_t s) {
    const Sizes z(M, K, N, r, n, dtype);
    return dtype == FREE_BF16 ? forward_of<bf16_t>(z, a, static_cast<char*>(ws), s) : forward_of<float>(z, a, static_cast<char*>(ws), s);
}

int32_t launch_adapters_backward(const AdapterArgs& a, int32_t M, int32_t K, int32_t N, int32_t r, int32_t n, int32_t dtype, void* ws, hipStream_t s) {
    const Sizes z(M, K, N, r, n, dtype);
    return dtype == FREE_BF16 ? backward_of<bf16_t>(z, a, static_cast<char*>(ws), s) : backward_of<float>(z, a, static_cast<char*>(ws), s);
}

}  // namespace freemi
