// The gradient of cross attention (cross_attn.hip), from its inputs, its result and lse:
//   P = exp(scale q k^T - lse) on the keys that count,  delta = sum dout out,  dS = P (dout v^T - delta)
//   dq = scale dS k,   dk = scale dS^T q,   dv = P^T dout      (dk, dv: summed over the queries of all heads that share them)
// Nothing of the size of the scores is kept between the passes: both kernels compute their tiles of scores again.
//  * dq: a workgroup has 128 rows (query and head of a group) and passes tiles of K and V through LDS; it also leaves delta for
//  * dk, dv: a workgroup has 128 or 64 keys and passes tiles of q and dout through LDS, so that both sums stay in registers.
// The score tile's rows are the streamed tensor's rows and its columns the workgroup's own (cross_attn.h), in both.
// Where a launch would have few workgroups the streamed axis is cut in parts, whose fp32 results a second launch adds in order: no
// atomics, equal inputs give equal bits.
// A streamed tile is read by rows (16 bytes of a row per lane: scores) and by columns (transposing reads: the last product), so bf16 rows
// of 128 or 256 bytes have their chunks at places that keep both off each other's banks (Tile::at).
#include <algorithm>
#include <cmath>

#include "cross_attn.h"

namespace freemi {

namespace {

constexpr int kThreads = 256;

// A tile in LDS, rows of CH chunks
template <typename T, int DP>
struct Tile {
    using H = HeadShape<T, DP>;
    static constexpr int kRows = sizeof(T) == 2 ? 64 : 32;
    static constexpr int kPitch = sizeof(T) == 4 ? (H::CH | 1) * 16 : DP <= 64 ? 128 : 256;
    static constexpr int kBytes = kRows * kPitch + (sizeof(T) == 4 ? 128 : 0);        // (fp32: columns past a row's end are read)
    static constexpr int kLoads = (kRows * H::CH + kThreads - 1) / kThreads;
    // where chunk c of a row is.  256-byte rows: 16 rows of one c on 16 places, and the four rows and chunks of a transposing read too;
    // 128-byte rows: the same of two rows that share 256 bytes.
    static __device__ __forceinline__ int turn(int row) {
        if constexpr (sizeof(T) == 4) return 0;
        else if constexpr (kPitch == 256) return (row & 3) << 2 | (row >> 2 & 3);
        else return (row >> 1 & 1) << 2 | (row >> 2 & 3);
    }
    static __device__ __forceinline__ int at(int row, int c) { return row * kPitch + ((c ^ turn(row)) << 4); }
};

// acc += (32 rows of the tile from row0 on) . own, rows of scores in block_row's order
template <typename T, int DP>
__device__ __forceinline__ void tile_scores(const char* tile, int row0, int lane, const xu32x4_t (&own)[HeadShape<T, DP>::KSTEPS], xf32x16_t& acc) {
    const int row = block_row<T>(lane & 31), g = lane >> 5;
    const char* const base = tile + row0 * Tile<T, DP>::kPitch;
#pragma unroll
    for (int ks = 0; ks < HeadShape<T, DP>::KSTEPS; ++ks)
        chunk_product<T>(*reinterpret_cast<const xu32x4_t*>(base + Tile<T, DP>::at(row, 2 * ks + g)), own[ks], acc);
}

// o[d, column] += sum over the 32 rows from row0 on of tile[row, d] s[row, column]
template <typename T, int DP>
__device__ __forceinline__ void tile_sums(const char* tile, int row0, int lane, const xf32x16_t& s, xf32x16_t (&o)[HeadShape<T, DP>::DT]) {
    using TL = Tile<T, DP>;
    constexpr int DT = HeadShape<T, DP>::DT;
    const int l32 = lane & 31, g = lane >> 5;
    const char* const base = tile + row0 * TL::kPitch;
    if constexpr (sizeof(T) == 2) {
        const int row = 8 * g + ((lane & 15) >> 2), c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), in = 8 * (lane & 1);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const xu32x4_t pk = pack8({s[8 * hh], s[8 * hh + 1], s[8 * hh + 2], s[8 * hh + 3], s[8 * hh + 4], s[8 * hh + 5], s[8 * hh + 6], s[8 * hh + 7]});
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                chunk_product<T>(transposed_chunk(base + hh * 16 * TL::kPitch + TL::at(row, 4 * dt + c) + in,
                                                  base + hh * 16 * TL::kPitch + TL::at(row + 4, 4 * dt + c) + in), pk, o[dt]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const float x = *reinterpret_cast<const float*>(base + register_row<T>(e, g) * TL::kPitch + (32 * dt + l32) * 4);
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[e], o[dt], 0, 0, 0);
            }
    }
}

__device__ __forceinline__ int attended(const CrossArgs& a, int b) {
    if (!a.key_len) return a.Nk;
    const int n = a.key_len[b];
    return n < 0 ? 0 : n < a.Nk ? n : a.Nk;
}

// parts of the streamed axis: tiles of each; fp32 results [part][pair][row][dh]
struct GradParts {
    int32_t parts, tiles;
    float *sum0, *sum1;
};

// ---- dq and delta
template <typename T, int DP, bool kVec>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 || DP <= 64) ? 2 : 1) void cross_dq_kernel(CrossArgs a, float* delta, GradParts pt, int32_t q_tiles) {
    using H = HeadShape<T, DP>;
    using TL = Tile<T, DP>;
    constexpr int CH = H::CH, KSTEPS = H::KSTEPS, DT = H::DT, BKV = TL::kRows;
    extern __shared__ __attribute__((aligned(16))) char lds[];          // [stage][K, V]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int pairs = a.B * a.kv_heads, group = a.heads / a.kv_heads;
    const int per_part = pairs * q_tiles;
    const int part = blockIdx.x / per_part, id = blockIdx.x % per_part;
    const bool by_xcd = pairs % kXcds == 0;          // the query tiles of a (sample, head) on one XCD
    const int pair = by_xcd ? id % kXcds + kXcds * (id / (kXcds * q_tiles)) : id / q_tiles;
    const int q_tile = by_xcd ? id / kXcds % q_tiles : id % q_tiles;
    const int kvh = pair % a.kv_heads, b = pair / a.kv_heads;
    const int64_t rows = static_cast<int64_t>(a.Nq) * group;
    const int64_t row = static_cast<int64_t>(q_tile) * 128 + wave * 32 + l32;
    const int len = attended(a, b);
    const int t0 = part * pt.tiles, t1 = min(t0 + pt.tiles, (len + BKV - 1) / BKV);

    const T* const kp = static_cast<const T*>(a.k) + static_cast<int64_t>(b) * a.Nk * a.k_stride + static_cast<int64_t>(kvh) * a.dh;
    const T* const vp = static_cast<const T*>(a.v) + static_cast<int64_t>(b) * a.Nk * a.v_stride + static_cast<int64_t>(kvh) * a.dh;
    const uint8_t* const mask = a.key_mask ? a.key_mask + static_cast<int64_t>(b) * a.Nk : nullptr;
    const int k_row = static_cast<int>(a.k_stride) * static_cast<int>(sizeof(T)), v_row = static_cast<int>(a.v_stride) * static_cast<int>(sizeof(T));
    xu32x4_t kreg[TL::kLoads], vreg[TL::kLoads];
    uint32_t mask_next = 1;
    const auto fetch = [&](int t) {
        const int64_t kv0 = static_cast<int64_t>(t) * BKV;
        const auto kb = rows_buffer(kp + kv0 * a.k_stride, len - kv0, a.k_stride, a.dh), vb = rows_buffer(vp + kv0 * a.v_stride, len - kv0, a.v_stride, a.dh);
#pragma unroll
        for (int i = 0; i < TL::kLoads; ++i) {
            const int idx = tid + kThreads * i, r = idx / CH, c = idx % CH;
            if (idx < BKV * CH) {
                kreg[i] = buffer_chunk<T, kVec>(kb, r * k_row + c * 16, c, a.dh);
                vreg[i] = buffer_chunk<T, kVec>(vb, r * v_row + c * 16, c, a.dh);
            }
        }
        if (mask) mask_next = kv0 + lane < len ? mask[kv0 + lane] : 0;
    };
    const auto valid_of = [&](int t) {
        const uint64_t v = keys_below(min(len - t * BKV, BKV));
        return mask ? v & __ballot(mask_next != 0) : v;
    };
    const auto stash = [&](int stage, uint64_t valid) {
        char* const sK = lds + stage * 2 * TL::kBytes;
#pragma unroll
        for (int i = 0; i < TL::kLoads; ++i) {
            const int idx = tid + kThreads * i, r = idx / CH, c = idx % CH;
            if (idx < BKV * CH) {
                if (mask && !(valid >> r & 1)) kreg[i] = xu32x4_t{0, 0, 0, 0};       // (multiplied by zeros: NaN must not get there)
                *reinterpret_cast<xu32x4_t*>(sK + TL::at(r, c)) = kreg[i];
                *reinterpret_cast<xu32x4_t*>(sK + TL::kBytes + TL::at(r, c)) = vreg[i];
            }
        }
    };
    if (t0 < t1) fetch(t0);

    const int64_t q_row = row < rows ? row : rows - 1, token = q_row / group;
    const int head = kvh * group + static_cast<int>(q_row - token * group);
    const int64_t q_at = static_cast<int64_t>(b) * a.Nq + token, h_at = static_cast<int64_t>(head) * a.dh;
    const int64_t stat = (static_cast<int64_t>(b) * a.heads + head) * a.Nq + token;
    xu32x4_t qf[KSTEPS], gf[KSTEPS];
    float dl = 0.f;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
        qf[ks] = row_chunk<T, kVec>(static_cast<const T*>(a.q) + q_at * a.q_stride + h_at, 2 * ks + g, a.dh);
        gf[ks] = row_chunk<T, kVec>(static_cast<const T*>(a.dout) + q_at * a.dout_stride + h_at, 2 * ks + g, a.dh);
        const xu32x4_t of = row_chunk<T, kVec>(static_cast<const T*>(a.out) + q_at * a.out_stride + h_at, 2 * ks + g, a.dh);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) {
                dl = fmaf(__uint_as_float(gf[ks][e] << 16), __uint_as_float(of[e] << 16), dl);
                dl = fmaf(__uint_as_float(gf[ks][e] & 0xffff0000u), __uint_as_float(of[e] & 0xffff0000u), dl);
            } else {
                dl = fmaf(__uint_as_float(gf[ks][e]), __uint_as_float(of[e]), dl);
            }
        }
    }
    dl = add_lane_xor<32>(dl);
    const float lse2 = a.lse[stat] * kLog2e, scale_log2 = a.scale * kLog2e;
    if (part == 0 && g == 0 && row < rows) delta[stat] = dl;

    xf32x16_t dq[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) clear_tile(dq[dt]);
    uint64_t valid = 0;
    if (t0 < t1) {
        valid = valid_of(t0);
        stash(0, valid);
        if (t0 + 1 < t1) fetch(t0 + 1);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int stage = (t - t0) & 1;
        const char* const sK = lds + stage * 2 * TL::kBytes;
        uint64_t valid_next = 0;
        if (t + 1 < t1) {
            valid_next = valid_of(t + 1);
            stash(stage ^ 1, valid_next);
            if (t + 2 < t1) fetch(t + 2);
        }
#pragma unroll
        for (int kb = 0; kb < BKV / 32; ++kb) {
            xf32x16_t st, dp;
            clear_tile(st);
            clear_tile(dp);
            tile_scores<T, DP>(sK, kb * 32, lane, qf, st);
            tile_scores<T, DP>(sK + TL::kBytes, kb * 32, lane, gf, dp);
            const uint32_t bits = static_cast<uint32_t>(valid >> (32 * kb)) >> (sizeof(T) == 2 ? 8 * g : 4 * g);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float ds = __builtin_amdgcn_exp2f(fmaf(st[e], scale_log2, -lse2)) * (dp[e] - dl);
                st[e] = bits >> register_row<T>(e, 0) & 1 ? ds : 0.f;
            }
            tile_sums<T, DP>(sK, kb * 32, lane, st, dq);
        }
        valid = valid_next;
        __syncthreads();
    }
    if (row >= rows) return;
    if (pt.parts > 1) {
        float* const dst = pt.sum0 + ((part * static_cast<int64_t>(pairs) + pair) * rows + row) * a.dh;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                store4<float, false>(dst, 32 * dt + 8 * e4 + 4 * g, a.dh, dq[dt][4 * e4], dq[dt][4 * e4 + 1], dq[dt][4 * e4 + 2], dq[dt][4 * e4 + 3]);
        return;
    }
    T* const dst = static_cast<T*>(a.dq) + q_at * a.dq_stride + h_at;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
            store4<T, kVec>(dst, 32 * dt + 8 * e4 + 4 * g, a.dh, dq[dt][4 * e4] * a.scale, dq[dt][4 * e4 + 1] * a.scale, dq[dt][4 * e4 + 2] * a.scale,
                            dq[dt][4 * e4 + 3] * a.scale);
}

// ---- dk and dv.  KW wavefronts have 32 keys each; with KW 2 the two halves of a tile's rows go to two wavefronts, whose sums are parts of
// their own.
template <typename T, int DP, int KW, bool kVec>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 && DP <= 80) || DP <= 32 ? 2 : 1) void cross_dkv_kernel(CrossArgs a, const float* delta, GradParts pt, int32_t k_tiles) {
    using H = HeadShape<T, DP>;
    using TL = Tile<T, DP>;
    constexpr int CH = H::CH, KSTEPS = H::KSTEPS, DT = H::DT, BR = TL::kRows, QW = 4 / KW, RB = BR / 32 / QW;
    static_assert(RB >= 1, "a block of rows for each wavefront");
    extern __shared__ __attribute__((aligned(16))) char lds[];          // [stage][q, dout], then [stage][lse, delta][BR]
    float* const stats = reinterpret_cast<float*>(lds + 4 * TL::kBytes);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int kw = wave % KW, qw = wave / KW;
    const int pairs = a.B * a.kv_heads, group = a.heads / a.kv_heads;
    // the key tiles of a (sample, head, part) read the same rows: one XCD, next to each other
    const int units = pairs * (pt.parts / QW);
    const bool by_xcd = units % kXcds == 0;
    const int unit = by_xcd ? blockIdx.x % kXcds + kXcds * (blockIdx.x / (kXcds * k_tiles)) : blockIdx.x / k_tiles;
    const int k_tile = by_xcd ? blockIdx.x / kXcds % k_tiles : blockIdx.x % k_tiles;
    const int part = unit / pairs, pair = unit % pairs;
    const int kvh = pair % a.kv_heads, b = pair / a.kv_heads;
    const int64_t rows = static_cast<int64_t>(a.Nq) * group;
    const int key = k_tile * 32 * KW + kw * 32 + l32;
    const int len = attended(a, b);
    const int64_t tiles = (rows + BR - 1) / BR;
    const int64_t t0 = static_cast<int64_t>(part) * pt.tiles;
    // keys that do not count have no gradient: a workgroup without others has nothing to sum
    const int64_t t1 = k_tile * 32 * KW < len ? min(t0 + pt.tiles, tiles) : t0;
    const bool there = key < len && (!a.key_mask || a.key_mask[static_cast<int64_t>(b) * a.Nk + key] != 0);

    const int q_row = static_cast<int>(a.q_stride) * static_cast<int>(sizeof(T)), g_row = static_cast<int>(a.dout_stride) * static_cast<int>(sizeof(T));
    const int head_bytes = a.dh * static_cast<int>(sizeof(T));
    const int64_t first_row = static_cast<int64_t>(b) * a.Nq, h0 = static_cast<int64_t>(kvh) * group * a.dh;
    xu32x4_t qreg[TL::kLoads], greg[TL::kLoads];
    float lse_next = 0.f, delta_next = 0.f;
    const auto fetch = [&](int64_t t) {
        const int64_t r0 = t * BR, token0 = r0 / group;
        const int rest = static_cast<int>(r0 - token0 * group);         // of the group's heads: row r0 + r is token0 + (rest + r) / group
        const auto qb = rows_buffer(static_cast<const T*>(a.q) + (first_row + token0) * a.q_stride + h0, a.Nq - token0, a.q_stride, group * a.dh);
        const auto gb = rows_buffer(static_cast<const T*>(a.dout) + (first_row + token0) * a.dout_stride + h0, a.Nq - token0, a.dout_stride, group * a.dh);
#pragma unroll
        for (int i = 0; i < TL::kLoads; ++i) {
            const int idx = tid + kThreads * i, r = idx / CH, c = idx % CH;
            if (idx < BR * CH) {
                const int token = (rest + r) / group, h = rest + r - token * group;
                qreg[i] = buffer_chunk<T, kVec>(qb, token * q_row + h * head_bytes + c * 16, c, a.dh);
                greg[i] = buffer_chunk<T, kVec>(gb, token * g_row + h * head_bytes + c * 16, c, a.dh);
            }
        }
        if (tid < BR) {
            const int64_t token = token0 + (rest + tid) / group;
            const int64_t at = (static_cast<int64_t>(b) * a.heads + kvh * group + (rest + tid) % group) * a.Nq + token;
            const bool on = r0 + tid < rows;
            lse_next = on ? a.lse[at] * kLog2e : INFINITY;              // (rows past the end: probabilities of zero)
            delta_next = on ? delta[at] : 0.f;
        }
    };
    const auto stash = [&](int stage) {
        char* const sQ = lds + stage * 2 * TL::kBytes;
#pragma unroll
        for (int i = 0; i < TL::kLoads; ++i) {
            const int idx = tid + kThreads * i, r = idx / CH, c = idx % CH;
            if (idx < BR * CH) {
                *reinterpret_cast<xu32x4_t*>(sQ + TL::at(r, c)) = qreg[i];
                *reinterpret_cast<xu32x4_t*>(sQ + TL::kBytes + TL::at(r, c)) = greg[i];
            }
        }
        if (tid < BR) {
            stats[stage * 2 * BR + tid] = lse_next;
            stats[stage * 2 * BR + BR + tid] = delta_next;
        }
    };
    if (t0 < t1) fetch(t0);

    const int64_t kv_at = static_cast<int64_t>(b) * a.Nk + (key < a.Nk ? key : 0), h_at = static_cast<int64_t>(kvh) * a.dh;
    xu32x4_t kf[KSTEPS], vf[KSTEPS];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
        kf[ks] = vf[ks] = xu32x4_t{0, 0, 0, 0};
        if (there) {
            kf[ks] = row_chunk<T, kVec>(static_cast<const T*>(a.k) + kv_at * a.k_stride + h_at, 2 * ks + g, a.dh);
            vf[ks] = row_chunk<T, kVec>(static_cast<const T*>(a.v) + kv_at * a.v_stride + h_at, 2 * ks + g, a.dh);
        }
    }
    const float scale_log2 = a.scale * kLog2e;
    xf32x16_t dk[DT], dv[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        clear_tile(dk[dt]);
        clear_tile(dv[dt]);
    }
    if (t0 < t1) {
        stash(0);
        if (t0 + 1 < t1) fetch(t0 + 1);
    }
    __syncthreads();
    for (int64_t t = t0; t < t1; ++t) {
        const int stage = static_cast<int>(t - t0) & 1;
        const char* const sQ = lds + stage * 2 * TL::kBytes;
        if (t + 1 < t1) {
            stash(stage ^ 1);
            if (t + 2 < t1) fetch(t + 2);
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row0 = (qw * RB + rb) * 32;
            xf32x16_t st, dp;
            clear_tile(st);
            clear_tile(dp);
            tile_scores<T, DP>(sQ, row0, lane, kf, st);
            tile_scores<T, DP>(sQ + TL::kBytes, row0, lane, vf, dp);
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const float* const at = stats + stage * 2 * BR + row0 + register_row<T>(4 * e4, g);
                const xf32x4_t lse = *reinterpret_cast<const xf32x4_t*>(at), dl = *reinterpret_cast<const xf32x4_t*>(at + BR);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = 4 * e4 + i;
                    st[e] = __builtin_amdgcn_exp2f(fmaf(st[e], scale_log2, -lse[i]));
                    dp[e] = st[e] * (dp[e] - dl[i]);
                }
            }
            tile_sums<T, DP>(sQ + TL::kBytes, row0, lane, st, dv);
            tile_sums<T, DP>(sQ, row0, lane, dp, dk);
        }
        __syncthreads();
    }
    if (key >= a.Nk) return;
    // (what a key that does not count has got are sums over zeros in place of it, not a gradient)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            dk[dt][e] = there ? dk[dt][e] : 0.f;
            dv[dt][e] = there ? dv[dt][e] : 0.f;
        }
    if (pt.parts > 1) {
        const int64_t at = (((part * QW + qw) * static_cast<int64_t>(pairs) + pair) * a.Nk + key) * a.dh;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const int d = 32 * dt + 8 * e4 + 4 * g;
                store4<float, false>(pt.sum0 + at, d, a.dh, dk[dt][4 * e4], dk[dt][4 * e4 + 1], dk[dt][4 * e4 + 2], dk[dt][4 * e4 + 3]);
                store4<float, false>(pt.sum1 + at, d, a.dh, dv[dt][4 * e4], dv[dt][4 * e4 + 1], dv[dt][4 * e4 + 2], dv[dt][4 * e4 + 3]);
            }
        return;
    }
    T* const dkp = static_cast<T*>(a.dk) + kv_at * a.dk_stride + h_at;
    T* const dvp = static_cast<T*>(a.dv) + kv_at * a.dv_stride + h_at;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const int d = 32 * dt + 8 * e4 + 4 * g;
            store4<T, kVec>(dkp, d, a.dh, dk[dt][4 * e4] * a.scale, dk[dt][4 * e4 + 1] * a.scale, dk[dt][4 * e4 + 2] * a.scale, dk[dt][4 * e4 + 3] * a.scale);
            store4<T, kVec>(dvp, d, a.dh, dv[dt][4 * e4], dv[dt][4 * e4 + 1], dv[dt][4 * e4 + 2], dv[dt][4 * e4 + 3]);
        }
}

// The parts of a sum, added in order, times `factor`: a thread per value.  Row r of a pair is token r / group, head r % group of the pair's.
template <typename T>
__global__ __launch_bounds__(kThreads) void cross_sum_kernel(const float* parts, int32_t n, int64_t pairs, int32_t kv_heads, int32_t tokens, int32_t group, int32_t dh,
                                                             float factor, T* out, int64_t stride) {
    const int64_t rows = static_cast<int64_t>(tokens) * group, all = pairs * rows * dh;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= all) return;
    float s = parts[i];
    for (int p = 1; p < n; ++p) s += parts[p * all + i];
    const int64_t at = i / dh, pair = at / rows, r = at % rows, token = r / group;
    const int64_t head = pair % kv_heads * group + (r - token * group);
    store_f(out + (pair / kv_heads * tokens + token) * stride + head * dh + i % dh, s * factor);
}

template <typename T>
int32_t launch_sum(const float* parts, int32_t n, const CrossArgs& a, int32_t tokens, int32_t group, float factor, void* out, int64_t stride, hipStream_t s) {
    const int64_t pairs = static_cast<int64_t>(a.B) * a.kv_heads, all = pairs * tokens * group * a.dh;
    hipLaunchKernelGGL(cross_sum_kernel<T>, dim3(static_cast<uint32_t>((all + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, parts, n, pairs, a.kv_heads, tokens,
                       group, a.dh, factor, static_cast<T*>(out), stride);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

// How the two launches are cut; by the sizes alone
struct Plan {
    int32_t q_parts, q_part_tiles;
    int64_t q_tiles;
    int kw;
    int32_t k_parts, k_part_tiles;                // (parts: those of the wavefronts counted)
    int64_t k_tiles;
};
constexpr int kUnits = 256;

Plan plan_of(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dtype) {
    const int64_t pairs = static_cast<int64_t>(B) * kv_heads, rows = static_cast<int64_t>(Nq) * (heads / kv_heads);
    const int tile = dtype == FREE_BF16 ? 64 : 32;
    const auto cut = [](int64_t work, int64_t tiles, int64_t least, int64_t* parts, int64_t* per) {
        *parts = std::min<int64_t>(std::max<int64_t>(1, std::min(2 * kUnits / std::max<int64_t>(work, 1), tiles / least)), 64);
        *per = (tiles + *parts - 1) / *parts;
        *parts = (tiles + *per - 1) / *per;
    };
    Plan p{};
    int64_t parts, per;
    p.q_tiles = std::max<int64_t>(1, (rows + 127) / 128);
    cut(pairs * p.q_tiles, std::max<int64_t>(1, (static_cast<int64_t>(Nk) + tile - 1) / tile), 4, &parts, &per);
    p.q_parts = static_cast<int32_t>(parts);
    p.q_part_tiles = static_cast<int32_t>(per);
    p.kw = dtype == FREE_BF16 && Nk <= 64 ? 2 : 4;
    p.k_tiles = std::max<int64_t>(1, (static_cast<int64_t>(Nk) + 32 * p.kw - 1) / (32 * p.kw));
    cut(pairs * p.k_tiles, std::max<int64_t>(1, (rows + tile - 1) / tile), 4, &parts, &per);
    p.k_parts = static_cast<int32_t>(parts * (4 / p.kw));
    p.k_part_tiles = static_cast<int32_t>(per);
    return p;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

struct Space {
    size_t delta, dq, dk, dv, bytes;              // offsets
    Space(const Plan& p, int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh) {
        delta = 0;
        // the parts of dq and those of dk, dv take turns
        dq = dk = up256(static_cast<size_t>(B) * heads * Nq * sizeof(float));
        const size_t q = p.q_parts > 1 ? static_cast<size_t>(p.q_parts) * B * Nq * heads * dh * sizeof(float) : 0;
        const size_t kv = p.k_parts > 1 ? up256(static_cast<size_t>(p.k_parts) * B * Nk * kv_heads * dh * sizeof(float)) : 0;
        dv = dk + kv;
        bytes = dq + std::max(up256(q), 2 * kv) + 256;
    }
};

template <typename T, int DP, bool kVec>
int32_t launch_shape(const CrossArgs& a, const Plan& p, const Space& w, char* ws, hipStream_t s) {
    using TL = Tile<T, DP>;
    const int64_t pairs = static_cast<int64_t>(a.B) * a.kv_heads;
    const int64_t q_blocks = pairs * p.q_tiles * p.q_parts, k_blocks = pairs * p.k_tiles * (p.k_parts / (4 / p.kw));
    if (q_blocks > 0x7fffffff || k_blocks > 0x7fffffff) return FREE_ERR_LIMIT;
    float* const delta = reinterpret_cast<float*>(ws + w.delta);
    const int32_t group = a.heads / a.kv_heads;
    {
        const GradParts pt{p.q_parts, p.q_part_tiles, reinterpret_cast<float*>(ws + w.dq), nullptr};
        auto kern = cross_dq_kernel<T, DP, kVec>;
        const size_t lds = 4 * TL::kBytes;
        static LdsLimit limit;
        if (!limit.allow(reinterpret_cast<const void*>(kern), lds)) return FREE_ERR_HIP;
        hipLaunchKernelGGL(kern, dim3(static_cast<uint32_t>(q_blocks)), dim3(kThreads), lds, s, a, delta, pt, static_cast<int32_t>(p.q_tiles));
        if (!launch_ok()) return FREE_ERR_HIP;
        if (p.q_parts > 1) {
            const int32_t st = launch_sum<T>(pt.sum0, p.q_parts, a, a.Nq, group, a.scale, a.dq, a.dq_stride, s);
            if (st != FREE_OK) return st;
        }
    }
    const GradParts pt{p.k_parts, p.k_part_tiles, reinterpret_cast<float*>(ws + w.dk), reinterpret_cast<float*>(ws + w.dv)};
    const size_t lds = 4 * TL::kBytes + 4 * TL::kRows * sizeof(float);
    const auto launch = [&](auto kw) {
        auto kern = cross_dkv_kernel<T, DP, decltype(kw)::value, kVec>;
        static LdsLimit limit;
        if (!limit.allow(reinterpret_cast<const void*>(kern), lds)) return FREE_ERR_HIP;
        hipLaunchKernelGGL(kern, dim3(static_cast<uint32_t>(k_blocks)), dim3(kThreads), lds, s, a, delta, pt, static_cast<int32_t>(p.k_tiles));
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;
    };
    int32_t st = FREE_OK;
    if constexpr (sizeof(T) == 2) st = p.kw == 2 ? launch(std::integral_constant<int, 2>{}) : launch(std::integral_constant<int, 4>{});
    else st = launch(std::integral_constant<int, 4>{});
    if (st != FREE_OK || p.k_parts == 1) return st;
    st = launch_sum<T>(pt.sum0, p.k_parts, a, a.Nk, 1, a.scale, a.dk, a.dk_stride, s);
    return st != FREE_OK ? st : launch_sum<T>(pt.sum1, p.k_parts, a, a.Nk, 1, 1.0f, a.dv, a.dv_stride, s);
}

template <typename T, bool kVec>
int32_t launch_width(const CrossArgs& a, const Plan& p, const Space& w, char* ws, hipStream_t s) {
    if (a.dh <= 32) return launch_shape<T, 32, kVec>(a, p, w, ws, s);
    if (a.dh <= 64) return launch_shape<T, 64, kVec>(a, p, w, ws, s);
    if (a.dh <= 80) return launch_shape<T, 80, kVec>(a, p, w, ws, s);
    if (a.dh <= 96) return launch_shape<T, 96, kVec>(a, p, w, ws, s);
    return launch_shape<T, 128, kVec>(a, p, w, ws, s);
}

template <typename T>
int32_t launch_type(const CrossArgs& a, void* ws, hipStream_t s) {
    const Plan p = plan_of(a.B, a.Nq, a.Nk, a.heads, a.kv_heads, sizeof(T) == 2 ? FREE_BF16 : FREE_FP32);
    const Space w(p, a.B, a.Nq, a.Nk, a.heads, a.kv_heads, a.dh);
    const auto al = [](const void* x, int64_t stride) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && stride % static_cast<int64_t>(16 / sizeof(T)) == 0; };
    const bool vec = a.dh % static_cast<int>(16 / sizeof(T)) == 0 && al(a.q, a.q_stride) && al(a.k, a.k_stride) && al(a.v, a.v_stride) && al(a.out, a.out_stride) &&
                     al(a.dout, a.dout_stride) && al(a.dq, a.dq_stride) && al(a.dk, a.dk_stride) && al(a.dv, a.dv_stride);
    char* const base = static_cast<char*>(ws);
    return vec ? launch_width<T, true>(a, p, w, base, s) : launch_width<T, false>(a, p, w, base, s);
}

}  // namespace

size_t cross_backward_bytes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype) {
    return Space(plan_of(B, Nq, Nk, heads, kv_heads, dtype), B, Nq, Nk, heads, kv_heads, dh).bytes;
}

int32_t launch_cross_backward(const CrossArgs& a, int32_t dtype, void* ws, hipStream_t s) {
    return dtype == FREE_BF16 ? launch_type<bf16_t>(a, ws, s) : launch_type<float>(a, ws, s);
}

}  // namespace freemi
