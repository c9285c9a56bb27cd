// The gradient of cross attention (cross_attn.hip), from its inputs, its result and lse:
//   P = exp(scale q k^T - lse) on the keys that count,  dP = dout v^T,  delta = sum P dP (= sum dout out),  dS = P (dP - delta)
//   dq = scale dS k,   dk = scale dS^T q,   dv = P^T dout      (dk, dv: summed over the queries of all heads that share them)
// Nothing of the size of the scores is kept between the passes: both kernels compute their tiles of scores again.
//  * dq: a wavefront has 32 rows (query and head of a group), and K and V stay in LDS or pass through it in tiles; it also leaves -lse / scale and
//    -delta of its rows for
//  * dk, dv: a wavefront has 32 keys, and tiles of q and dout pass through LDS, so that both sums stay in registers.
// The score tile's rows are the streamed tensor's rows and its columns the workgroup's own (cross_attn.h), in both.
// delta: out is rounded to its type, and dS is a difference that is small where few keys share the weight.  A sample of up to 256 keys (kTwiceKeys), and
// one whose keys stay in LDS, is passed over twice, first for sum P dP in fp32; of more keys delta is sum dout out, and the keys' gradient is given what
// the sum of a row's dS shows it to be off by (over all keys dS is zero; not where the keys are cut in parts).  In bf16, error of dq relative to that of a result computed in 64 bits and rounded: with
// delta from out 1.86 / 1.58 / 1.52 at 16 / 64 / 256 keys, so 1.42 / 1.43 / 1.44 (1.41 is dS's rounding and the result's); the second pass costs 32 -> 37 us
// at 8 x 1024 queries to 256 keys of 16 heads of 72.
// What bounds them: heads of 72, the latency of a block's chain (LDS, products, exponentials, products) with two wavefronts per SIMD, which wait 43 % of their
// time in dk and dv and 27 in dq, the matrix pipe busy 26 and 33 % (8 x 1024 queries to 256 keys of 16 heads: 35 and 37 us).  Heads of 128, one
// wavefront per SIMD whose vector and matrix instructions take turns, the pipe busy 35 and 28 % (32760 to 512: 367 us, 0.75 PFLOP/s, and 346, of which 170 are
// the rows' way to and from memory).  fp32 the matrix instructions, an eighth as fast (3 x 333 to 141 of 6 heads of 64: 25 and 15).
// Where a launch would have few workgroups the streamed axis is cut in parts, whose fp32 results a second launch adds in order: no
// atomics, equal inputs give equal bits.
#include <algorithm>
#include <cmath>

#include "cross_attn.h"

namespace freemi {

namespace {

constexpr int kThreads = kStreamThreads;
constexpr int kTwiceKeys = 256;                   // bf16: up to as many keys are passed over twice for delta

// parts of the streamed axis: tiles of each; fp32 results [part][pair][row][dh]
struct GradParts {
    int32_t parts, tiles;
    float *sum0, *sum1;
};

// what a row of queries is to the keys' gradient: -lse / scale and -delta, each [B, heads, Nq]
struct RowStats {
    float *lse, *delta;
};

// A block of 32 keys by a wavefront's rows: the scores in st, dout v^T on top of what is in dp.  Operands are read a group of chunks ahead of the
// products, through both tensors.
template <typename T, int DP>
__device__ __forceinline__ void score_products(const char* tile_k, const char* tile_v, int row0, int lane, const xu32x4_t (&qf)[HeadShape<T, DP>::KSTEPS],
                                               const xu32x4_t (&gf)[HeadShape<T, DP>::KSTEPS], xf32x16_t& st, xf32x16_t& dp) {
    constexpr int KSTEPS = HeadShape<T, DP>::KSTEPS, G = kRowGroup<T, DP>, kGroups = (KSTEPS + G - 1) / G;
    constexpr bool kOrder = DP <= 96;
    xu32x4_t f[2][G];
    clear_tile(st);
    read_rows<T, DP>(tile_k, row0, lane, 0, f[0]);
#pragma unroll
    for (int i = 0; i < 2 * kGroups; ++i) {
        const int first = i % kGroups * G;
        if (i + 1 < 2 * kGroups) read_rows<T, DP>(i + 1 < kGroups ? tile_k : tile_v, row0, lane, (i + 1) % kGroups * G, f[(i + 1) & 1]);
        if constexpr (kOrder) fence();
#pragma unroll
        for (int k = 0; k < G; ++k)
            if (first + k < KSTEPS) {
                if (i < kGroups) chunk_product<T>(f[i & 1][k], qf[first + k], st);
                else chunk_product<T>(f[i & 1][k], gf[first + k], dp);
            }
    }
}

// P times what stands in dp, for the keys that count
template <typename T>
__device__ __forceinline__ void weigh(xf32x16_t& st, const xf32x16_t& dp, uint32_t bits, float lse2, float scale_log2) {
#pragma unroll
    for (int e = 0; e < 16; ++e) st[e] = __builtin_amdgcn_exp2f(fmaf(st[e], scale_log2, -lse2)) * dp[e];
    if (__builtin_amdgcn_readfirstlane(bits) != ~0u) {
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e] = bits >> register_row<T>(e, 0) & 1 ? st[e] : 0.f;
    }
}

__device__ __forceinline__ float sum_of(const xf32x16_t& v) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) s += v[e];
    return s;
}

// delta += sum P dP over one 32-key block; bits: which of its keys count, from this half-wave's first on
template <typename T, int DP>
__device__ __forceinline__ void delta_block(const char* tile_k, const char* tile_v, int row0, int lane, uint32_t bits, const xu32x4_t (&qf)[HeadShape<T, DP>::KSTEPS],
                                            const xu32x4_t (&gf)[HeadShape<T, DP>::KSTEPS], float lse2, float scale_log2, float& delta) {
    xf32x16_t st, dp;
    clear_tile(dp);
    score_products<T, DP>(tile_k, tile_v, row0, lane, qf, gf, st, dp);
    weigh<T>(st, dp, bits, lse2, scale_log2);
    delta += sum_of(st);
}

// What is subtracted from a score or from dP is where the bf16 products' sums begin.  In fp32 each addition would be rounded at its size, lse / scale being
// some ten times a score (error of dk and dv of 3 x 333 queries to 141 keys against 64 bits 9.5e-7, without 4.8e-7): there it is added at the end.
template <typename T>
constexpr bool kLateStats = sizeof(T) == 4;

// dq += over one 32-key block; rest += the sum of its dS, which is zero over all keys but for what delta is off by
template <typename T, int DP, bool kRest>
__device__ __forceinline__ void dq_block(const char* tile_k, const char* tile_v, int row0, int lane, uint32_t bits, const xu32x4_t (&qf)[HeadShape<T, DP>::KSTEPS],
                                         const xu32x4_t (&gf)[HeadShape<T, DP>::KSTEPS], float dl, float lse2, float scale_log2, float& rest,
                                         xf32x16_t (&dq)[HeadShape<T, DP>::DT]) {
    Columns<T, DP> ck;
    xf32x16_t st, dp;
#pragma unroll
    for (int e = 0; e < 16; ++e) dp[e] = kLateStats<T> ? 0.f : -dl;
    score_products<T, DP>(tile_k, tile_v, row0, lane, qf, gf, st, dp);
    if constexpr (kLateStats<T>) {
#pragma unroll
        for (int e = 0; e < 16; ++e) dp[e] -= dl;
    }
    ck.read(tile_k, row0, lane, 0);
    weigh<T>(st, dp, bits, lse2, scale_log2);
    if constexpr (kRest) rest += sum_of(st);
    column_products<T, DP, (DP <= 96)>(tile_k, row0, lane, ck, st, dq);
}

// of the instructions since the last fence: N times a product, then `valu` and `trans` others
template <int N, int valu, int trans>
__device__ __forceinline__ void between_products() {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (valu > 0) __builtin_amdgcn_sched_group_barrier(0x002, valu, 0);
        if (trans > 0) __builtin_amdgcn_sched_group_barrier(0x400, trans, 0);
    }
}

// dk, dv += over one block of 32 rows, whose -lse / scale and -delta are at `lse` and `delta`: the sums of scores begin with them
template <typename T, int DP>
__device__ __forceinline__ void dkv_block(const char* tile_q, const char* tile_g, int row0, int lane, const float* lse, const float* delta,
                                          const xu32x4_t (&kf)[HeadShape<T, DP>::KSTEPS], const xu32x4_t (&vf)[HeadShape<T, DP>::KSTEPS], float scale_log2,
                                          xf32x16_t (&dk)[HeadShape<T, DP>::DT], xf32x16_t (&dv)[HeadShape<T, DP>::DT]) {
    xu32x4_t fq[kRowGroup<T, DP>], fg[kRowGroup<T, DP>];
    Columns<T, DP> cg, cq;
    xf32x16_t st, dp;
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
        const int at = row0 + register_row<T>(4 * e4, lane >> 5);
        const xf32x4_t l = *reinterpret_cast<const xf32x4_t*>(lse + at), d = *reinterpret_cast<const xf32x4_t*>(delta + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            st[4 * e4 + i] = kLateStats<T> ? 0.f : l[i];
            dp[4 * e4 + i] = kLateStats<T> ? 0.f : d[i];
        }
    }
    if constexpr (sizeof(T) == 2) {
        // A wavefront's matrix instructions run on while it issues others: the exponentials stand between the products of the second tensor, and what is
        // left of dS between those of dv.
        constexpr int KSTEPS = HeadShape<T, DP>::KSTEPS, G = kRowGroup<T, DP>, kGroups = (KSTEPS + G - 1) / G, DT = HeadShape<T, DP>::DT, kPer = 16 / kGroups;
        xu32x4_t f[2][G];
        read_rows<T, DP>(tile_q, row0, lane, 0, f[0]);
#pragma unroll
        for (int i = 0; i < 2 * kGroups; ++i) {
            const int first = i % kGroups * G;
            if (i + 1 < 2 * kGroups) read_rows<T, DP>(i + 1 < kGroups ? tile_q : tile_g, row0, lane, (i + 1) % kGroups * G, f[(i + 1) & 1]);
            else cg.read(tile_g, row0, lane, 0);
            fence();
#pragma unroll
            for (int k = 0; k < G; ++k)
                if (first + k < KSTEPS) {
                    if (i < kGroups) chunk_product<T>(f[i & 1][k], kf[first + k], st);
                    else chunk_product<T>(f[i & 1][k], vf[first + k], dp);
                }
            if (i >= kGroups) {
#pragma unroll
                for (int e = (i - kGroups) * kPer; e < (i - kGroups + 1) * kPer; ++e) st[e] = __builtin_amdgcn_exp2f(st[e] * scale_log2);
                between_products<G, (2 * kPer + G - 1) / G, (kPer + G - 1) / G>();
            }
        }
        cq.read(tile_g, row0, lane, 1);
        fence();
        cg.multiply(st, 0, dv);
#pragma unroll
        for (int e = 0; e < 8; ++e) dp[e] *= st[e];
        between_products<DT, (16 + DT - 1) / DT, 0>();
        cg.read(tile_q, row0, lane, 0);
        fence();
        cq.multiply(st, 1, dv);
#pragma unroll
        for (int e = 8; e < 16; ++e) dp[e] *= st[e];
        between_products<DT, (16 + DT - 1) / DT, 0>();
        cq.read(tile_q, row0, lane, 1);
        fence();
        cg.multiply(dp, 0, dk);
        cq.multiply(dp, 1, dk);
        return;
    }
    read_rows<T, DP>(tile_q, row0, lane, 0, fq);
    read_rows<T, DP>(tile_g, row0, lane, 0, fg);
    fence();
    row_products<T, DP>(tile_q, row0, lane, fq, kf, st);
    cg.read(tile_g, row0, lane, 0);
    fence();
    row_products<T, DP>(tile_g, row0, lane, fg, vf, dp);
    if constexpr (kLateStats<T>) {
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const int at = row0 + register_row<T>(4 * e4, lane >> 5);
            const xf32x4_t l = *reinterpret_cast<const xf32x4_t*>(lse + at), d = *reinterpret_cast<const xf32x4_t*>(delta + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                st[4 * e4 + i] += l[i];
                dp[4 * e4 + i] += d[i];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        st[e] = __builtin_amdgcn_exp2f(st[e] * scale_log2);
        dp[e] *= st[e];
    }
    cq.read(tile_q, row0, lane, 0);
    fence();
    column_products<T, DP>(tile_g, row0, lane, cg, st, dv);
    column_products<T, DP>(tile_q, row0, lane, cq, dp, dk);
}

// A row's chunks of q and dout; delta of its chunks of out, too
template <typename T, int DP, bool kVec>
struct RowOperands {
    static constexpr int KSTEPS = HeadShape<T, DP>::KSTEPS;
    xu32x4_t q[KSTEPS], g[KSTEPS];
    int64_t q_at, h_at, stat;        // its row, its head's first value in it, and its place among [B, heads, Nq]
    float lse;
    __device__ __forceinline__ void load(const CrossArgs& a, int b, int kvh, int row, int half) {
        const int group = a.heads / a.kv_heads, r = min(row, a.Nq * group - 1), token = over_group(r, group), head = kvh * group + r - token * group;
        q_at = static_cast<int64_t>(b) * a.Nq + token;
        h_at = static_cast<int64_t>(head) * a.dh;
        stat = (static_cast<int64_t>(b) * a.heads + head) * a.Nq + token;
        lse = a.lse[stat];
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
            g[ks] = row_chunk<T, kVec>(static_cast<const T*>(a.dout) + q_at * a.dout_stride + h_at, 2 * ks + half, a.dh);
            q[ks] = row_chunk<T, kVec>(static_cast<const T*>(a.q) + q_at * a.q_stride + h_at, 2 * ks + half, a.dh);
        }
    }
    __device__ __forceinline__ float delta(const CrossArgs& a, int half) const {
        xu32x4_t o[KSTEPS];
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) o[ks] = row_chunk<T, kVec>(static_cast<const T*>(a.out) + q_at * a.out_stride + h_at, 2 * ks + half, a.dh);
        float dl = 0.f;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (sizeof(T) == 2) {
                    dl = fmaf(__uint_as_float(g[ks][e] << 16), __uint_as_float(o[ks][e] << 16), dl);
                    dl = fmaf(__uint_as_float(g[ks][e] & 0xffff0000u), __uint_as_float(o[ks][e] & 0xffff0000u), dl);
                } else {
                    dl = fmaf(__uint_as_float(g[ks][e]), __uint_as_float(o[ks][e]), dl);
                }
            }
        return add_lane_xor<32>(dl);
    }
    __device__ __forceinline__ void leave(const RowStats& stats, float dl, float scale) const {
        stats.lse[stat] = -lse / scale;
        stats.delta[stat] = -dl;
    }
};

// ---- dq and delta
template <typename T, int DP, bool kVec>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 && kVec) || DP <= 64 ? 2 : 1) void cross_dq_kernel(CrossArgs a, RowStats stats, GradParts pt, int32_t q_tiles) {
    using H = HeadShape<T, DP>;
    using TL = Tile<T, DP>;
    constexpr int KSTEPS = H::KSTEPS, DT = H::DT, BKV = TL::kRows;
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
    const int rows = a.Nq * group, row = q_tile * 128 + wave * 32 + l32;
    KeyStream<T, DP, kVec> keys(a, b, kvh);
    const int t0 = part * pt.tiles, t1 = min(t0 + pt.tiles, keys.tiles());
    const uint32_t lds_base = lds_address(lds);
    const bool twice = sizeof(T) == 2 && keys.len <= kTwiceKeys;         // (which are all in the first part then)
    uint64_t valid;
    const auto begin_tiles = [&] {
        keys.request_mask(t0, lane);
        valid = keys.valid_of(t0);
        if (t0 < t1) keys.request(t0, lds_base, lds_base + TL::kBytes, wave, lane, valid);
        keys.request_mask(t0 + 1, lane);
    };
    const auto each_block = [&](auto&& use) {
        if (t0 < t1) keys.deliver(lds, lds + TL::kBytes, tid, valid);
        keys.k.settle();
        for (int t = t0; t < t1; ++t) {
            const int stage = (t - t0) & 1, other = (stage ^ 1) * 2 * TL::kBytes;
            const char* const sK = lds + stage * 2 * TL::kBytes;
            const uint64_t valid_next = keys.valid_of(t + 1);
            if (t + 1 < t1) {
                keys.request(t + 1, lds_base + other, lds_base + other + TL::kBytes, wave, lane, valid_next);
                keys.request_mask(t + 2, lane);
            }
#pragma unroll
            for (int kb = 0; kb < BKV / 32; ++kb) {
                // (fp32 has 32 keys to a tile, and a full mask of them)
                const uint32_t bits = static_cast<uint32_t>(valid >> (32 * kb));
                use(sK, kb * 32, bits == ~0u ? bits : bits >> (sizeof(T) == 2 ? 8 * g : 4 * g));
            }
            if (t + 1 < t1) keys.deliver(lds + other, lds + other + TL::kBytes, tid, valid_next);
            valid = valid_next;
            keys.k.settle();
        }
    };
    begin_tiles();
    RowOperands<T, DP, kVec> own;
    own.load(a, b, kvh, row, g);
    const float lse2 = own.lse * kLog2e, scale_log2 = a.scale * kLog2e;
    float dl = 0.f, rest = 0.f;
    if (!twice) dl = own.delta(a, g);

    xf32x16_t dq[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) clear_tile(dq[dt]);
    arrived(own.q);
    arrived(own.g);
    if constexpr (sizeof(T) == 2) {
        if (twice) {
            each_block([&](const char* tile, int row0, uint32_t bits) {
                delta_block<T, DP>(tile, tile + TL::kBytes, row0, lane, bits, own.q, own.g, lse2, scale_log2, dl);
            });
            dl = add_lane_xor<32>(dl);
            begin_tiles();
        }
    }
    each_block([&](const char* tile, int row0, uint32_t bits) {
        dq_block<T, DP, true>(tile, tile + TL::kBytes, row0, lane, bits, own.q, own.g, dl, lse2, scale_log2, rest, dq);
    });
    // (a part has not all keys; with both passes the rest is what rounding leaves)
    rest = pt.parts > 1 ? 0.f : add_lane_xor<32>(rest);
    if (part == 0 && g == 0 && row < rows) own.leave(stats, dl + rest, a.scale);
    if (pt.parts > 1) store_column<float, kVec, DT>(pt.sum0 + ((part * static_cast<int64_t>(pairs) + pair) * rows + row) * a.dh, a.dh, g, dq, 1.0f, row < rows);
    else store_column<T, kVec, DT>(static_cast<T*>(a.dq) + own.q_at * a.dq_stride + own.h_at, a.dh, g, dq, a.scale, row < rows);
}

// ---- dk and dv.  KW wavefronts have 32 keys each; where the keys leave some without, the rows of a step are shared out among QW, whose sums are
// parts of their own: the two halves of a tile (bf16), or a tile for each (fp32, whose products take eight times as long; 7 x 5303 queries to one key, 16
// heads of 64: 452 -> 165 us).  With four tiles to a step there is one stage.
template <typename T, int KW>
constexpr int kStepTiles = sizeof(T) == 4 ? 4 / KW : 1;

template <typename T, int DP, int KW, bool kVec>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 && DP <= 80) || DP <= 32 ? 2 : 1) void cross_dkv_kernel(CrossArgs a, RowStats row_stats, GradParts pt, int32_t k_tiles) {
    using H = HeadShape<T, DP>;
    using TL = Tile<T, DP>;
    constexpr int KSTEPS = H::KSTEPS, DT = H::DT, BR = TL::kRows, QW = 4 / KW;
    constexpr int SUB = kStepTiles<T, KW>, STAGES = SUB == 4 ? 1 : 2, MR = BR * SUB, RB = SUB > 1 ? 1 : BR / 32 / QW;
    static_assert(RB >= 1, "a block of rows for each wavefront");
    extern __shared__ __attribute__((aligned(16))) char lds[];          // [stage][tile][q, dout], then [stage][lse, delta][MR]
    float* const stats = reinterpret_cast<float*>(lds + STAGES * SUB * 2 * TL::kBytes);
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
    const int rows = a.Nq * group, key = k_tile * 32 * KW + kw * 32 + l32;
    const int len = attended(a, b);
    const int steps = (rows + MR - 1) / MR, t0 = part * pt.tiles;
    // keys that do not count have no gradient: a workgroup without others has nothing to sum
    const int t1 = k_tile * 32 * KW < len ? min(t0 + pt.tiles, steps) : t0;
    const bool there = key < len && (!a.key_mask || a.key_mask[static_cast<int64_t>(b) * a.Nk + key] != 0);

    const int q_row = static_cast<int>(a.q_stride) * static_cast<int>(sizeof(T)), g_row = static_cast<int>(a.dout_stride) * static_cast<int>(sizeof(T));
    const int head_bytes = a.dh * static_cast<int>(sizeof(T));
    const int64_t first_row = static_cast<int64_t>(b) * a.Nq, h0 = static_cast<int64_t>(kvh) * group * a.dh;
    TileStream<T, DP, kVec> queries[SUB], grads[SUB];
    float lse_next = 0.f, delta_next = 0.f;
    const uint32_t lds_base = lds_address(lds);
    const auto request = [&](int t, int stage) {
#pragma unroll
        for (int j = 0; j < SUB; ++j) {
            const int r0 = t * MR + j * BR, token0 = over_group(r0, group), rest = r0 - token0 * group;      // of the group's heads: row r0 + r is token0 + (rest + r) / group
            const int64_t left = a.Nq - token0;
            const auto place = [&](int stride) {
                return [=](int r) {
                    const int token = over_group(rest + r, group);
                    return token * stride + (rest + r - token * group) * head_bytes;
                };
            };
            const uint32_t to = lds_base + (stage * SUB + j) * 2 * TL::kBytes;
            queries[j].request(static_cast<const T*>(a.q) + (first_row + token0) * a.q_stride + h0, (left - 1) * q_row + group * head_bytes, to, wave, lane, a.dh, false, 0,
                               place(q_row));
            grads[j].request(static_cast<const T*>(a.dout) + (first_row + token0) * a.dout_stride + h0, (left - 1) * g_row + group * head_bytes, to + TL::kBytes, wave,
                             lane, a.dh, false, 0, place(g_row));
        }
        const int r0 = t * MR, token0 = over_group(r0, group), rest = r0 - token0 * group;
        if (tid < MR) {
            const int token = over_group(rest + tid, group), h = rest + tid - token * group;
            const int64_t at = (static_cast<int64_t>(b) * a.heads + kvh * group + h) * a.Nq + token0 + token;
            const bool on = r0 + tid < rows;
            lse_next = on ? row_stats.lse[at] : 0.f;                    // (rows past the end are zero, and add nothing)
            delta_next = on ? row_stats.delta[at] : 0.f;
        }
    };
    const auto deliver = [&](int stage) {
#pragma unroll
        for (int j = 0; j < SUB; ++j) {
            char* const sQ = lds + (stage * SUB + j) * 2 * TL::kBytes;
            queries[j].deliver(sQ, tid, false, 0);
            grads[j].deliver(sQ + TL::kBytes, tid, false, 0);
        }
        if (tid < MR) {
            stats[stage * 2 * MR + tid] = lse_next;
            stats[stage * 2 * MR + MR + tid] = delta_next;
        }
    };
    if (t0 < t1) request(t0, 0);

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
    if (t0 < t1) deliver(0);
    arrived(kf);
    arrived(vf);
    TileStream<T, DP, kVec>::settle();
    for (int t = t0; t < t1; ++t) {
        const int stage = STAGES == 2 ? (t - t0) & 1 : 0, other = STAGES == 2 ? stage ^ 1 : 0, sub = SUB > 1 ? qw : 0;
        const char* const sQ = lds + (stage * SUB + sub) * 2 * TL::kBytes;
        if (t + 1 < t1) request(t + 1, other);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row0 = SUB > 1 ? 0 : (qw * RB + rb) * 32;
            const float* const at = stats + stage * 2 * MR + sub * BR;
            dkv_block<T, DP>(sQ, sQ + TL::kBytes, row0, lane, at, at + MR, kf, vf, scale_log2, dk, dv);
        }
        if (STAGES == 1) __syncthreads();
        if (t + 1 < t1) deliver(other);
        TileStream<T, DP, kVec>::settle();
    }
    const bool on = key < a.Nk;
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
        store_column<float, kVec, DT>(pt.sum0 + at, a.dh, g, dk, 1.0f, on);
        store_column<float, kVec, DT>(pt.sum1 + at, a.dh, g, dv, 1.0f, on);
    } else {
        store_column<T, kVec, DT>(static_cast<T*>(a.dk) + kv_at * a.dk_stride + h_at, a.dh, g, dk, a.scale, on);
        store_column<T, kVec, DT>(static_cast<T*>(a.dv) + kv_at * a.dv_stride + h_at, a.dh, g, dv, 1.0f, on);
    }
}

// ---- the same for bf16 of whole chunks and many rows (cross_ring_kernel of cross_attn.hip)
template <int DP, bool kResident>
__global__ __launch_bounds__((kResident ? kRingWaves : kPassWaves) * 64, 2) void cross_dq_ring_kernel(CrossArgs a, RowStats stats, int32_t chunks, int32_t blocks_per_chunk) {
    using T = bf16_t;
    using H = HeadShape<T, DP>;
    constexpr int KSTEPS = H::KSTEPS, DT = H::DT, NW = kResident ? kRingWaves : kPassWaves, kSlots = kPassTiles<DP>;
    using Ring = PairRing<DP, NW>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ uint64_t masks[kMaxTiles];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, g = lane >> 5;
    const int pairs = a.B * a.kv_heads, group = a.heads / a.kv_heads;
    const WorkPlace at(blockIdx.x, pairs);
    const int pair = at.pair, chunk = at.place, kvh = pair % a.kv_heads, b = pair / a.kv_heads;
    const int rows = a.Nq * group, blocks = (rows + 31) / 32;
    RingKeys<DP, NW> keys(a, b, kvh, wave, lane);
    const int tiles = keys.tiles();
    const uint32_t lds_base = lds_address(lds);
    const auto request = [&](int t, int slot) { keys.request(t, lds_base + slot * Ring::kTileBytes, wave); };
    const float scale_log2 = a.scale * kLog2e;
    RowOperands<T, DP, true> own;
    xf32x16_t dq[DT];
    float dl = 0.f, rest = 0.f;
    const auto begin = [&] {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) clear_tile(dq[dt]);
        arrived(own.q);
        arrived(own.g);
    };
    const auto multiply = [&](const char* tile, uint64_t valid) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const uint32_t bits = static_cast<uint32_t>(valid >> (32 * kb));
            dq_block<T, DP, !kResident>(tile, tile + Ring::kSecond, kb * 32, lane, bits == ~0u ? bits : bits >> (8 * g), own.q, own.g, dl, own.lse * kLog2e, scale_log2, rest, dq);
        }
    };
    const auto measure = [&](const char* tile, uint64_t valid) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const uint32_t bits = static_cast<uint32_t>(valid >> (32 * kb));
            delta_block<T, DP>(tile, tile + Ring::kSecond, kb * 32, lane, bits == ~0u ? bits : bits >> (8 * g), own.q, own.g, own.lse * kLog2e, scale_log2, dl);
        }
    };
    const auto finish = [&](int block) {
        if (!kResident) dl += add_lane_xor<32>(rest);
        if (g == 0 && block * 32 + l32 < rows) own.leave(stats, dl, a.scale);
        store_column<T, true, DT>(static_cast<T*>(a.dq) + own.q_at * a.dq_stride + own.h_at, a.dh, g, dq, a.scale, block * 32 + l32 < rows);
    };
    if constexpr (kResident) {
        // the next block's rows are requested ahead of this one's products where there are registers for them
        constexpr bool kNext = DP <= 80;
        for (int t = 0; t < tiles; ++t) request(t, t);
        const int first = chunk * blocks_per_chunk, last = min(first + blocks_per_chunk, blocks);
        if (first + wave < last) own.load(a, b, kvh, (first + wave) * 32 + l32, g);
        bring_keys(keys, lds, masks, 0, wave, lane);
        for (int block = first + wave; block < last; block += NW) {
            begin();
            RowOperands<T, DP, true> next = own;
            const bool more = block + NW < last;
            if (kNext && more) next.load(a, b, kvh, (block + NW) * 32 + l32, g);
            const auto bits_of = [&](int t) { return keys.mask ? masks[t] : keys_below(keys.len - t * Tile<T, DP>::kRows); };
            dl = 0.f;
            for (int t = 0; t < tiles; ++t) measure(lds + t * Ring::kTileBytes, bits_of(t));
            dl = add_lane_xor<32>(dl);
            for (int t = 0; t < tiles; ++t) multiply(lds + t * Ring::kTileBytes, bits_of(t));
            finish(block);
            own = next;
            if (!kNext && more) own.load(a, b, kvh, (block + NW) * 32 + l32, g);
        }
    } else {
        const int block = chunk * NW + wave;
        const auto begin_tiles = [&] {
#pragma unroll
            for (int s = 0; s < kSlots - 1; ++s)
                if (s < tiles) request(s, s);
        };
        const auto each_tile = [&](auto&& use) {
            int slot = 0, free_slot = kSlots - 1;
            for (int t = 0; t < tiles; ++t) {
                const uint64_t valid = keys.valid(t, lane);
                if (t + kSlots - 1 <= tiles) wait_vm_barrier<(kSlots - 2) * Ring::N>();
                else wait_vm_barrier<0>();
                char* const tile = lds + slot * Ring::kTileBytes;
                if (keys.mask && valid != ~0ull) {
                    keys.drop(tile, 0, valid, wave, lane);
                    __syncthreads();
                }
                if (t + kSlots - 1 < tiles) request(t + kSlots - 1, free_slot);
                use(tile, valid);
                free_slot = slot;
                slot = slot + 1 == kSlots ? 0 : slot + 1;
            }
        };
        begin_tiles();
        own.load(a, b, kvh, block * 32 + l32, g);
        if (keys.len <= kTwiceKeys) {
            begin();
            each_tile(measure);
            dl = add_lane_xor<32>(dl);
            __syncthreads();
            begin_tiles();
        } else {
            dl = own.delta(a, g);
            begin();
        }
        each_tile(multiply);
        finish(block);
    }
}

// Head dimensions over 96: a wavefront has two blocks of 32 rows and the registers of two wavefronts, so that what it reads from LDS is multiplied twice.
// delta += sum P dP over one 32-key block, or dq += of it
template <int DP, bool kDelta>
__device__ __forceinline__ void dq_wide_block(const char* tile_k, const char* tile_v, int row0, int lane, uint32_t bits, const RowOperands<bf16_t, DP, true> (&own)[2],
                                              float scale_log2, float (&dl)[2], float (&rest)[2], xf32x16_t (&dq)[2][HeadShape<bf16_t, DP>::DT]) {
    using T = bf16_t;
    constexpr int KSTEPS = HeadShape<T, DP>::KSTEPS, G = 2, kGroups = KSTEPS / G, DT = HeadShape<T, DP>::DT;
    static_assert(KSTEPS % G == 0, "whole groups");
    xu32x4_t f[2][G];                // the operands multiplied and those read ahead
    xf32x16_t st[2], dp[2];
    const auto read = [&](int i) {
        const int row = block_row<T>(lane & 31), g = lane >> 5;
        const char* const base = (i < kGroups ? tile_k : tile_v) + row0 * Tile<T, DP>::kPitch;
#pragma unroll
        for (int k = 0; k < G; ++k) f[i & 1][k] = *reinterpret_cast<const xu32x4_t*>(base + Tile<T, DP>::at(row, 2 * (i % kGroups * G + k) + g));
    };
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        clear_tile(st[r]);
        clear_tile(dp[r]);
    }
    const float nlse[2] = {-own[0].lse * kLog2e, -own[1].lse * kLog2e};
    Columns<T, DP> c;
    read(0);
#pragma unroll
    for (int i = 0; i < 2 * kGroups; ++i) {
        if (i + 1 < 2 * kGroups) read(i + 1);
        else if (!kDelta) c.read(tile_k, row0, lane, 0);
        fence();
#pragma unroll
        for (int k = 0; k < G; ++k)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (i < kGroups) chunk_product<T>(f[i & 1][k], own[r].q[i * G + k], st[r]);
                else chunk_product<T>(f[i & 1][k], own[r].g[(i - kGroups) * G + k], dp[r]);
            }
        if (i >= kGroups) {                              // (exponentials between the products of the second tensor)
            const int r = (i - kGroups) / (kGroups / 2), e0 = (i - kGroups) % (kGroups / 2) * (32 / kGroups);
#pragma unroll
            for (int e = e0; e < e0 + 32 / kGroups; ++e) st[r][e] = __builtin_amdgcn_exp2f(fmaf(st[r][e], scale_log2, nlse[r]));
#pragma unroll
            for (int k = 0; k < 2 * G; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
            }
        }
    }
    const auto weigh_row = [&](int r) {
#pragma unroll
        for (int e = 0; e < 16; ++e) st[r][e] *= kDelta ? dp[r][e] : dp[r][e] - dl[r];
        if (__builtin_amdgcn_readfirstlane(bits) != ~0u) {
#pragma unroll
            for (int e = 0; e < 16; ++e) st[r][e] = bits >> register_row<T>(e, 0) & 1 ? st[r][e] : 0.f;
        }
        if (kDelta) dl[r] += sum_of(st[r]);
        else rest[r] += sum_of(st[r]);
    };
    weigh_row(0);
    if constexpr (kDelta) {
        weigh_row(1);
    } else {
        Columns<T, DP> next;
        next.read(tile_k, row0, lane, 1);
        fence();
        c.multiply(st[0], 0, dq[0]);
        next.multiply(st[0], 1, dq[0]);
        weigh_row(1);
#pragma unroll
        for (int k = 0; k < 2 * DT; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);
        }
        c.multiply(st[1], 0, dq[1]);
        next.multiply(st[1], 1, dq[1]);
    }
}

constexpr int kWideWaves = 4;

template <int DP>
__global__ __launch_bounds__(kWideWaves * 64, 1) void cross_dq_wide_kernel(CrossArgs a, RowStats stats) {
    using T = bf16_t;
    using H = HeadShape<T, DP>;
    using Ring = PairRing<DP, kWideWaves>;
    constexpr int DT = H::DT;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, g = lane >> 5;
    const int pairs = a.B * a.kv_heads, group = a.heads / a.kv_heads;
    const WorkPlace at(blockIdx.x, pairs);
    const int pair = at.pair, kvh = pair % a.kv_heads, b = pair / a.kv_heads;
    const int rows = a.Nq * group, row0 = (at.place * kWideWaves + wave) * 64 + l32;
    RingKeys<DP, kWideWaves> keys(a, b, kvh, wave, lane);
    const int tiles = keys.tiles();
    const uint32_t lds_base = lds_address(lds);
    const auto request = [&](int t, int slot) { keys.request(t, lds_base + slot * Ring::kTileBytes, wave); };
    const auto begin_tiles = [&] {
#pragma unroll
        for (int s = 0; s < kRing - 1; ++s)
            if (s < tiles) request(s, s);
    };
    begin_tiles();
    const float scale_log2 = a.scale * kLog2e;
    RowOperands<T, DP, true> own[2];
    xf32x16_t dq[2][DT];
    float dl[2] = {0.f, 0.f}, rest[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 2; ++r) own[r].load(a, b, kvh, row0 + 32 * r, g);
    const auto each_tile = [&](auto delta) {
        int slot = 0, free_slot = kRing - 1;
        for (int t = 0; t < tiles; ++t) {
            const uint64_t valid = keys.valid(t, lane);
            if (t + kRing - 1 <= tiles) wait_vm_barrier<(kRing - 2) * Ring::N>();
            else wait_vm_barrier<0>();
            char* const tile = lds + slot * Ring::kTileBytes;
            if (keys.mask && valid != ~0ull) {
                keys.drop(tile, 0, valid, wave, lane);
                __syncthreads();
            }
            if (t + kRing - 1 < tiles) request(t + kRing - 1, free_slot);
#pragma unroll 1
            for (int kb = 0; kb < 2; ++kb) {
                const uint32_t bits = static_cast<uint32_t>(valid >> (32 * kb));
                dq_wide_block<DP, decltype(delta)::value>(tile, tile + Ring::kSecond, kb * 32, lane, bits == ~0u ? bits : bits >> (8 * g), own, scale_log2, dl, rest, dq);
            }
            free_slot = slot;
            slot = slot + 1 == kRing ? 0 : slot + 1;
        }
    };
    if (keys.len > kTwiceKeys) {
#pragma unroll
        for (int r = 0; r < 2; ++r) dl[r] = own[r].delta(a, g);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        arrived(own[r].q);
        arrived(own[r].g);
    }
    if (keys.len <= kTwiceKeys) {
        each_tile(std::true_type{});
#pragma unroll
        for (int r = 0; r < 2; ++r) dl[r] = add_lane_xor<32>(dl[r]);
        __syncthreads();
        begin_tiles();
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) clear_tile(dq[r][dt]);
    each_tile(std::false_type{});
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const bool on = row0 + 32 * r < rows;
        const float sum = add_lane_xor<32>(rest[r]);
        if (g == 0 && on) own[r].leave(stats, dl[r] + sum, a.scale);
        store_column<T, true, DT>(static_cast<T*>(a.dq) + own[r].q_at * a.dq_stride + own[r].h_at, a.dh, g, dq[r], a.scale, on);
    }
}

// NW wavefronts: KW of them have 32 keys each, and with KW < NW the blocks of a tile's rows go to two, whose sums are added at the end
template <int DP, int NW, int KW>
__global__ __launch_bounds__(NW * 64, NW / 4) void cross_dkv_ring_kernel(CrossArgs a, RowStats row_stats, GradParts pt, int32_t k_tiles) {
    using T = bf16_t;
    using H = HeadShape<T, DP>;
    using TL = Tile<T, DP>;
    using Ring = PairRing<DP, NW>;
    constexpr int KSTEPS = H::KSTEPS, DT = H::DT, BR = TL::kRows, QW = NW / KW, RB = 2 / QW;
    constexpr int kSlot = Ring::kTileBytes + NW * 256;                   // a tile, then -lse / scale and -delta of its rows (and room for the other wavefronts' loads)
    static_assert(QW == 1 || QW == 2, "blocks of a tile");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, g = lane >> 5;
    const int kw = wave % KW, qw = wave / KW;
    const int pairs = a.B * a.kv_heads, group = a.heads / a.kv_heads;
    const WorkPlace at(blockIdx.x, pairs);
    const int pair = at.pair, k_tile = at.place % k_tiles, part = at.place / k_tiles;
    const int kvh = pair % a.kv_heads, b = pair / a.kv_heads;
    const int rows = a.Nq * group, first_key = (k_tile * KW + kw) * 32, key = first_key + l32;
    const int len = attended(a, b);
    const int t0 = part * pt.tiles, t1 = k_tile * 32 * KW < len ? min(t0 + pt.tiles, (rows + BR - 1) / BR) : t0;
    const bool there = key < len && (!a.key_mask || a.key_mask[static_cast<int64_t>(b) * a.Nk + key] != 0);
    const bool busy = first_key < len;                                   // (a wavefront without keys takes part in the loads alone)

    const int64_t first_row = static_cast<int64_t>(b) * a.Nq, h0 = static_cast<int64_t>(kvh) * group * a.dh;
    const bf16_t* const qp = static_cast<const T*>(a.q) + first_row * a.q_stride + h0;
    const bf16_t* const gp = static_cast<const T*>(a.dout) + first_row * a.dout_stride + h0;
    const int64_t stat0 = (static_cast<int64_t>(b) * a.heads + kvh * group) * a.Nq;
    const uint32_t lds_base = lds_address(lds);
    Ring ring;
    const auto aim = [&](int rest) {                                     // row r of a tile is token (rest + r) / group of it
        ring.aim(wave, lane, a.dh, [&](int second, int r) {
            const int token = over_group(rest + r, group);
            return (token * static_cast<int>(second ? a.dout_stride : a.q_stride) + (rest + r - token * group) * a.dh) * 2;
        });
    };
    aim(0);
    const bool turn = BR % group != 0;                                   // tiles begin at other heads of the group
    const auto request = [&](int t, int slot) {
        const int r0 = t * BR, token0 = over_group(r0, group), rest = r0 - token0 * group;
        if (turn) aim(rest);
        const uint32_t to = lds_base + slot * kSlot;
        ring.request(rows_rsrc(qp, token0, a.Nq - token0, a.q_stride, group * a.dh), rows_rsrc(gp, token0, a.Nq - token0, a.dout_stride, group * a.dh), to, wave);
        const int token = over_group(rest + lane, group), head = rest + lane - token * group;
        const int off = wave < 2 && r0 + lane < rows ? (head * a.Nq + token) * 4 : kNowhere;         // (rows past the end are zero, and add nothing)
        const float* const from = (wave == 0 ? row_stats.lse : row_stats.delta) + stat0 + token0;
        dma_floats(to + Ring::kTileBytes + wave * 256, off, make_rsrc(from, (static_cast<int64_t>(rows) - token0) * 4));
    };
#pragma unroll
    for (int s = 0; s < kRing - 1; ++s)
        if (t0 + s < t1) request(t0 + s, s);

    const int64_t kv_at = static_cast<int64_t>(b) * a.Nk + (key < a.Nk ? key : 0), h_at = static_cast<int64_t>(kvh) * a.dh;
    xu32x4_t kf[KSTEPS], vf[KSTEPS];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
        kf[ks] = vf[ks] = xu32x4_t{0, 0, 0, 0};
        if (there) {
            kf[ks] = row_chunk<T, true>(static_cast<const T*>(a.k) + kv_at * a.k_stride + h_at, 2 * ks + g, a.dh);
            vf[ks] = row_chunk<T, true>(static_cast<const T*>(a.v) + kv_at * a.v_stride + h_at, 2 * ks + g, a.dh);
        }
    }
    const float scale_log2 = a.scale * kLog2e;
    xf32x16_t dk[DT], dv[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        clear_tile(dk[dt]);
        clear_tile(dv[dt]);
    }
    arrived(kf);
    arrived(vf);
    int slot = 0, free_slot = kRing - 1;
    for (int t = t0; t < t1; ++t) {
        if (t + kRing - 1 <= t1) wait_vm_barrier<(kRing - 2) * (Ring::N + 1)>();
        else wait_vm_barrier<0>();
        if (t + kRing - 1 < t1) request(t + kRing - 1, free_slot);
        const char* const tile = lds + slot * kSlot;
        const float* const lse = reinterpret_cast<const float*>(tile + Ring::kTileBytes);
        if (busy) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) dkv_block<T, DP>(tile, tile + Ring::kSecond, (qw * RB + rb) * 32, lane, lse, lse + 64, kf, vf, scale_log2, dk, dv);
        }
        free_slot = slot;
        slot = slot + 1 == kRing ? 0 : slot + 1;
    }
    if constexpr (QW == 2) {
        // the second blocks' sums to the first's wavefronts, dk and dv in turn
        static_assert(KW * DT * 4096 <= kRing * kSlot, "the sums of half the wavefronts fit in the ring");
        char* const to = lds + kw * DT * 4096 + lane * 16;
        const auto add = [&](xf32x16_t (&v)[DT]) {
            __syncthreads();
            if (qw > 0) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4)
                        *reinterpret_cast<xf32x4_t*>(to + (dt * 4 + e4) * 1024) = xf32x4_t{v[dt][4 * e4], v[dt][4 * e4 + 1], v[dt][4 * e4 + 2], v[dt][4 * e4 + 3]};
            }
            __syncthreads();
            if (qw == 0) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4) {
                        const xf32x4_t o = *reinterpret_cast<const xf32x4_t*>(to + (dt * 4 + e4) * 1024);
#pragma unroll
                        for (int c = 0; c < 4; ++c) v[dt][4 * e4 + c] += o[c];
                    }
            }
        };
        add(dk);
        add(dv);
        if (qw > 0) return;
    }
    const bool on = key < a.Nk;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            dk[dt][e] = there ? dk[dt][e] : 0.f;
            dv[dt][e] = there ? dv[dt][e] : 0.f;
        }
    if (pt.parts > 1) {
        const int64_t to = ((part * static_cast<int64_t>(pairs) + pair) * a.Nk + key) * a.dh;
        store_column<float, true, DT>(pt.sum0 + to, a.dh, g, dk, 1.0f, on);
        store_column<float, true, DT>(pt.sum1 + to, a.dh, g, dv, 1.0f, on);
    } else {
        store_column<T, true, DT>(static_cast<T*>(a.dk) + kv_at * a.dk_stride + h_at, a.dh, g, dk, a.scale, on);
        store_column<T, true, DT>(static_cast<T*>(a.dv) + kv_at * a.dv_stride + h_at, a.dh, g, dv, 1.0f, on);
    }
}

// The parts of a sum [part][pair][row][dh], added in order, times `factor`: a thread per V values.  Row r of a pair is token r / group, head r % group
// of the pair's.  blockIdx.y: which of two sums of one shape.
struct SumJob {
    const float* parts;
    void* out;
    int64_t stride;
    float factor;
};
struct SumJobs {
    SumJob job[2];
    int32_t n, kv_heads, tokens, group, dh;
    int64_t pairs;
};

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void cross_sum_kernel(SumJobs a) {
    const SumJob& j = blockIdx.y ? a.job[1] : a.job[0];
    const uint32_t rows = static_cast<uint32_t>(a.tokens) * a.group, per_row = a.dh / V;
    const int64_t all = a.pairs * rows * per_row;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * kThreads) {
        float s[V];
        __builtin_memcpy(s, j.parts + i * V, sizeof(s));
#pragma unroll 8
        for (int p = 1; p < a.n; ++p) {
            float v[V];
            __builtin_memcpy(v, j.parts + (p * all + i) * V, sizeof(v));
#pragma unroll
            for (int e = 0; e < V; ++e) s[e] += v[e];
        }
        const int64_t at = i / per_row, pair = at / rows;
        const int r = static_cast<int>(at - pair * rows), token = over_group(r, a.group), head = static_cast<int>(pair % a.kv_heads) * a.group + r - token * a.group;
        T* const out = static_cast<T*>(j.out) + (pair / a.kv_heads * a.tokens + token) * j.stride + static_cast<int64_t>(head) * a.dh + (i - at * per_row) * V;
        if constexpr (V == 4) store4<T, true>(out, 0, 4, s[0] * j.factor, s[1] * j.factor, s[2] * j.factor, s[3] * j.factor);
        else store_f(out, s[0] * j.factor);
    }
}

template <typename T, bool kVec>
int32_t launch_sum(const SumJobs& a, int jobs, hipStream_t s) {
    constexpr int V = kVec ? 4 : 1;
    const int64_t all = a.pairs * a.tokens * a.group * (a.dh / V);
    const int64_t blocks = std::min<int64_t>((all + kThreads - 1) / kThreads, 1 << 20);
    hipLaunchKernelGGL((cross_sum_kernel<T, V>), dim3(static_cast<uint32_t>(blocks), jobs), dim3(kThreads), 0, s, a);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

// How the two launches are cut; by the sizes and by whether rows are whole aligned chunks
struct Plan {
    bool q_ring, resident;
    int32_t q_parts, q_part_tiles, q_blocks;      // q_blocks: resident, 32-row blocks of a workgroup
    int64_t q_tiles;                              // workgroups of a (sample, key head) and part
    bool k_ring;
    int kw;                                       // wavefronts with keys of their own
    int32_t k_parts, k_part_tiles;                // (parts: where two wavefronts have the same keys and keep their sums, those counted)
    int64_t k_tiles, k_units;                     // workgroups of a (sample, key head) and part; parts that a workgroup has
};
constexpr int kUnits = 256;

// wavefronts of cross_dkv_ring_kernel: head dimensions over 80 need the registers of two
template <int DP>
constexpr int kKeyWaves = DP <= 80 ? 8 : 4;

Plan plan_of(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype, bool whole_chunks) {
    const int64_t pairs = static_cast<int64_t>(B) * kv_heads, rows = static_cast<int64_t>(Nq) * (heads / kv_heads), units = std::max<int64_t>(pairs, 1);
    const int tile = dtype == FREE_BF16 ? 64 : 32;
    const auto cut = [](int64_t work, int64_t want, int64_t tiles, int64_t least, int64_t* parts, int64_t* per) {
        *parts = std::min<int64_t>(std::max<int64_t>(1, std::min(want / std::max<int64_t>(work, 1), tiles / least)), 64);
        *per = (tiles + *parts - 1) / *parts;
        *parts = (tiles + *per - 1) / *per;
    };
    const bool ring = dtype == FREE_BF16 && whole_chunks && rows < 1 << 29;       // (32-bit offsets of a row's floats)
    const int64_t key_tiles = std::max<int64_t>(1, (static_cast<int64_t>(Nk) + tile - 1) / tile), row_tiles = std::max<int64_t>(1, (rows + tile - 1) / tile);
    Plan p{};
    int64_t parts, per;
    // Tiles of a part: fewer cost more in sums than they spare, bf16 (2 x 300 queries to 400 keys of 8 heads of 64, dq and dk, dv 25 us with 4 and 28 with 2);
    // an fp32 tile is some 5 us of a workgroup (3 x 333 to 141 of 6 heads, dq 25, 20 + 4, 15 + 4 with 4, 2, 1; dk and dv 38, 26, 29).
    const int64_t blocks = (rows + 31) / 32;
    if (ring && pairs * blocks >= kUnits * kRingWaves) {
        p.q_ring = true;
        p.resident = dh <= 96 && key_tiles <= tiles_that_fit(dh);
        p.q_parts = 1;
        p.q_part_tiles = static_cast<int32_t>(key_tiles);
        const int64_t per_group = dh > 96 ? 2 * kWideWaves : kPassWaves;
        p.q_tiles = (blocks + per_group - 1) / per_group;
        if (p.resident) {
            p.q_tiles = (blocks + kRingWaves - 1) / kRingWaves;
            const int64_t want = std::max<int64_t>(1, kUnits / units), rounds = std::max<int64_t>(1, (p.q_tiles + want - 1) / want);
            p.q_blocks = static_cast<int32_t>(rounds * kRingWaves);
            p.q_tiles = (blocks + p.q_blocks - 1) / p.q_blocks;
        }
    } else {
        p.q_tiles = std::max<int64_t>(1, (rows + 127) / 128);
        cut(pairs * p.q_tiles, 2 * kUnits, key_tiles, dtype == FREE_BF16 ? 4 : 1, &parts, &per);
        p.q_parts = static_cast<int32_t>(parts);
        p.q_part_tiles = static_cast<int32_t>(per);
    }
    // (fewer rows leave the ring without a tile to be ahead of)
    if (ring && pairs * row_tiles >= kUnits * 4) {
        p.k_ring = true;
        p.kw = 4;                    // (eight, with both blocks of a tile each, leave twice the parts to add)
        p.k_tiles = std::max<int64_t>(1, (static_cast<int64_t>(Nk) + 32 * p.kw - 1) / (32 * p.kw));
        cut(pairs * p.k_tiles, kUnits, row_tiles, 4, &parts, &per);
        p.k_parts = static_cast<int32_t>(parts);
        p.k_units = 1;
    } else {
        p.kw = dtype == FREE_FP32 && Nk <= 32 ? 1 : Nk <= 64 ? 2 : 4;
        p.k_tiles = std::max<int64_t>(1, (static_cast<int64_t>(Nk) + 32 * p.kw - 1) / (32 * p.kw));
        const int64_t steps = dtype == FREE_FP32 ? (row_tiles * p.kw + 3) / 4 : row_tiles;       // (kStepTiles)
        cut(pairs * p.k_tiles, 2 * kUnits, steps, dtype == FREE_BF16 ? 4 : std::min(p.kw, 2), &parts, &per);
        p.k_units = 4 / p.kw;
        p.k_parts = static_cast<int32_t>(parts * p.k_units);
    }
    p.k_part_tiles = static_cast<int32_t>(per);
    return p;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

struct Space {
    size_t lse, delta, dq, dk, dv, bytes;         // offsets
    Space(const Plan& p, int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh) {
        lse = 0;
        delta = up256(static_cast<size_t>(B) * heads * Nq * sizeof(float));
        // the parts of dq and those of dk, dv take turns
        dq = dk = 2 * delta;
        const size_t q = p.q_parts > 1 ? static_cast<size_t>(p.q_parts) * B * Nq * heads * dh * sizeof(float) : 0;
        const size_t kv = p.k_parts > 1 ? up256(static_cast<size_t>(p.k_parts) * B * Nk * kv_heads * dh * sizeof(float)) : 0;
        dv = dk + kv;
        bytes = dq + std::max(up256(q), 2 * kv) + 256;
    }
};

template <typename K>
bool allow(K kern, LdsLimit& limit, size_t lds) { return limit.allow(reinterpret_cast<const void*>(kern), lds); }

template <typename T, int DP, bool kVec>
int32_t launch_dq(const CrossArgs& a, const Plan& p, const RowStats& stats, const GradParts& pt, hipStream_t s) {
    using TL = Tile<T, DP>;
    const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(a.B) * a.kv_heads * p.q_tiles * p.q_parts));
    if constexpr (sizeof(T) == 2 && kVec) {
        if constexpr (DP > 96) {
            if (p.q_ring) {
                auto kern = cross_dq_wide_kernel<DP>;
                static LdsLimit limit;
                constexpr size_t lds = ring_bytes<DP, kWideWaves>(kRing);
                if (!allow(kern, limit, lds)) return FREE_ERR_HIP;
                hipLaunchKernelGGL(kern, grid, dim3(kWideWaves * 64), lds, s, a, stats);
                return launch_ok() ? FREE_OK : FREE_ERR_HIP;
            }
        } else if (p.q_ring) {
            const size_t lds = p.resident ? ring_bytes<DP, kRingWaves>(p.q_part_tiles) : ring_bytes<DP, kPassWaves>(kPassTiles<DP>);
            const auto launch = [&](auto resident) {
                auto kern = cross_dq_ring_kernel<DP, decltype(resident)::value>;
                static LdsLimit limit;
                if (!allow(kern, limit, kLdsBytes)) return FREE_ERR_HIP;
                hipLaunchKernelGGL(kern, grid, dim3((p.resident ? kRingWaves : kPassWaves) * 64), lds, s, a, stats, static_cast<int32_t>(p.q_tiles), p.q_blocks);
                return launch_ok() ? FREE_OK : FREE_ERR_HIP;
            };
            return p.resident ? launch(std::true_type{}) : launch(std::false_type{});
        }
    }
    auto kern = cross_dq_kernel<T, DP, kVec>;
    static LdsLimit limit;
    if (!allow(kern, limit, 4 * TL::kBytes)) return FREE_ERR_HIP;
    hipLaunchKernelGGL(kern, grid, dim3(kThreads), 4 * TL::kBytes, s, a, stats, pt, static_cast<int32_t>(p.q_tiles));
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <typename T, int DP, bool kVec>
int32_t launch_dkv(const CrossArgs& a, const Plan& p, const RowStats& stats, const GradParts& pt, hipStream_t s) {
    using TL = Tile<T, DP>;
    const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(a.B) * a.kv_heads * p.k_tiles * (p.k_parts / p.k_units)));
    if constexpr (sizeof(T) == 2 && kVec) {
        if (p.k_ring) {
            constexpr int NW = kKeyWaves<DP>;
            const size_t lds = ring_bytes<DP, NW>(kRing) + kRing * NW * 256;
            auto kern = cross_dkv_ring_kernel<DP, NW, 4>;
            static LdsLimit limit;
            if (!allow(kern, limit, lds)) return FREE_ERR_HIP;
            hipLaunchKernelGGL(kern, grid, dim3(NW * 64), lds, s, a, stats, pt, static_cast<int32_t>(p.k_tiles));
            return launch_ok() ? FREE_OK : FREE_ERR_HIP;
        }
    }
    const auto launch = [&](auto kw) {
        constexpr int SUB = kStepTiles<T, decltype(kw)::value>, STAGES = SUB == 4 ? 1 : 2;
        constexpr size_t lds = STAGES * SUB * 2 * (TL::kBytes + TL::kRows * sizeof(float));
        auto kern = cross_dkv_kernel<T, DP, decltype(kw)::value, kVec>;
        static LdsLimit limit;
        if (!allow(kern, limit, lds)) return FREE_ERR_HIP;
        hipLaunchKernelGGL(kern, grid, dim3(kThreads), lds, s, a, stats, pt, static_cast<int32_t>(p.k_tiles));
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;
    };
    if constexpr (sizeof(T) == 4) {
        if (p.kw == 1) return launch(std::integral_constant<int, 1>{});
    }
    if (p.kw == 2) return launch(std::integral_constant<int, 2>{});
    return launch(std::integral_constant<int, 4>{});
}

template <typename T, int DP, bool kVec>
int32_t launch_shape(const CrossArgs& a, const Plan& p, const Space& w, char* ws, hipStream_t s) {
    const int64_t pairs = static_cast<int64_t>(a.B) * a.kv_heads;
    if (pairs * p.q_tiles * p.q_parts >= 1 << 23 || pairs * p.k_tiles * (p.k_parts / p.k_units) >= 1 << 23) return FREE_ERR_LIMIT;
    const RowStats stats{reinterpret_cast<float*>(ws + w.lse), reinterpret_cast<float*>(ws + w.delta)};
    if (a.Nq > 0) {
        const GradParts pt{p.q_parts, p.q_part_tiles, reinterpret_cast<float*>(ws + w.dq), nullptr};
        int32_t st = launch_dq<T, DP, kVec>(a, p, stats, pt, s);
        if (st == FREE_OK && p.q_parts > 1) {
            const SumJobs sum{{{pt.sum0, a.dq, a.dq_stride, a.scale}, {}}, p.q_parts, a.kv_heads, a.Nq, a.heads / a.kv_heads, a.dh, pairs};
            st = launch_sum<T, kVec>(sum, 1, s);
        }
        if (st != FREE_OK) return st;
    }
    if (a.Nk == 0) return FREE_OK;
    const GradParts pt{p.k_parts, p.k_part_tiles, reinterpret_cast<float*>(ws + w.dk), reinterpret_cast<float*>(ws + w.dv)};
    const int32_t st = launch_dkv<T, DP, kVec>(a, p, stats, pt, s);
    if (st != FREE_OK || p.k_parts == 1) return st;
    const SumJobs sum{{{pt.sum0, a.dk, a.dk_stride, a.scale}, {pt.sum1, a.dv, a.dv_stride, 1.0f}}, p.k_parts, a.kv_heads, a.Nk, 1, a.dh, pairs};
    return launch_sum<T, kVec>(sum, 2, s);
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
    const auto al = [](const void* x, int64_t stride) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && stride % static_cast<int64_t>(16 / sizeof(T)) == 0; };
    const bool vec = a.dh % static_cast<int>(16 / sizeof(T)) == 0 && al(a.q, a.q_stride) && al(a.k, a.k_stride) && al(a.v, a.v_stride) && al(a.out, a.out_stride) &&
                     al(a.dout, a.dout_stride) && al(a.dq, a.dq_stride) && al(a.dk, a.dk_stride) && al(a.dv, a.dv_stride);
    const Plan p = plan_of(a.B, a.Nq, a.Nk, a.heads, a.kv_heads, a.dh, sizeof(T) == 2 ? FREE_BF16 : FREE_FP32, vec);
    const Space w(p, a.B, a.Nq, a.Nk, a.heads, a.kv_heads, a.dh);
    char* const base = static_cast<char*>(ws);
    return vec ? launch_width<T, true>(a, p, w, base, s) : launch_width<T, false>(a, p, w, base, s);
}

}  // namespace

size_t cross_backward_bytes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype) {
    // (whichever way the tensors' alignment leaves)
    const auto bytes = [&](bool whole) { return Space(plan_of(B, Nq, Nk, heads, kv_heads, dh, dtype, whole), B, Nq, Nk, heads, kv_heads, dh).bytes; };
    return std::max(bytes(true), bytes(false));
}

int32_t launch_cross_backward(const CrossArgs& a, int32_t dtype, void* ws, hipStream_t s) {
    return dtype == FREE_BF16 ? launch_type<bf16_t>(a, ws, s) : launch_type<float>(a, ws, s);
}

}  // namespace freemi
