// The gradient of cross attention (cross_attn.hip), from its inputs, its result and lse:
//   P = exp(scale q k^T - lse) on the keys that count,  delta = sum dout out,  dS = P (dout v^T - delta)
//   dq = scale dS k,   dk = scale dS^T q,   dv = P^T dout      (dk, dv: summed over the queries of all heads that share them)
// Nothing of the size of the scores is kept between the passes: both kernels compute their tiles of scores again.
//  * dq: a workgroup has 128 rows (query and head of a group) and passes tiles of K and V through LDS; it also leaves delta for
//  * dk, dv: a workgroup has 128 or 64 keys and passes tiles of q and dout through LDS, so that both sums stay in registers.
// The score tile's rows are the streamed tensor's rows and its columns the workgroup's own (cross_attn.h), in both.
// Where a launch would have few workgroups the streamed axis is cut in parts, whose fp32 results a second launch adds in order: no
// atomics, equal inputs give equal bits.
#include <algorithm>
#include <cmath>

#include "cross_attn.h"

namespace freemi {

namespace {

constexpr int kThreads = kStreamThreads;

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
    keys.request_mask(t0, lane);
    uint64_t valid = keys.valid_of(t0);
    if (t0 < t1) keys.request(t0, lds_base, lds_base + TL::kBytes, wave, lane, valid);
    keys.request_mask(t0 + 1, lane);

    const int q_row = row < rows ? row : rows - 1, token = over_group(q_row, group), head = kvh * group + q_row - token * group;
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
    if (t0 < t1) keys.deliver(lds, lds + TL::kBytes, tid, valid);
    arrived(qf);
    arrived(gf);
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
            xu32x4_t fk[kRowGroup<T, DP>], fv[kRowGroup<T, DP>];
            Columns<T, DP> ck;
            xf32x16_t st, dp;
            clear_tile(st);
#pragma unroll
            for (int e = 0; e < 16; ++e) dp[e] = -dl;
            read_rows<T, DP>(sK, kb * 32, lane, 0, fk);
            read_rows<T, DP>(sK + TL::kBytes, kb * 32, lane, 0, fv);
            fence();
            row_products<T, DP>(sK, kb * 32, lane, fk, qf, st);
            ck.read(sK, kb * 32, lane, 0);
            fence();
            row_products<T, DP>(sK + TL::kBytes, kb * 32, lane, fv, gf, dp);
            const uint32_t bits = static_cast<uint32_t>(valid >> (32 * kb)) >> (sizeof(T) == 2 ? 8 * g : 4 * g);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float ds = __builtin_amdgcn_exp2f(fmaf(st[e], scale_log2, -lse2)) * dp[e];
                st[e] = bits >> register_row<T>(e, 0) & 1 ? ds : 0.f;
            }
            column_products<T, DP>(sK, kb * 32, lane, ck, st, dq);
        }
        if (t + 1 < t1) keys.deliver(lds + other, lds + other + TL::kBytes, tid, valid_next);
        valid = valid_next;
        keys.k.settle();
    }
    if (pt.parts > 1) store_column<float, kVec, DT>(pt.sum0 + ((part * static_cast<int64_t>(pairs) + pair) * rows + row) * a.dh, a.dh, g, dq, 1.0f, row < rows);
    else store_column<T, kVec, DT>(static_cast<T*>(a.dq) + q_at * a.dq_stride + h_at, a.dh, g, dq, a.scale, row < rows);
}

// ---- dk and dv.  KW wavefronts have 32 keys each; with KW 2 the two halves of a tile's rows go to two wavefronts, whose sums are parts of
// their own.
template <typename T, int DP, int KW, bool kVec>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 && DP <= 80) || DP <= 32 ? 2 : 1) void cross_dkv_kernel(CrossArgs a, const float* delta, GradParts pt, int32_t k_tiles) {
    using H = HeadShape<T, DP>;
    using TL = Tile<T, DP>;
    constexpr int KSTEPS = H::KSTEPS, DT = H::DT, BR = TL::kRows, QW = 4 / KW, RB = BR / 32 / QW;
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
    const int rows = a.Nq * group, key = k_tile * 32 * KW + kw * 32 + l32;
    const int len = attended(a, b);
    const int tiles = (rows + BR - 1) / BR, t0 = part * pt.tiles;
    // keys that do not count have no gradient: a workgroup without others has nothing to sum
    const int t1 = k_tile * 32 * KW < len ? min(t0 + pt.tiles, tiles) : t0;
    const bool there = key < len && (!a.key_mask || a.key_mask[static_cast<int64_t>(b) * a.Nk + key] != 0);

    const int q_row = static_cast<int>(a.q_stride) * static_cast<int>(sizeof(T)), g_row = static_cast<int>(a.dout_stride) * static_cast<int>(sizeof(T));
    const int head_bytes = a.dh * static_cast<int>(sizeof(T));
    const int64_t first_row = static_cast<int64_t>(b) * a.Nq, h0 = static_cast<int64_t>(kvh) * group * a.dh;
    const float inv_scale = 1.0f / a.scale;
    TileStream<T, DP, kVec> queries, grads;
    float lse_next = 0.f, delta_next = 0.f;
    const uint32_t lds_base = lds_address(lds);
    const auto request = [&](int t, int stage) {
        const int r0 = t * BR, token0 = over_group(r0, group), rest = r0 - token0 * group;         // of the group's heads: row r0 + r is token0 + (rest + r) / group
        const int64_t left = a.Nq - token0;
        const auto place = [&](int stride) {
            return [=](int r) {
                const int token = over_group(rest + r, group);
                return token * stride + (rest + r - token * group) * head_bytes;
            };
        };
        const uint32_t to = lds_base + stage * 2 * TL::kBytes;
        queries.request(static_cast<const T*>(a.q) + (first_row + token0) * a.q_stride + h0, (left - 1) * q_row + group * head_bytes, to, wave, lane, a.dh, false, 0,
                        place(q_row));
        grads.request(static_cast<const T*>(a.dout) + (first_row + token0) * a.dout_stride + h0, (left - 1) * g_row + group * head_bytes, to + TL::kBytes, wave, lane,
                      a.dh, false, 0, place(g_row));
        if (tid < BR) {
            const int token = over_group(rest + tid, group), h = rest + tid - token * group;
            const int64_t at = (static_cast<int64_t>(b) * a.heads + kvh * group + h) * a.Nq + token0 + token;
            const bool on = r0 + tid < rows;
            lse_next = on ? a.lse[at] : INFINITY;                       // (rows past the end: probabilities of zero)
            delta_next = on ? delta[at] : 0.f;
        }
    };
    const auto deliver = [&](int stage) {
        char* const sQ = lds + stage * 2 * TL::kBytes;
        queries.deliver(sQ, tid, false, 0);
        grads.deliver(sQ + TL::kBytes, tid, false, 0);
        if (tid < BR) {
            stats[stage * 2 * BR + tid] = -lse_next * inv_scale;
            stats[stage * 2 * BR + BR + tid] = -delta_next;
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
    queries.settle();
    for (int t = t0; t < t1; ++t) {
        const int stage = (t - t0) & 1;
        const char* const sQ = lds + stage * 2 * TL::kBytes;
        if (t + 1 < t1) request(t + 1, stage ^ 1);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row0 = (qw * RB + rb) * 32;
            xu32x4_t fq[kRowGroup<T, DP>], fg[kRowGroup<T, DP>];
            Columns<T, DP> cg, cq;
            xf32x16_t st, dp;
            // the sums begin with -lse / scale and -delta of their row
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const float* const at = stats + stage * 2 * BR + row0 + register_row<T>(4 * e4, g);
                const xf32x4_t lse = *reinterpret_cast<const xf32x4_t*>(at), dl = *reinterpret_cast<const xf32x4_t*>(at + BR);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    st[4 * e4 + i] = lse[i];
                    dp[4 * e4 + i] = dl[i];
                }
            }
            read_rows<T, DP>(sQ, row0, lane, 0, fq);
            read_rows<T, DP>(sQ + TL::kBytes, row0, lane, 0, fg);
            fence();
            row_products<T, DP>(sQ, row0, lane, fq, kf, st);
            cg.read(sQ + TL::kBytes, row0, lane, 0);
            fence();
            row_products<T, DP>(sQ + TL::kBytes, row0, lane, fg, vf, dp);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                st[e] = __builtin_amdgcn_exp2f(st[e] * scale_log2);
                dp[e] *= st[e];
            }
            cq.read(sQ, row0, lane, 0);
            fence();
            column_products<T, DP>(sQ + TL::kBytes, row0, lane, cg, st, dv);
            column_products<T, DP>(sQ, row0, lane, cq, dp, dk);
        }
        if (t + 1 < t1) deliver(stage ^ 1);
        queries.settle();
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
    const int64_t all = a.pairs * rows * per_row, i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= all) return;
    float s[V];
    __builtin_memcpy(s, j.parts + i * V, sizeof(s));
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

template <typename T, bool kVec>
int32_t launch_sum(const SumJobs& a, int jobs, hipStream_t s) {
    constexpr int V = kVec ? 4 : 1;
    const int64_t all = a.pairs * a.tokens * a.group * (a.dh / V);
    hipLaunchKernelGGL((cross_sum_kernel<T, V>), dim3(static_cast<uint32_t>((all + kThreads - 1) / kThreads), jobs), dim3(kThreads), 0, s, a);
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
    {
        const GradParts pt{p.q_parts, p.q_part_tiles, reinterpret_cast<float*>(ws + w.dq), nullptr};
        auto kern = cross_dq_kernel<T, DP, kVec>;
        const size_t lds = 4 * TL::kBytes;
        static LdsLimit limit;
        if (!limit.allow(reinterpret_cast<const void*>(kern), lds)) return FREE_ERR_HIP;
        hipLaunchKernelGGL(kern, dim3(static_cast<uint32_t>(q_blocks)), dim3(kThreads), lds, s, a, delta, pt, static_cast<int32_t>(p.q_tiles));
        if (!launch_ok()) return FREE_ERR_HIP;
        if (p.q_parts > 1) {
            const SumJobs sum{{{pt.sum0, a.dq, a.dq_stride, a.scale}, {}}, p.q_parts, a.kv_heads, a.Nq, a.heads / a.kv_heads, a.dh, pairs};
            const int32_t st = launch_sum<T, kVec>(sum, 1, s);
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
