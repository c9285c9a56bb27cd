// Cross attention to an encoder's states of another length: per sample and head
//   out = softmax(scale q k^T over the keys that count) v,   lse = log sum exp(scale q k^T)
// with a length and a mask per sample over its keys, heads in groups that share keys and values, rows any distance apart; bf16 and fp32.
// One pass over the keys with a running maximum and sum in fp32 (cross_attn.h has the layout of the products).  Keys that do not count are
// not only given no weight: their scores are replaced and their values read as zero, so that nothing they hold, NaN included, gets through.  A
// sample without keys: out zero, lse -inf.
//
// The queries of a group of heads are rows of one problem (row r: token r / group, head r % group), so that keys and values are read once for
// all of them.  Three kernels (us on one MI355X):
//  * cross_ring_kernel, bf16 of whole chunks, 2048 blocks of 32 rows and more: keys that fit stay in LDS, others pass through it.  Bound by the vector
//    unit: of a tile of 64 keys by 32 queries of 72 the softmax is 1360 cycles of a SIMD (16 of them per exponential of a register), the products 704.
//    12288 queries to 64 / 256 keys of 16 heads of 64: 14 / 23 against 17 / 25 with tiles that all pass through; 32760 to 512 of 128: 174, 0.79
//    PFLOP/s, 52 of them the rows' way to and from memory.
//  * cross_many_kernel, the rest of more than 32 rows, fp32, odd strides: a workgroup has 128 or 64 of them and passes tiles of keys through LDS in two
//    stages.  2 x 256 queries to 77 keys: 7.5, a launch and four dependent trips to memory.
//  * cross_few_kernel, up to 32 rows (a single query, a few learned ones): bound by reading keys and values once.  Every wavefront streams key tiles of
//    its own, K straight into the matrix instructions, V through a private piece of LDS; partial results (maximum, sum, out) are joined in order.
//    4 queries of 32 heads of 128 to up to 16384 keys of 8: 33 and 5 for the join, 155 MB of keys and values at 4.7 TB/s.
// Where rows alone leave compute units idle the keys are cut in parts, each a workgroup's, and a second launch joins them.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cross_attn.h"
#include "wave_rows.h"

namespace freemi {

namespace {

constexpr int kThreads = kStreamThreads;
constexpr int kFewRows = 32;
// log2 by which a maximum may grow before the sums are rescaled: they stay below 2^8 times their value, and a branch that is hardly ever taken spares
// 16 products per tile of a result.  It is taken for a wavefront: a row's last bits may depend on the rows beside it.
constexpr float kLazy = 8.0f;
constexpr float kNoScore = -3.402823466e38f;      // a part's maximum where it has keys and all their scores are -inf

// What a launch does: parts of the keys, tiles of a part; partial results [part][pair][row]
struct Parts {
    int32_t parts, tiles;
    float *o, *ml;                                // [..][dh] sums, [..][2] maximum (of the scaled scores, log2) and sum
};

// The end of a row (on: there is one): out and lse, or a part's sums.  m: the maximum that l and o are relative to (log2 of the scaled scores).
template <typename T, bool kVec, int DT>
__device__ __forceinline__ void write_row(const CrossArgs& a, const Parts& pt, int part, int64_t pair, int b, int kvh, int r, int g, float m, float l, bool any,
                                          const xf32x16_t (&o)[DT], bool on) {
    const int group = a.heads / a.kv_heads;
    if (pt.parts > 1) {
        const int64_t at = (part * static_cast<int64_t>(a.B) * a.kv_heads + pair) * a.Nq * group + r;
        store_column<float, kVec, DT>(pt.o + at * a.dh, a.dh, g, o, 1.0f, on);
        if (on && g == 0) {
            pt.ml[2 * at] = any && m == -INFINITY ? kNoScore : m;
            pt.ml[2 * at + 1] = l;
        }
        return;
    }
    const int token = over_group(r, group), head = kvh * group + r - token * group;
    T* const dst = static_cast<T*>(a.out) + (static_cast<int64_t>(b) * a.Nq + token) * a.out_stride + static_cast<int64_t>(head) * a.dh;
    store_column<T, kVec, DT>(dst, a.dh, g, o, any ? 1.0f / l : 0.f, on);
    if (on && a.lse && g == 0) a.lse[(static_cast<int64_t>(b) * a.heads + head) * a.Nq + token] = any ? (m + __builtin_log2f(l)) * kLn2 : -INFINITY;
}

// One online-softmax step of a query column: scores in st (KB blocks of 16 registers, those that do not count at -inf) -> probabilities in
// place; m, l and o follow.
template <int KB, int DT>
__device__ __forceinline__ void softmax_step(xf32x16_t (&st)[KB], float scale_log2, float& m_ref, float& l, xf32x16_t (&o)[DT]) {
    float mx = st[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, st[kb][e]);
    mx = max_lane_xor32(mx);
    // the reference follows the maximum lazily: sums are rescaled once it has grown by a factor of 2^kLazy (true for the first scores)
    if (__builtin_expect(__any((mx - m_ref) * scale_log2 > kLazy), 0)) {
        const float m_new = fmaxf(m_ref, mx);
        const float alpha = m_new == m_ref ? 1.0f : __builtin_amdgcn_exp2f((m_ref - m_new) * scale_log2);
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
        m_ref = m_new;
    }
    const float mb = m_ref == -INFINITY ? 0.f : m_ref * scale_log2;       // (no score yet: probabilities of zero, not NaN)
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            st[kb][e] = __builtin_amdgcn_exp2f(fmaf(st[kb][e], scale_log2, -mb));
            sum += st[kb][e];
        }
    l += sum;
}

// o += V^T P^T for one 32-key block: v at the block's first key, rows VROW bytes apart
template <typename T, int DT, int VROW>
__device__ __forceinline__ void add_values(const char* v, int lane, const xf32x16_t& p, xf32x16_t (&o)[DT]) {
    const int l32 = lane & 31, g = lane >> 5;
    if constexpr (sizeof(T) == 2) {
        const char* at = v + (8 * g + ((lane & 15) >> 2)) * VROW + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const xu32x4_t pk = pack8({p[8 * hh], p[8 * hh + 1], p[8 * hh + 2], p[8 * hh + 3], p[8 * hh + 4], p[8 * hh + 5], p[8 * hh + 6], p[8 * hh + 7]});
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                chunk_product<T>(transposed_chunk(at + hh * 16 * VROW + dt * 64, at + (hh * 16 + 4) * VROW + dt * 64), pk, o[dt]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const float x = *reinterpret_cast<const float*>(v + register_row<T>(e, g) * VROW + (32 * dt + l32) * 4);
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p[e], o[dt], 0, 0, 0);
            }
    }
}

// bytes from a value's row to the next (few rows): bf16, 4 rows x 64 bytes of a transposing read on different banks; fp32, rows four apart on the other 32 banks
template <typename T, int DP>
constexpr int kValueRow = sizeof(T) == 4 ? (DP + 8) * 4 : DP <= 32 ? 64 : DP <= 96 ? 192 : 320;

// Heads of up to 80 leave the registers for three wavefronts per SIMD, if the compiler orders reads and products: 2 x 6144 queries to 300 keys 39 -> 35 us
template <typename T, int DP, int KS, bool kVec>
constexpr bool kThreeWaves = sizeof(T) == 2 && DP <= 80 && KS == 1 && kVec;

// KS wavefronts share the keys of a block of 32 queries: two where there are few blocks
template <typename T, int DP, int KS, bool kVec>
__global__ __launch_bounds__(kThreads, (kThreeWaves<T, DP, KS, kVec> ? 3 : 2)) void cross_many_kernel(CrossArgs a, Parts pt, int32_t q_tiles) {
    using H = HeadShape<T, DP>;
    using TL = Tile<T, DP>;
    constexpr int KSTEPS = H::KSTEPS, DT = H::DT;
    constexpr int BKV = TL::kRows, KB = BKV / 32 / KS, BQ = 128 / KS;     // keys of a tile, 32-key blocks per wavefront, queries
    static_assert(KB >= 1, "a block of keys for each wavefront");
    constexpr bool kAhead = !kThreeWaves<T, DP, KS, kVec>;
    extern __shared__ __attribute__((aligned(16))) char lds[];           // [stage][K, V]

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int qw = wave / KS, kb0 = wave % KS * KB;
    const int pairs = a.B * a.kv_heads, group = a.heads / a.kv_heads;
    // the query tiles of a (sample, head) re-read its keys: all on one XCD, next to each other
    const int per_part = pairs * q_tiles;
    const int part = blockIdx.x / per_part, id = blockIdx.x % per_part;
    const bool by_xcd = pairs % kXcds == 0;
    const int pair = by_xcd ? id % kXcds + kXcds * (id / (kXcds * q_tiles)) : id / q_tiles;
    const int q_tile = by_xcd ? id / kXcds % q_tiles : id % q_tiles;
    const int kvh = pair % a.kv_heads, b = pair / a.kv_heads;
    const int rows = a.Nq * group, row = q_tile * BQ + qw * 32 + l32;
    KeyStream<T, DP, kVec> keys(a, b, kvh);
    const int t0 = part * pt.tiles, t1 = min(t0 + pt.tiles, keys.tiles());
    const uint32_t lds_base = lds_address(lds);
    keys.request_mask(t0, lane);
    uint64_t valid = keys.valid_of(t0);
    if (t0 < t1) keys.request(t0, lds_base, lds_base + TL::kBytes, wave, lane, valid);
    keys.request_mask(t0 + 1, lane);

    const int q_row = row < rows ? row : rows - 1, q_token = over_group(q_row, group);
    const int q_head = kvh * group + q_row - q_token * group;
    const T* const qp = static_cast<const T*>(a.q) + (static_cast<int64_t>(b) * a.Nq + q_token) * a.q_stride + static_cast<int64_t>(q_head) * a.dh;
    xu32x4_t qf[KSTEPS];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) qf[ks] = row_chunk<T, kVec>(qp, 2 * ks + g, a.dh);
    xf32x16_t o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) clear_tile(o[dt]);
    float m_ref = -INFINITY, l = 0.f;
    const float scale_log2 = a.scale * kLog2e;
    bool any = false;
    if (t0 < t1) keys.deliver(lds, lds + TL::kBytes, tid, valid);
    arrived(qf);
    keys.k.settle();
    for (int t = t0; t < t1; ++t) {
        const int stage = (t - t0) & 1, other = (stage ^ 1) * 2 * TL::kBytes;
        const char *const sK = lds + stage * 2 * TL::kBytes, *const sV = sK + TL::kBytes;
        const uint64_t valid_next = keys.valid_of(t + 1);
        if (t + 1 < t1) {
            keys.request(t + 1, lds_base + other, lds_base + other + TL::kBytes, wave, lane, valid_next);
            keys.request_mask(t + 2, lane);
        }
        xf32x16_t st[KB];
        xu32x4_t fk[KB][kRowGroup<T, DP>];
        Columns<T, DP> cv;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            clear_tile(st[kb]);
            read_rows<T, DP>(sK, (kb0 + kb) * 32, lane, 0, fk[kb]);
        }
        if constexpr (kAhead) fence();
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) row_products<T, DP, kAhead>(sK, (kb0 + kb) * 32, lane, fk[kb], qf, st[kb]);
        if constexpr (kAhead) {
            cv.read(sV, kb0 * 32, lane, 0);
            fence();
        }
        any |= valid != 0;
        constexpr uint64_t kFull = BKV == 64 ? ~0ull : 0xffffffffull;
        if (valid != kFull) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const uint32_t bits = static_cast<uint32_t>(valid >> (32 * (kb0 + kb))) >> (sizeof(T) == 2 ? 8 * g : 4 * g);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!(bits >> register_row<T>(e, 0) & 1)) st[kb][e] = -INFINITY;
            }
        }
        softmax_step<KB, DT>(st, scale_log2, m_ref, l, o);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            if (!kAhead || kb > 0) cv.read(sV, (kb0 + kb) * 32, lane, 0);
            column_products<T, DP, kAhead>(sV, (kb0 + kb) * 32, lane, cv, st[kb], o);
        }
        if (t + 1 < t1) keys.deliver(lds + other, lds + other + TL::kBytes, tid, valid_next);
        valid = valid_next;
        keys.k.settle();
    }
    l = add_lane_xor<32>(l);
    if constexpr (KS == 2) {
        // the second half of the keys hands its sums to the first
        static_assert(2 * DT * 4096 + 2 * 512 <= 4 * TL::kBytes, "the partial results must fit in the stages");
        float* const ml = reinterpret_cast<float*>(lds) + qw * 128 + lane;
        char* const so = lds + 1024 + qw * DT * 4096 + lane * 16;
        if (kb0 > 0) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4)
                    *reinterpret_cast<xf32x4_t*>(so + (dt * 4 + e4) * 1024) = xf32x4_t{o[dt][4 * e4], o[dt][4 * e4 + 1], o[dt][4 * e4 + 2], o[dt][4 * e4 + 3]};
            ml[0] = m_ref;
            ml[64] = l;
        }
        __syncthreads();
        if (kb0 > 0) return;
        const float m1 = ml[0], m = fmaxf(m_ref, m1);
        const float a0 = m == m_ref ? 1.0f : __builtin_amdgcn_exp2f((m_ref - m) * scale_log2), a1 = m == m1 ? 1.0f : __builtin_amdgcn_exp2f((m1 - m) * scale_log2);
        l = a0 * l + a1 * ml[64];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const xf32x4_t v = *reinterpret_cast<const xf32x4_t*>(so + (dt * 4 + e4) * 1024);
#pragma unroll
                for (int c = 0; c < 4; ++c) o[dt][4 * e4 + c] = a0 * o[dt][4 * e4 + c] + a1 * v[c];
            }
        m_ref = m;
    }
    write_row<T, kVec, DT>(a, pt, part, pair, b, kvh, row, g, m_ref * scale_log2, l, any, o, row < rows);
}

// bf16 of whole chunks, wavefronts of 32 queries at a time.
// kResident: all keys and values of a (sample, key head) fit in LDS.  They are brought there once, and each wavefront takes one block of queries after
// the other, without a barrier, the next block's queries requested ahead.  Otherwise tiles pass through a ring, and two workgroups share a
// compute unit, so that one multiplies while the other brings or stores its rows (one of eight wavefronts: 32760 queries to 512 keys of 16 heads of 128,
// 199 us; two of four, 174).
template <int DP, bool kResident>
__global__ __launch_bounds__((kResident ? kRingWaves : kPassWaves) * 64, 2) void cross_ring_kernel(CrossArgs a, Parts pt, int32_t chunks, int32_t blocks_per_chunk) {
    using T = bf16_t;
    using H = HeadShape<T, DP>;
    constexpr int KSTEPS = H::KSTEPS, DT = H::DT, NW = kResident ? kRingWaves : kPassWaves, kSlots = kPassTiles<DP>;
    using Ring = PairRing<DP, NW>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ uint64_t masks[kMaxTiles];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, g = lane >> 5;
    const int pairs = a.B * a.kv_heads, group = a.heads / a.kv_heads, part = blockIdx.x / (pairs * chunks);
    const WorkPlace at(blockIdx.x % (pairs * chunks), pairs);
    const int pair = at.pair, chunk = at.place, kvh = pair % a.kv_heads, b = pair / a.kv_heads;
    const int rows = a.Nq * group, blocks = (rows + 31) / 32;
    RingKeys<DP, NW> keys(a, b, kvh, wave, lane);
    const int tiles = keys.tiles(), t0 = part * pt.tiles, t1 = min(t0 + pt.tiles, tiles);
    const uint32_t lds_base = lds_address(lds);
    const auto request = [&](int t, int slot) { keys.request(t, lds_base + slot * Ring::kTileBytes, wave); };
    const auto load_queries = [&](int block, xu32x4_t (&f)[KSTEPS]) {
        const int r = min(lane_row(block, l32), rows - 1), token = over_group(r, group), head = kvh * group + r - token * group;
        const T* const p = static_cast<const T*>(a.q) + (static_cast<int64_t>(b) * a.Nq + token) * a.q_stride + static_cast<int64_t>(head) * a.dh;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) f[ks] = row_chunk<T, true>(p, 2 * ks + g, a.dh);
    };
    const float scale_log2 = a.scale * kLog2e;
    xf32x16_t o[DT];
    xu32x4_t qf[KSTEPS];
    float m_ref, l;
    const auto begin = [&]() {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) clear_tile(o[dt]);
        m_ref = -INFINITY;
        l = 0.f;
    };
    const auto multiply = [&](const char* tile, uint64_t valid) {
        const char* const values = tile + Ring::kSecond;
        xf32x16_t st[2];
        xu32x4_t fk[2][kRowGroup<T, DP>];
        Columns<T, DP> cv;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            clear_tile(st[kb]);
            read_rows<T, DP>(tile, kb * 32, lane, 0, fk[kb]);
        }
        fence();
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) row_products<T, DP>(tile, kb * 32, lane, fk[kb], qf, st[kb]);
        cv.read(values, 0, lane, 0);
        fence();
        if (valid != ~0ull) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const uint32_t bits = static_cast<uint32_t>(valid >> (32 * kb)) >> (8 * g);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!(bits >> register_row<T>(e, 0) & 1)) st[kb][e] = -INFINITY;
            }
        }
        softmax_step<2, DT>(st, scale_log2, m_ref, l, o);
        column_products<T, DP>(values, 0, lane, cv, st[0], o);
        cv.read(values, 32, lane, 0);
        column_products<T, DP>(values, 32, lane, cv, st[1], o);
    };
    const auto finish = [&](int block, bool any) {
        l = add_lane_xor<32>(l);
        const int r = lane_row(block, l32);
        write_row<T, true, DT>(a, pt, part, pair, b, kvh, r, g, m_ref * scale_log2, l, any, o, r < rows);
    };

    if constexpr (kResident) {
        for (int t = 0; t < tiles; ++t) request(t, t);
        const int first = chunk * blocks_per_chunk, last = min(first + blocks_per_chunk, blocks);
        if (first + wave < last) load_queries(first + wave, qf);
        const bool any = bring_keys(keys, lds, masks, 1, wave, lane);
        for (int block = first + wave; block < last; block += NW) {
            xu32x4_t next[KSTEPS];
            arrived(qf);
            if (block + NW < last) load_queries(block + NW, next);
            begin();
            for (int t = 0; t < tiles; ++t) {
                const uint64_t valid = keys.mask ? masks[t] : keys_below(keys.len - t * Tile<T, DP>::kRows);
                multiply(lds + t * Ring::kTileBytes, valid);
            }
            finish(block, any);
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) qf[ks] = next[ks];
        }
    } else {
        const int block = wave_block(chunk, NW, wave);       // (past the last one: it takes part in the loads, and has no row)
#pragma unroll
        for (int s = 0; s < kSlots - 1; ++s)
            if (t0 + s < t1) request(t0 + s, s);
        load_queries(block, qf);
        begin();
        bool any = false;
        arrived(qf);
        int slot = 0, free_slot = kSlots - 1;
        for (int t = t0; t < t1; ++t) {
            const uint64_t valid = keys.valid(t, lane);
            any |= valid != 0;
            // tile t has arrived, and everybody is done with the one before it
            if (t + kSlots - 1 <= t1) wait_vm_barrier<(kSlots - 2) * Ring::N>();
            else wait_vm_barrier<0>();
            char* const tile = lds + slot * Ring::kTileBytes;
            if (keys.mask && valid != ~0ull) {
                keys.drop(tile, 1, valid, wave, lane);
                __syncthreads();
            }
            if (t + kSlots - 1 < t1) request(t + kSlots - 1, free_slot);
            multiply(tile, valid);
            free_slot = slot;
            slot = slot + 1 == kSlots ? 0 : slot + 1;
        }
        finish(block, any);
    }
}

// Up to 32 rows per (sample, key head): workgroup (part, pair), its four wavefronts take the part's key tiles of 32 in turn
template <typename T, int DP, bool kVec>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void cross_few_kernel(CrossArgs a, Parts pt) {
    using H = HeadShape<T, DP>;
    constexpr int E = H::E, CH = H::CH, KSTEPS = H::KSTEPS, DT = H::DT;
    constexpr int VROW = kValueRow<T, DP>, kWaveV = 32 * VROW + (sizeof(T) == 4 ? 128 : 0), NV = CH / 2;
    constexpr int kWaveLds = kWaveV > DT * 4096 + 512 ? kWaveV : DT * 4096 + 512;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int pairs = a.B * a.kv_heads, group = a.heads / a.kv_heads;
    const int part = blockIdx.x / pairs, pair = blockIdx.x % pairs;
    const int kvh = pair % a.kv_heads, b = pair / a.kv_heads;
    const int rows = a.Nq * group, row = l32;
    const int len = attended(a, b);
    const int t0 = part * pt.tiles + wave, t1 = min((part + 1) * pt.tiles, (len + 31) / 32);
    const T* const kp = static_cast<const T*>(a.k) + static_cast<int64_t>(b) * a.Nk * a.k_stride + static_cast<int64_t>(kvh) * a.dh;
    const T* const vp = static_cast<const T*>(a.v) + static_cast<int64_t>(b) * a.Nk * a.v_stride + static_cast<int64_t>(kvh) * a.dh;
    const uint8_t* const mask = a.key_mask ? a.key_mask + static_cast<int64_t>(b) * a.Nk : nullptr;
    const int k_row = static_cast<int>(a.k_stride) * static_cast<int>(sizeof(T)), v_row = static_cast<int>(a.v_stride) * static_cast<int>(sizeof(T));
    char* const sV = lds + wave * kWaveLds;
    const int key_at = block_row<T>(l32);

    xu32x4_t kf[KSTEPS], vf[NV];
    uint32_t mask_next = 1;
    const auto fetch = [&](int t) {
        const int64_t kv0 = static_cast<int64_t>(t) * 32;
        const auto kb = rows_buffer(kp + kv0 * a.k_stride, len - kv0, a.k_stride, a.dh), vb = rows_buffer(vp + kv0 * a.v_stride, len - kv0, a.v_stride, a.dh);
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) kf[ks] = buffer_chunk<T, kVec>(kb, key_at * k_row + (2 * ks + g) * 16, 2 * ks + g, a.dh);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int idx = lane + 64 * i, r = idx / CH, c = idx % CH;
            vf[i] = buffer_chunk<T, kVec>(vb, r * v_row + c * 16, c, a.dh);
        }
        if (mask) mask_next = l32 < len - kv0 ? mask[kv0 + l32] : 0;
    };
    if (t0 < t1) fetch(t0);
    const int q_row = row < rows ? row : rows - 1, q_token = q_row / group;
    const T* const qp = static_cast<const T*>(a.q) + (static_cast<int64_t>(b) * a.Nq + q_token) * a.q_stride +
                        static_cast<int64_t>(kvh * group + q_row - q_token * group) * a.dh;
    xu32x4_t qf[KSTEPS];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) qf[ks] = row_chunk<T, kVec>(qp, 2 * ks + g, a.dh);
    xf32x16_t o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) clear_tile(o[dt]);
    float m_ref = -INFINITY, l = 0.f;
    const float scale_log2 = a.scale * kLog2e;
    bool any = false;
    arrived(qf);
    for (int t = t0; t < t1; t += 4) {
        uint64_t valid = keys_below(min(len - t * 32, 32));
        if (mask) valid &= __ballot(mask_next != 0);
        any |= valid != 0;
        xf32x16_t st[1];
        clear_tile(st[0]);
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) chunk_product<T>(kf[ks], qf[ks], st[0]);
        // (a wavefront's LDS accesses keep their order; the fences keep the compiler's)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int idx = lane + 64 * i, r = idx / CH, c = idx % CH;
            if (mask && !(valid >> r & 1)) vf[i] = xu32x4_t{0, 0, 0, 0};
            *reinterpret_cast<xu32x4_t*>(sV + r * VROW + c * 16) = vf[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (t + 4 < t1) fetch(t + 4);
        if ((valid & 0xffffffffull) != 0xffffffffull) {
            const uint32_t bits = static_cast<uint32_t>(valid) >> (sizeof(T) == 2 ? 8 * g : 4 * g);
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (!(bits >> register_row<T>(e, 0) & 1)) st[0][e] = -INFINITY;
        }
        softmax_step<1, DT>(st, scale_log2, m_ref, l, o);
        add_values<T, DT, VROW>(sV, lane, st[0], o);
    }
    l = add_lane_xor<32>(l);
    // the wavefronts' sums, in order
    __shared__ int seen[4];
    if (lane == 0) seen[wave] = any;
    float* const ml = reinterpret_cast<float*>(lds + wave * kWaveLds + DT * 4096);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (wave > 0) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                *reinterpret_cast<xf32x4_t*>(sV + (dt * 4 + e4) * 1024 + lane * 16) = xf32x4_t{o[dt][4 * e4], o[dt][4 * e4 + 1], o[dt][4 * e4 + 2], o[dt][4 * e4 + 3]};
        if (g == 0) {
            ml[l32] = m_ref;
            ml[32 + l32] = l;
        }
    }
    __syncthreads();
    if (wave > 0) return;
    float m = m_ref;
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        any |= seen[w] != 0;
        m = fmaxf(m, reinterpret_cast<const float*>(lds + w * kWaveLds + DT * 4096)[l32]);
    }
    const auto factor = [&](float from) { return from == m ? 1.0f : __builtin_amdgcn_exp2f((from - m) * scale_log2); };
    const float a0 = factor(m_ref);
    l *= a0;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= a0;
    for (int w = 1; w < 4; ++w) {
        const float* const wml = reinterpret_cast<const float*>(lds + w * kWaveLds + DT * 4096);
        const float aw = factor(wml[l32]);
        l += aw * wml[32 + l32];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const xf32x4_t v = *reinterpret_cast<const xf32x4_t*>(lds + w * kWaveLds + (dt * 4 + e4) * 1024 + lane * 16);
#pragma unroll
                for (int c = 0; c < 4; ++c) o[dt][4 * e4 + c] += aw * v[c];
            }
    }
    write_row<T, kVec, DT>(a, pt, part, pair, b, kvh, row, g, m * scale_log2, l, any, o, row < rows);
}

// The parts of a row's sums, added in order: WPR wavefronts per row take them in turn, lane p having part p's maximum and sum (at most 64
// parts)
template <typename T, int WPR>
__global__ __launch_bounds__(kThreads) void cross_join_kernel(CrossArgs a, Parts pt) {
    __shared__ float sums[4][128];
    const int group = a.heads / a.kv_heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = wave % WPR;
    const int64_t per_pair = static_cast<int64_t>(a.Nq) * group, all = static_cast<int64_t>(a.B) * a.kv_heads * per_pair;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (4 / WPR) + wave / WPR, at = row < all ? row : all - 1;
    const float mp = lane < pt.parts ? pt.ml[2 * (lane * all + at)] : -INFINITY, lp = lane < pt.parts ? pt.ml[2 * (lane * all + at) + 1] : 0.f;
    float m = max_lane_xor32(mp);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
    // (parts without keys are left out; one with keys counts however small its weight is: its sums may be NaN)
    const bool keyed = mp != -INFINITY;
    const uint64_t keyed_parts = __ballot(keyed);
    const float w = !keyed ? 0.f : mp == m ? 1.0f : __builtin_amdgcn_exp2f(mp - m);
    const float l = wave_sum(keyed ? w * lp : 0.f);
    float o[2] = {0.f, 0.f};
    for (int p = first; p < pt.parts; p += WPR) {
        if (!(keyed_parts >> p & 1)) continue;
        const float wp = __shfl(w, p, 64);
        const float* const from = pt.o + (p * all + at) * a.dh;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (lane + 64 * k < a.dh) o[k] = fmaf(wp, from[lane + 64 * k], o[k]);
    }
    if constexpr (WPR > 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k) sums[wave][lane + 64 * k] = o[k];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 1; i < WPR; ++i) o[k] += sums[i][lane + 64 * k];
    }
    if (row >= all) return;
    const int64_t pair = at / per_pair, r = at - pair * per_pair, token = r / group;
    const int b = static_cast<int>(pair / a.kv_heads), head = static_cast<int>(pair % a.kv_heads * group + (r - token * group));
    T* const out = static_cast<T*>(a.out) + (static_cast<int64_t>(b) * a.Nq + token) * a.out_stride + static_cast<int64_t>(head) * a.dh;
    const float inv = m == -INFINITY ? 0.f : 1.0f / l;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (lane + 64 * k < a.dh) store_f(out + lane + 64 * k, o[k] * inv);
    if (a.lse && lane == 0) a.lse[(static_cast<int64_t>(b) * a.heads + head) * a.Nq + token] = m == -INFINITY ? m : (m + __builtin_log2f(l)) * kLn2;
}

// How a problem is cut; by its sizes and by whether rows are whole aligned chunks, not by the device (a workspace is as large as either way needs)
struct Plan {
    bool few, ring, resident;
    int ks;                                       // wavefronts that share a query block's keys (many rows)
    int32_t parts, tiles;                         // tiles: of 32 keys (few rows, fp32) or 64
    int64_t q_tiles;                              // workgroups of a (sample, key head) and part
    int32_t blocks;                               // resident: 32-query blocks of each
};
constexpr int kUnits = 256;

Plan plan_of(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype, bool ring_covers) {
    const int64_t pairs = static_cast<int64_t>(B) * kv_heads, rows = static_cast<int64_t>(Nq) * (heads / kv_heads);
    Plan p{};
    p.few = rows <= kFewRows;
    p.ks = 1;
    p.q_tiles = 1;
    const int tile = p.few || dtype == FREE_FP32 ? 32 : 64;
    const int64_t tiles = std::max<int64_t>(1, (static_cast<int64_t>(Nk) + tile - 1) / tile);
    const int64_t blocks = (rows + 31) / 32;
    if (!p.few && dtype == FREE_BF16 && ring_covers && pairs * blocks >= kUnits * kRingWaves) {
        p.ring = true;
        p.resident = tiles <= tiles_that_fit(dh);
        p.parts = 1;
        p.tiles = static_cast<int32_t>(tiles);
        p.q_tiles = (blocks + kPassWaves - 1) / kPassWaves;
        if (p.resident) {
            p.q_tiles = (blocks + kRingWaves - 1) / kRingWaves;
            // one workgroup per compute unit
            const int64_t want = std::max<int64_t>(1, kUnits / std::max<int64_t>(pairs, 1)), rounds = std::max<int64_t>(1, (p.q_tiles + want - 1) / want);
            p.blocks = static_cast<int32_t>(rounds * kRingWaves);
            p.q_tiles = (blocks + p.blocks - 1) / p.blocks;
        }
        return p;
    }
    if (!p.few) {
        p.q_tiles = (rows + 127) / 128;
        if (dtype == FREE_BF16 && pairs * p.q_tiles <= 2 * kUnits) {
            p.ks = 2;
            p.q_tiles = (rows + 63) / 64;
        }
    }
    const int64_t work = pairs * p.q_tiles, least = p.few ? 8 : dtype == FREE_BF16 ? 4 : 2, want = 2 * kUnits;      // tiles of a part; workgroups
    int64_t parts = 1;
    if (work < want) parts = std::max<int64_t>(1, std::min(want / std::max<int64_t>(work, 1), tiles / least));
    parts = std::min<int64_t>(parts, 64);
    p.tiles = static_cast<int32_t>((tiles + parts - 1) / parts);
    p.parts = static_cast<int32_t>((tiles + p.tiles - 1) / p.tiles);
    return p;
}

template <typename T, int DP, bool kVec>
int32_t launch_shape(const CrossArgs& a, const Plan& p, const Parts& pt, hipStream_t s) {
    const int64_t blocks = static_cast<int64_t>(a.B) * a.kv_heads * p.q_tiles * p.parts;
    if (blocks >= 1 << 23) return FREE_ERR_LIMIT;
    constexpr int DT = HeadShape<T, DP>::DT;
    if (p.few) {
        const size_t lds = 4 * std::max<size_t>(32 * kValueRow<T, DP> + (sizeof(T) == 4 ? 128 : 0), DT * 4096 + 512);
        auto kern = cross_few_kernel<T, DP, kVec>;
        static LdsLimit limit;
        if (!limit.allow(reinterpret_cast<const void*>(kern), lds)) return FREE_ERR_HIP;
        hipLaunchKernelGGL(kern, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), lds, s, a, pt);
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;
    }
    if constexpr (sizeof(T) == 2 && kVec) {
        if (p.ring) {
            const size_t lds = p.resident ? ring_bytes<DP, kRingWaves>(p.tiles) : ring_bytes<DP, kPassWaves>(kPassTiles<DP>);
            const auto launch = [&](auto resident) {
                auto kern = cross_ring_kernel<DP, decltype(resident)::value>;
                static LdsLimit limit;
                if (!limit.allow(reinterpret_cast<const void*>(kern), kLdsBytes)) return FREE_ERR_HIP;
                hipLaunchKernelGGL(kern, dim3(static_cast<uint32_t>(blocks)), dim3((p.resident ? kRingWaves : kPassWaves) * 64), lds, s, a, pt, static_cast<int32_t>(p.q_tiles),
                                   p.blocks);
                return launch_ok() ? FREE_OK : FREE_ERR_HIP;
            };
            return p.resident ? launch(std::true_type{}) : launch(std::false_type{});
        }
    }
    constexpr size_t lds = 4 * Tile<T, DP>::kBytes;
    const auto launch = [&](auto ks) {
        auto kern = cross_many_kernel<T, DP, decltype(ks)::value, kVec>;
        static LdsLimit limit;
        if (!limit.allow(reinterpret_cast<const void*>(kern), lds)) return FREE_ERR_HIP;
        hipLaunchKernelGGL(kern, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), lds, s, a, pt, static_cast<int32_t>(p.q_tiles));
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;
    };
    if constexpr (sizeof(T) == 2) {
        if (p.ks == 2) return launch(std::integral_constant<int, 2>{});
    }
    return launch(std::integral_constant<int, 1>{});
}

template <typename T, bool kVec>
int32_t launch_width(const CrossArgs& a, const Plan& p, const Parts& pt, hipStream_t s) {
    if (a.dh <= 32) return launch_shape<T, 32, kVec>(a, p, pt, s);
    if (a.dh <= 64) return launch_shape<T, 64, kVec>(a, p, pt, s);
    if (a.dh <= 80) return launch_shape<T, 80, kVec>(a, p, pt, s);
    if (a.dh <= 96) return launch_shape<T, 96, kVec>(a, p, pt, s);
    return launch_shape<T, 128, kVec>(a, p, pt, s);
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T>
bool whole_chunks(const CrossArgs& a) {
    const auto al = [](const void* x, int64_t stride) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && stride % static_cast<int64_t>(16 / sizeof(T)) == 0; };
    return a.dh % static_cast<int>(16 / sizeof(T)) == 0 && al(a.q, a.q_stride) && al(a.k, a.k_stride) && al(a.v, a.v_stride) && al(a.out, a.out_stride);
}

size_t space_of(const Plan& p, int32_t B, int32_t Nq, int32_t heads, int32_t dh) {
    if (p.parts == 1) return 256;
    const size_t rows = static_cast<size_t>(B) * Nq * heads * p.parts;
    return up256(rows * dh * sizeof(float)) + up256(rows * 2 * sizeof(float));
}

template <typename T>
int32_t launch_type(const CrossArgs& a, void* ws, hipStream_t s) {
    const bool vec = whole_chunks<T>(a);
    const Plan p = plan_of(a.B, a.Nq, a.Nk, a.heads, a.kv_heads, a.dh, sizeof(T) == 2 ? FREE_BF16 : FREE_FP32, vec);
    Parts pt{p.parts, p.tiles, nullptr, nullptr};
    if (p.parts > 1) {
        pt.o = static_cast<float*>(ws);
        pt.ml = reinterpret_cast<float*>(static_cast<char*>(ws) + up256(static_cast<size_t>(a.B) * a.Nq * a.heads * p.parts * a.dh * sizeof(float)));
    }
    const int32_t st = vec ? launch_width<T, true>(a, p, pt, s) : launch_width<T, false>(a, p, pt, s);
    if (st != FREE_OK || p.parts == 1) return st;
    const int64_t rows = static_cast<int64_t>(a.B) * a.Nq * a.heads;
    if (p.parts > 8) hipLaunchKernelGGL((cross_join_kernel<T, 4>), dim3(static_cast<uint32_t>(rows)), dim3(kThreads), 0, s, a, pt);
    else hipLaunchKernelGGL((cross_join_kernel<T, 1>), dim3(static_cast<uint32_t>((rows + 3) / 4)), dim3(kThreads), 0, s, a, pt);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

}  // namespace

size_t cross_forward_bytes(int32_t B, int32_t Nq, int32_t Nk, int32_t heads, int32_t kv_heads, int32_t dh, int32_t dtype) {
    // (whichever way the tensors' alignment leaves)
    return std::max(space_of(plan_of(B, Nq, Nk, heads, kv_heads, dh, dtype, true), B, Nq, heads, dh),
                    space_of(plan_of(B, Nq, Nk, heads, kv_heads, dh, dtype, false), B, Nq, heads, dh));
}

int32_t launch_cross_forward(const CrossArgs& a, int32_t dtype, void* ws, hipStream_t s) {
    return dtype == FREE_BF16 ? launch_type<bf16_t>(a, ws, s) : launch_type<float>(a, ws, s);
}

}  // namespace freemi
