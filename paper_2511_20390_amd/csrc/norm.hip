// Layer norm over the last axis and its gradient:
//   xh = (x - mean) r,  r = 1 / sqrt(var + eps),  y = xh w_s + b_s
//   dx = r (g - mean(g) - xh mean(g xh)),  g = dy w_s;   dw_s = sum over the rows of sample s of dy xh,  db_s = sum of dy
// with s = row / rows_per_sample (one sample: the affine layer norm) and w_s the given weight, or 1 + it (adaLN's scale).
//
// Both passes are bound by HBM: forward reads x and writes y, backward reads x and dy and writes dx.  So a row is read once and stays
// in registers, over 16 lanes (rows of up to 256 values: 100000 x 130 bf16, forward 40 -> 20 us, gradient 110 -> 46 against a wavefront each) or 1 to 8
// wavefronts; nothing but the inputs is needed again, so no statistics are kept between the passes.
// Variance and products with xh are summed around a mean, so that nothing cancels: every wavefront takes the mean of its own values
// first, without waiting for the others, and sums around that; then the wavefronts of a row exchange all their sums at once - one
// barrier per row - and each moves them to the row's mean:
//     sum (x - mean)^2   = sum over wavefronts of  S2_w + n_w (mean_w - mean)^2
//     sum g (x - mean)   = sum over wavefronts of  GX_w + (mean_w - mean) G_w
// All sums and statistics are fp32.
//
// The weight's gradient sums over rows.  A workgroup walks the rows of one sample with a stride, the next row's loads under way while
// it computes, and adds dy xh and dy to registers, per column; at its end its wavefronts add theirs through LDS, in order, and write
// one partial row; a second launch adds the partial rows of a sample in a fixed order (no atomics: equal inputs give equal bits).  A sample
// that one workgroup walks is written directly.
//
// us, in a row of launches on inputs from memory (at the 5.1 TB/s of a large copy): forward 12288 x 1152 fp32 -> bf16 19.0 (16.7), 16384 x
// 4096 bf16 49 (53), 32768 x 768 bf16 20.5 (19.8); gradient with its second launch 32.0 (27.8), 86 (79), 37 (29.7), and 4096 x 8192 fp32 69 (66),
// 1531 x 1001 fp32 14.2 (3.6: two launches and their round trips).
#include <algorithm>

#include "free_internal.h"
#include "lanes.h"

namespace freemi {

namespace {

constexpr int kThreads = 256;
// threads of a workgroup of the backward pass
constexpr int back_threads(int lanes) { return lanes > 256 ? lanes : 256; }

struct NormArgs {
    const void *x, *dy;
    const float *weight, *bias;
    int32_t stride;              // of weight and bias, and of nothing else: elements from one sample's to the next
    float plus;                  // added to the weight: 0, or 1 for adaLN's scale
    float eps, inv_d;
    int32_t M, D, rows_per_sample;
    void *out;                   // y, or dx
};

// Where the column sums go: a partial row per workgroup, [sample][chunk][2][D] (chunks > 1), or the gradients themselves
struct NormGrad {
    float *part, *dw, *db;
    int32_t chunks, stride;
};

// VE values as they lie in memory.  No alignment is asked of rows (a row of odd width starts anywhere): the memory pipe takes wide
// accesses at any address.  kTail: the last piece of a row may have fewer, `left` of them; what is missing reads as zero.
template <typename T, int VE>
struct Piece {
    uint32_t u[VE * sizeof(T) / 4];
    template <bool kTail>
    __device__ __forceinline__ void load(const T* p, int left) {
        if (!kTail || left >= VE) {
            __builtin_memcpy(u, p, sizeof(u));
        } else {
            T t[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) t[e] = e < left ? p[e] : T{};
            __builtin_memcpy(u, t, sizeof(u));
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (uint32_t& w : u) w = 0;
    }
    __device__ __forceinline__ float at(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u[e]);
        else return __uint_as_float(e % 2 == 0 ? u[e / 2] << 16 : u[e / 2] & 0xffff0000u);
    }
};

template <bool kTail, int VE>
__device__ __forceinline__ void load_vector(const float* p, int left, float (&v)[VE]) {
#pragma unroll
    for (int k = 0; k < VE; k += 4) {
        Piece<float, 4> q;
        q.load<kTail>(p + k, left - k);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k + e] = q.at(e);
    }
}

template <bool kTail, typename T, int VE>
__device__ __forceinline__ void store_piece(T* p, int left, const float (&v)[VE]) {
    uint32_t u[VE * sizeof(T) / 4];
#pragma unroll
    for (int k = 0; k < VE * static_cast<int>(sizeof(T)) / 4; ++k) {
        if constexpr (sizeof(T) == 4) u[k] = __float_as_uint(v[k]);
        else u[k] = pack_bf16_pair(v[2 * k], v[2 * k + 1]);
    }
    if (!kTail || left >= VE) {
        __builtin_memcpy(p, u, sizeof(u));
    } else {
        T t[VE];
        __builtin_memcpy(t, u, sizeof(u));
#pragma unroll
        for (int e = 0; e < VE; ++e)
            if (e < left) p[e] = t[e];
    }
}

// where a lane's pieces of a row lie: piece c at first + c * kStep; LANES lanes have a row
template <int VE, int NV, int LANES>
struct Place {
    static constexpr int kStep = LANES * VE;
    int first, D;
    float values;                // of the row in this wavefront
    __device__ __forceinline__ Place(int D_) : first(static_cast<int>(threadIdx.x) % LANES * VE), D(D_) {
        values = static_cast<float>(LANES < 64 ? D : count(__builtin_amdgcn_readfirstlane(threadIdx.x % LANES / 64)));
    }
    __device__ __forceinline__ int at(int c) const { return first + c * kStep; }
    __device__ __forceinline__ bool has(int c) const { return at(c) < D; }
    __device__ __forceinline__ int left(int c) const { return D - at(c); }
    __device__ __forceinline__ int count(int w) const {          // values of the row in its wavefront w
        int n = 0;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = D - (w * 64 * VE + c * kStep);
            n += k < 0 ? 0 : k > 64 * VE ? 64 * VE : k;
        }
        return n;
    }
};

// the sum over the lanes of a row within a wavefront, in each of them
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (LANES >= 64) return wave_sum(v);
    v += lane_xor<8>(v);
    v += lane_xor<4>(v);
    v += lane_xor<2>(v);
    return v + lane_xor<1>(v);
}

// a weight (nullable) of a piece
template <bool kTail, int VE>
__device__ __forceinline__ void load_weight(const float* w, float plus, int at, int left, float (&v)[VE]) {
    if (w) {
        load_vector<kTail, VE>(w + at, left, v);
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] += plus;
    } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = 1.0f;
    }
}

// Rows of LANES lanes, NV pieces of VE values per lane
template <typename XT, typename OT, int VE, int NV, int LANES, bool kTail>
__global__ __launch_bounds__(kThreads) void norm_forward_kernel(NormArgs a) {
    constexpr int kGroups = kThreads / LANES, WPR = LANES / 64;
    __shared__ float2 red[2][kGroups][WPR > 1 ? WPR : 1];
    const int wave_in_row = threadIdx.x % LANES / 64;
    const int group = LANES < 64 ? threadIdx.x / LANES : __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
    const Place<VE, NV, LANES> at(a.D);
    int parity = 0;
    // every wavefront takes part in every pass (barriers)
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kGroups; base < a.M; base += static_cast<int64_t>(gridDim.x) * kGroups, parity ^= 1) {
        const bool on = base + group < a.M;
        const int64_t row = on ? base + group : base;
        const XT* x = static_cast<const XT*>(a.x) + row * a.D;
        Piece<XT, VE> raw[NV];
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            if (at.has(c)) raw[c].template load<kTail>(x + at.at(c), at.left(c));
            else raw[c].clear();
        }
        float v[NV][VE], s = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                v[c][e] = raw[c].at(e);
                s += v[c][e];
            }
        s = lanes_sum<LANES>(s);
        float mean = at.values > 0.f ? s / at.values : 0.f;       // (quotients: rows of one value have no variance)
        float q = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                v[c][e] -= mean;
                const float d = at.has(c) && (!kTail || e < at.left(c)) ? v[c][e] : 0.f;
                q = fmaf(d, d, q);
            }
        q = lanes_sum<LANES>(q);
        float shift = 0.f;                                        // the wavefront's mean, off the row's
        if constexpr (WPR > 1) {
            if ((threadIdx.x & 63) == 0) red[parity][group][wave_in_row] = make_float2(s, q);
            __syncthreads();
            float total = 0.f, sq = 0.f;
#pragma unroll
            for (int w = 0; w < WPR; ++w) total += red[parity][group][w].x;
            const float row_mean = total / a.D;
#pragma unroll
            for (int w = 0; w < WPR; ++w) {
                const float n = static_cast<float>(at.count(w)), d = n > 0.f ? red[parity][group][w].x / n - row_mean : 0.f;
                sq += fmaf(n * d, d, red[parity][group][w].y);
            }
            shift = mean - row_mean;
            q = sq;
        }
        const float r = 1.0f / sqrtf(q * a.inv_d + a.eps);
        if (!on) continue;
        const int64_t sample = row / a.rows_per_sample;
        const float* w = a.weight ? a.weight + sample * a.stride : nullptr;
        const float* b = a.bias ? a.bias + sample * a.stride : nullptr;
        OT* out = static_cast<OT*>(a.out) + row * a.D;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            if (!at.has(c)) continue;
            float wv[VE], bv[VE], o[VE];
            load_weight<kTail, VE>(w, a.plus, at.at(c), at.left(c), wv);
            if (b) {
                load_vector<kTail, VE>(b + at.at(c), at.left(c), bv);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) bv[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) o[e] = fmaf((v[c][e] + shift) * r, wv[e], bv[e]);
            store_piece<kTail, OT, VE>(out + at.at(c), at.left(c), o);
        }
    }
}

// Workgroup (sample, chunk): rows chunk * groups + group, + chunks * groups, ... of the sample.
template <typename XT, typename OT, int VE, int NV, int LANES, bool kTail>
__global__ __launch_bounds__(back_threads(LANES)) void norm_backward_kernel(NormArgs a, NormGrad gr, int32_t chunks) {
    constexpr int kGroups = back_threads(LANES) / LANES, WPR = LANES / 64;
    // The weight is held in registers: read again for every row its loads would wait behind the next row's (12288 x 1152 35 -> 47 us).  32
    // values per lane leave no registers for the next row's beside it (4096 x 12288 bf16 75 us, with the next row's loads
    // and without the weight 98).
    constexpr bool kAhead = NV * VE <= 20;
    __shared__ float4 red[2][kGroups][WPR > 1 ? WPR : 1];
    extern __shared__ __attribute__((aligned(16))) float cols[];          // [2][NV VE LANES]: column sums of the workgroup (kGroups > 1)
    const int wave_in_row = threadIdx.x % LANES / 64;
    const int group = LANES < 64 ? threadIdx.x / LANES : __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
    const int sample = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const int64_t row0 = static_cast<int64_t>(sample) * a.rows_per_sample;
    const int64_t rows = row0 + a.rows_per_sample < a.M ? a.rows_per_sample : a.M - row0;
    const float* w = a.weight ? a.weight + static_cast<int64_t>(sample) * a.stride : nullptr;
    const Place<VE, NV, LANES> at(a.D);
    float dw[NV][VE], db[NV][VE], held[NV][VE];
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int e = 0; e < VE; ++e) dw[c][e] = db[c][e] = 0.f;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        if (at.has(c)) {
            load_weight<kTail, VE>(w, a.plus, at.at(c), at.left(c), held[c]);
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e) held[c][e] = 0.f;
        }
    }
    Piece<XT, VE> xr[NV];
    Piece<OT, VE> gradr[NV];
    const auto request = [&](int64_t base) {              // this group's row of a pass, the pass's first where there is none
        const int64_t row = row0 + (base + group < rows ? base + group : base);
        const XT* x = static_cast<const XT*>(a.x) + row * a.D;
        const OT* dy = static_cast<const OT*>(a.dy) + row * a.D;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            if (at.has(c)) {
                xr[c].template load<kTail>(x + at.at(c), at.left(c));
                gradr[c].template load<kTail>(dy + at.at(c), at.left(c));
            } else {
                xr[c].clear();
                gradr[c].clear();
            }
        }
    };
    const int64_t step = static_cast<int64_t>(chunks) * kGroups;
    const int64_t start = static_cast<int64_t>(chunk) * kGroups;
    if (kAhead && start < rows) request(start);
    int parity = 0;
    for (int64_t base = start; base < rows; base += step, parity ^= 1) {
        const bool on = base + group < rows;
        float v[NV][VE], g[NV][VE], s = 0.f;
        if constexpr (!kAhead) request(base);
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                v[c][e] = xr[c].at(e);
                g[c][e] = gradr[c].at(e);
                s += v[c][e];
            }
        if (kAhead && base + step < rows) request(base + step);
        s = lanes_sum<LANES>(s);
        const float mean = at.values > 0.f ? s / at.values : 0.f;
        float q = 0.f, sg = 0.f, sgx = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                v[c][e] = at.has(c) && (!kTail || e < at.left(c)) ? v[c][e] - mean : 0.f;
                q = fmaf(v[c][e], v[c][e], q);
                const float gw = g[c][e] * held[c][e];
                sg += gw;
                sgx = fmaf(gw, v[c][e], sgx);
            }
        }
        q = lanes_sum<LANES>(q);
        sg = lanes_sum<LANES>(sg);
        sgx = lanes_sum<LANES>(sgx);
        float shift = 0.f;
        if constexpr (WPR > 1) {
            if ((threadIdx.x & 63) == 0) red[parity][group][wave_in_row] = make_float4(s, q, sg, sgx);
            __syncthreads();
            float total = 0.f;
#pragma unroll
            for (int k = 0; k < WPR; ++k) total += red[parity][group][k].x;
            const float row_mean = total / a.D;
            q = sg = sgx = 0.f;
#pragma unroll
            for (int k = 0; k < WPR; ++k) {
                const float4 p = red[parity][group][k];
                const float n = static_cast<float>(at.count(k)), d = n > 0.f ? p.x / n - row_mean : 0.f;
                q += fmaf(n * d, d, p.y);
                sg += p.z;
                sgx += fmaf(d, p.z, p.w);
            }
            shift = mean - row_mean;
        }
        const float r = 1.0f / sqrtf(q * a.inv_d + a.eps);
        const float m1 = sg * a.inv_d, m2 = r * sgx * a.inv_d;
        if (!on) continue;
        XT* dx = static_cast<XT*>(a.out) + (row0 + base + group) * a.D;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            if (!at.has(c)) continue;
            float o[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float xh = (v[c][e] + shift) * r;
                dw[c][e] = fmaf(g[c][e], xh, dw[c][e]);
                db[c][e] += g[c][e];
                o[e] = r * (g[c][e] * held[c][e] - m1 - xh * m2);
            }
            store_piece<kTail, XT, VE>(dx + at.at(c), at.left(c), o);
        }
    }
    if (gr.dw == nullptr) return;
    float* pw = chunks > 1 ? gr.part + static_cast<int64_t>(blockIdx.x) * 2 * a.D : gr.dw + static_cast<int64_t>(sample) * gr.stride;
    float* pb = chunks > 1 ? pw + a.D : gr.db + static_cast<int64_t>(sample) * gr.stride;
    // the groups' sums: those of a wavefront, then one after the other
    if constexpr (LANES < 64) {
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                dw[c][e] = add_lane_xor<32>(add_lane_xor<16>(dw[c][e]));
                db[c][e] = add_lane_xor<32>(add_lane_xor<16>(db[c][e]));
            }
    }
    constexpr int kLast = LANES < 64 ? back_threads(LANES) / 64 : kGroups;
    const int turn = LANES < 64 ? (threadIdx.x % 64 < LANES ? threadIdx.x / 64 : -1) : group;
    if constexpr (kLast > 1) {
        for (int k = 0; k < kLast; ++k) {
            __syncthreads();
            if (turn != k) continue;
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int e = 0; e < VE; e += 4) {                 // (whole pieces, past the end of a row too)
                    float4* w4 = reinterpret_cast<float4*>(cols + at.at(c) + e);
                    float4* b4 = reinterpret_cast<float4*>(cols + NV * VE * LANES + at.at(c) + e);
                    if (k > 0) {
                        const float4 p = *w4, q = *b4;
                        dw[c][e] += p.x; dw[c][e + 1] += p.y; dw[c][e + 2] += p.z; dw[c][e + 3] += p.w;
                        db[c][e] += q.x; db[c][e + 1] += q.y; db[c][e + 2] += q.z; db[c][e + 3] += q.w;
                    }
                    if (k < kLast - 1) {
                        *w4 = make_float4(dw[c][e], dw[c][e + 1], dw[c][e + 2], dw[c][e + 3]);
                        *b4 = make_float4(db[c][e], db[c][e + 1], db[c][e + 2], db[c][e + 3]);
                    }
                }
        }
        if (turn != kLast - 1) return;
    }
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        if (!at.has(c)) continue;
        store_piece<kTail, float, VE>(pw + at.at(c), at.left(c), dw[c]);
        store_piece<kTail, float, VE>(pb + at.at(c), at.left(c), db[c]);
    }
}

// dw, db [sample] = the partial rows of its chunks, added: 64 columns per workgroup, 16 lanes of four columns, 64 threads per column that
// take every 64th chunk each, then 16 that add four of those, then one.
constexpr int kJoinRows = 64;
__global__ __launch_bounds__(16 * kJoinRows) void norm_join_kernel(NormGrad gr, int32_t D) {
    __shared__ float red[kJoinRows][64];
    const int x = threadIdx.x % 16, k = threadIdx.x / 16, which = blockIdx.y;
    const int64_t sample = blockIdx.z;
    const int col = blockIdx.x * 64 + x * 4, left = D - col;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (left > 0) {
        const float* p = gr.part + (sample * gr.chunks * 2 + which) * D + col;
#pragma unroll 4
        for (int c = k; c < gr.chunks; c += kJoinRows) {
            Piece<float, 4> q;
            q.load<true>(p + static_cast<int64_t>(c) * 2 * D, left);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += q.at(e);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) red[k][x * 4 + e] = s[e];
    __syncthreads();
    const int c = threadIdx.x % 64, r = threadIdx.x / 64;
    const float part = ((red[r][c] + red[r + 16][c]) + red[r + 32][c]) + red[r + 48][c];
    __syncthreads();
    red[r][c] = part;
    __syncthreads();
    if (r != 0 || blockIdx.x * 64 + c >= D) return;
    float total = red[0][c];
#pragma unroll
    for (int j = 1; j < 16; ++j) total += red[j][c];
    (which == 0 ? gr.dw : gr.db)[sample * gr.stride + blockIdx.x * 64 + c] = total;
}

__global__ __launch_bounds__(kThreads) void norm_zero_kernel(NormGrad gr, int32_t D) {
    const int col = blockIdx.x * kThreads + threadIdx.x;
    if (col < D) gr.dw[col] = gr.db[col] = 0.f;
}

// The layouts of a row: pieces of 16 bytes of the wider of the two types (VE values), NV per lane, over LANES lanes.  Forward: one
// wavefront up to 4096 values (64 registers), no exchange between wavefronts.  Backward: x, dy and the two column sums of every value are
// in registers, so 16 to 32 values per lane.
struct Layout {
    int nv, lanes;
};
constexpr int kMaxWidth = 16384;
constexpr int kMaxBlocks = 1 << 22;                                    // grids of less than 2^32 threads

#define FREE_NORM_FORWARD_4(CASE) \
    CASE(4, 1, 16) CASE(4, 2, 16) CASE(4, 4, 16) CASE(4, 2, 64) CASE(4, 3, 64) CASE(4, 5, 64) CASE(4, 8, 64) CASE(4, 16, 64) CASE(4, 16, 256)
#define FREE_NORM_FORWARD_8(CASE) CASE(8, 1, 16) CASE(8, 2, 16) CASE(8, 1, 64) CASE(8, 2, 64) CASE(8, 3, 64) CASE(8, 4, 64) CASE(8, 8, 64) CASE(8, 8, 256)
#define FREE_NORM_BACKWARD_4(CASE) \
    CASE(4, 1, 16) CASE(4, 2, 16) CASE(4, 4, 16) CASE(4, 2, 64) CASE(4, 3, 64) CASE(4, 5, 64) CASE(4, 4, 128) CASE(4, 5, 128) CASE(4, 4, 256) \
    CASE(4, 5, 256) CASE(4, 4, 512) CASE(4, 8, 512)
#define FREE_NORM_BACKWARD_8(CASE) \
    CASE(8, 1, 16) CASE(8, 2, 16) CASE(8, 1, 64) CASE(8, 2, 64) CASE(8, 2, 128) CASE(8, 2, 256) CASE(8, 2, 512) CASE(8, 4, 512)

// the first of the list that holds D
#define FREE_FIRST(VE, NV, LANES) if (VE * NV * LANES >= D) return Layout{NV, LANES};
Layout forward_layout(int ve, int32_t D) {
    if (ve == 8) { FREE_NORM_FORWARD_8(FREE_FIRST) } else { FREE_NORM_FORWARD_4(FREE_FIRST) }
    return {0, 0};
}
Layout backward_layout(int ve, int32_t D) {
    if (ve == 8) { FREE_NORM_BACKWARD_8(FREE_FIRST) } else { FREE_NORM_BACKWARD_4(FREE_FIRST) }
    return {0, 0};
}
#undef FREE_FIRST

template <typename XT, typename OT>
constexpr int kPiece = sizeof(XT) == 2 && sizeof(OT) == 2 ? 8 : 4;

template <typename XT, typename OT>
int32_t forward_of(const NormArgs& a, hipStream_t s) {
    constexpr int VEC = kPiece<XT, OT>;
    const Layout l = forward_layout(VEC, a.D);
    const int groups = kThreads / std::max(1, l.lanes);
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>((static_cast<int64_t>(a.M) + groups - 1) / groups, kMaxBlocks))), block(kThreads);
#define FREE_CASE(VE, NV, LANES)                                                                                                     \
    if (l.nv == NV && l.lanes == LANES) {                                                                                            \
        if (a.D % VE == 0) hipLaunchKernelGGL((norm_forward_kernel<XT, OT, VE, NV, LANES, false>), grid, block, 0, s, a);            \
        else hipLaunchKernelGGL((norm_forward_kernel<XT, OT, VE, NV, LANES, true>), grid, block, 0, s, a);                           \
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;                                                                                 \
    }
    if constexpr (VEC == 8) { FREE_NORM_FORWARD_8(FREE_CASE) } else { FREE_NORM_FORWARD_4(FREE_CASE) }
#undef FREE_CASE
    return FREE_ERR_SHAPE;
}

template <typename XT, typename OT>
int32_t backward_of(const NormArgs& a, const NormGrad& gr, int samples, hipStream_t s) {
    constexpr int VEC = kPiece<XT, OT>;
    const Layout l = backward_layout(VEC, a.D);
    const int threads = back_threads(l.lanes);
    const size_t lds = l.lanes == threads || gr.dw == nullptr ? 0 : static_cast<size_t>(2) * VEC * l.nv * l.lanes * sizeof(float);
    const dim3 grid(samples * gr.chunks), block(threads);
#define FREE_CASE(VE, NV, LANES)                                                                                                     \
    if (l.nv == NV && l.lanes == LANES) {                                                                                            \
        if (a.D % VE == 0) hipLaunchKernelGGL((norm_backward_kernel<XT, OT, VE, NV, LANES, false>), grid, block, lds, s, a, gr, gr.chunks); \
        else hipLaunchKernelGGL((norm_backward_kernel<XT, OT, VE, NV, LANES, true>), grid, block, lds, s, a, gr, gr.chunks);         \
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;                                                                                 \
    }
    if constexpr (VEC == 8) { FREE_NORM_BACKWARD_8(FREE_CASE) } else { FREE_NORM_BACKWARD_4(FREE_CASE) }
#undef FREE_CASE
    return FREE_ERR_SHAPE;
}

// Workgroups per sample in the backward pass.  A group of wavefronts takes `passes` rows; all workgroups should run at once or in full
// rounds (two on every compute unit, of eight wavefronts one), since each ends with sums over its wavefronts and a partial row of the weight's
// gradient that the second launch reads: together some three passes.  Groups and workgroups are counted as the layout of 4-value pieces has
// them, whatever the types: the size of the workspace, which is asked for without them, holds for all.  bf16 rows in 8-value pieces may
// have half as many groups (1025 to 1280 values two for four, 2049 to 2560 one for two) or workgroups of eight wavefronts for four (4097 to 5120);
// the rows are walked with the stride of the layout that is launched, so this moves the balance only.
int chunks_of(int32_t M, int32_t D, int32_t rows_per_sample) {
    const int64_t samples = (static_cast<int64_t>(M) + rows_per_sample - 1) / rows_per_sample;
    const int lanes = backward_layout(4, D).lanes, groups = back_threads(lanes) / lanes;
    const int64_t rows = std::min<int64_t>(M, rows_per_sample), slots = back_threads(lanes) > 256 ? 256 : 2 * 256;
    int64_t best = 1, best_cost = INT64_MAX;
    for (int64_t passes = 1; passes <= 64; ++passes) {
        const int64_t chunks = std::min<int64_t>((rows + passes * groups - 1) / (passes * groups), std::max<int64_t>(1, 2 * slots / samples));
        const int64_t real = (rows + chunks * groups - 1) / (chunks * groups);
        const int64_t cost = (samples * chunks + slots - 1) / slots * (real + 3);
        if (cost < best_cost) {
            best_cost = cost;
            best = chunks;
        }
        if (chunks == 1) break;
    }
    return static_cast<int>(best);
}

}  // namespace

bool norm_covers(int32_t D) { return D >= 1 && D <= kMaxWidth; }

size_t norm_backward_workspace_bytes(int32_t M, int32_t D, int32_t rows_per_sample) {
    const int64_t samples = (static_cast<int64_t>(M) + rows_per_sample - 1) / rows_per_sample;
    const int chunks = M > 0 ? chunks_of(M, D, rows_per_sample) : 1;
    const size_t bytes = chunks > 1 ? static_cast<size_t>(samples) * chunks * 2 * D * sizeof(float) : 0;
    return (bytes + 255) / 256 * 256 + 256;
}

int32_t launch_norm_forward(const void* x, int32_t x_dtype, const float* weight, const float* bias, int32_t stride, bool plus_one,
                            float eps, int32_t M, int32_t D, int32_t rows_per_sample, int32_t dtype, void* out, hipStream_t s) {
    if (M == 0) return FREE_OK;
    const NormArgs a{x, nullptr, weight, bias, stride, plus_one ? 1.f : 0.f, eps, 1.0f / static_cast<float>(D), M, D, rows_per_sample, out};
    if (x_dtype == FREE_FP32) return dtype == FREE_FP32 ? forward_of<float, float>(a, s) : forward_of<float, bf16_t>(a, s);
    return dtype == FREE_FP32 ? forward_of<bf16_t, float>(a, s) : forward_of<bf16_t, bf16_t>(a, s);
}

int32_t launch_norm_backward(const void* dout, int32_t dtype, const void* x, int32_t x_dtype, const float* weight, int32_t stride,
                             bool plus_one, float eps, int32_t M, int32_t D, int32_t rows_per_sample, void* dx, float* dweight,
                             float* dbias, int32_t grad_stride, void* ws, hipStream_t s) {
    NormGrad gr{static_cast<float*>(ws), dweight, dbias, 1, grad_stride};
    if (M == 0) {                                        // an empty sum: one sample, as of any M up to rows_per_sample
        if (dweight == nullptr) return FREE_OK;
        hipLaunchKernelGGL(norm_zero_kernel, dim3((D + kThreads - 1) / kThreads), dim3(kThreads), 0, s, gr, D);
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;
    }
    const int samples = static_cast<int>((static_cast<int64_t>(M) + rows_per_sample - 1) / rows_per_sample);
    if (samples > kMaxBlocks) return FREE_ERR_LIMIT;
    gr.chunks = chunks_of(M, D, rows_per_sample);
    const NormArgs a{x, dout, weight, nullptr, stride, plus_one ? 1.f : 0.f, eps, 1.0f / static_cast<float>(D), M, D, rows_per_sample, dx};
    int32_t st;
    if (x_dtype == FREE_FP32) st = dtype == FREE_FP32 ? backward_of<float, float>(a, gr, samples, s) : backward_of<float, bf16_t>(a, gr, samples, s);
    else st = dtype == FREE_FP32 ? backward_of<bf16_t, float>(a, gr, samples, s) : backward_of<bf16_t, bf16_t>(a, gr, samples, s);
    if (st != FREE_OK || gr.chunks == 1 || dweight == nullptr) return st;
    hipLaunchKernelGGL(norm_join_kernel, dim3((D + 63) / 64, 2, samples), dim3(16 * kJoinRows), 0, s, gr, D);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

}  // namespace freemi
