// Layer norm over the last axis and its gradient:
//   xh = (x - mean) r,  r = 1 / sqrt(var + eps),  y = xh w_s + b_s
//   dx = r (g - mean(g) - xh mean(g xh)),  g = dy w_s;   dw_s = sum over the rows of sample s of dy xh,  db_s = sum of dy
// with s = row / rows_per_sample (one sample: the affine layer norm) and w_s the given weight, or 1 + it (adaLN's scale).
//
// Both passes are bound by HBM: forward reads x and writes y, backward reads x and dy and writes dx.  So a row is read once and stays
// in registers: 1 to 16 wavefronts hold it, mean and variance are taken from the registers one after the other (centred, so that
// nothing cancels), and the gradient's two sums likewise; nothing but the inputs is needed again, so no statistics are kept between
// the passes.  All sums and statistics are fp32.
//
// The weight's gradient sums over rows.  A workgroup walks the rows of one sample with a stride and adds dy xh and dy to registers, per
// column; at its end its wavefronts add theirs through LDS, in order, and write one partial row; a second launch adds the partial rows
// of a sample in a fixed order (no atomics: equal inputs give equal bits).  A sample that one workgroup walks is written directly.
#include <algorithm>

#include "free_internal.h"
#include "lanes.h"

namespace freemi {

namespace {

constexpr int kThreads = 256;

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

template <typename T, int VE>
__device__ __forceinline__ void load_chunk(const T* p, float (&v)[VE]) {
    if constexpr (VE == 1) {
        v[0] = load_f(p);
    } else if constexpr (sizeof(T) == 4) {
        const float4 f = *reinterpret_cast<const float4*>(p);
        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    } else {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
        v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
    }
}

template <typename T, int VE>
__device__ __forceinline__ void store_chunk(T* p, const float (&v)[VE]) {
    if constexpr (VE == 1) store_f(p, v[0]);
    else if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16_pair(v[0], v[1]), pack_bf16_pair(v[2], v[3]));
}

// The sum over the WPR wavefronts of a row, in every lane.  slot: WPR floats of LDS.  A kernel uses two or more slots in turn: between
// the read of one and its next write lies the barrier of another.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* slot, int wave_in_row) {
    v = wave_sum(v);
    if constexpr (WPR == 1) return v;
    if ((threadIdx.x & 63) == 0) slot[wave_in_row] = v;
    __syncthreads();
    float s = slot[0];
#pragma unroll
    for (int w = 1; w < WPR; ++w) s += slot[w];
    return s;
}

// Weight (nullable) of a chunk.  Requested ahead of the sums it waits for nothing but the cache.
template <int VE>
__device__ __forceinline__ void load_weight(const float* w, float plus, int at, float (&v)[VE]) {
    if (w) {
        load_chunk<float, VE>(w + at, v);
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] += plus;
    } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = 1.0f;
    }
}

// One row per group of WPR wavefronts, NV chunks of VE values per lane.
template <typename XT, typename OT, int VE, int NV, int WPR>
__global__ __launch_bounds__(WPR > 4 ? WPR * 64 : kThreads) void norm_forward_kernel(NormArgs a) {
    constexpr int kGroups = WPR > 4 ? 1 : 4 / WPR;
    __shared__ float red[kGroups][2][WPR];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int group = wave / WPR, wave_in_row = wave % WPR;
    constexpr int kStep = WPR * 64 * VE;
    const int first = (wave_in_row * 64 + lane) * VE;
    // every wavefront takes part in every pass (barriers in row_sum)
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kGroups; base < a.M; base += static_cast<int64_t>(gridDim.x) * kGroups) {
        const bool on = base + group < a.M;
        const int64_t row = on ? base + group : base;
        const XT* x = static_cast<const XT*>(a.x) + row * a.D;
        float v[NV][VE];
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int at = first + c * kStep;
            if (at < a.D) {
                load_chunk<XT, VE>(x + at, v[c]);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) v[c][e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) s += v[c][e];
        }
        const float mean = row_sum<WPR>(s, red[group][0], wave_in_row) / a.D;       // (a quotient: rows of one value have no variance)
        float q = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int at = first + c * kStep;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                v[c][e] = at < a.D ? v[c][e] - mean : 0.f;
                q = fmaf(v[c][e], v[c][e], q);
            }
        }
        const float r = 1.0f / sqrtf(row_sum<WPR>(q, red[group][1], wave_in_row) * a.inv_d + a.eps);
        if (!on) continue;
        const int64_t sample = row / a.rows_per_sample;
        const float* w = a.weight ? a.weight + sample * a.stride : nullptr;
        const float* b = a.bias ? a.bias + sample * a.stride : nullptr;
        OT* out = static_cast<OT*>(a.out) + row * a.D;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int at = first + c * kStep;
            if (at >= a.D) continue;
            float wv[VE], bv[VE], o[VE];
            load_weight<VE>(w, a.plus, at, wv);
            if (b) {
                load_chunk<float, VE>(b + at, bv);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) bv[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) o[e] = fmaf(v[c][e] * r, wv[e], bv[e]);
            store_chunk<OT, VE>(out + at, o);
        }
    }
}

// Workgroup (sample, chunk): rows chunk * groups + group, + chunks * groups, ... of the sample.
template <typename XT, typename OT, int VE, int NV, int WPR>
__global__ __launch_bounds__(WPR > 4 ? WPR * 64 : kThreads) void norm_backward_kernel(NormArgs a, NormGrad gr, int32_t chunks) {
    constexpr int kGroups = WPR > 4 ? 1 : 4 / WPR;
    __shared__ float red[kGroups][4][WPR];
    extern __shared__ float cols[];                       // [2][D]: column sums of the workgroup (kGroups > 1)
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int group = wave / WPR, wave_in_row = wave % WPR;
    const int sample = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const int64_t row0 = static_cast<int64_t>(sample) * a.rows_per_sample;
    const int rows = static_cast<int>(row0 + a.rows_per_sample < a.M ? a.rows_per_sample : a.M - row0);
    const float* w = a.weight ? a.weight + static_cast<int64_t>(sample) * a.stride : nullptr;
    const int first = (wave_in_row * 64 + lane) * VE;
    constexpr int kStep = WPR * 64 * VE;
    float dw[NV][VE], db[NV][VE];
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int e = 0; e < VE; ++e) dw[c][e] = db[c][e] = 0.f;
    for (int64_t base = chunk * kGroups; base < rows; base += chunks * kGroups) {
        const bool on = base + group < rows;
        const int64_t row = row0 + (on ? base + group : base);
        const XT* x = static_cast<const XT*>(a.x) + row * a.D;
        const OT* dy = static_cast<const OT*>(a.dy) + row * a.D;
        float v[NV][VE], g[NV][VE];
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int at = first + c * kStep;
            if (at < a.D) {
                load_chunk<XT, VE>(x + at, v[c]);
                load_chunk<OT, VE>(dy + at, g[c]);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) v[c][e] = g[c][e] = 0.f;
            }
        }
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < VE; ++e) s += v[c][e];
        const float mean = row_sum<WPR>(s, red[group][0], wave_in_row) / a.D;       // (a quotient: rows of one value have no variance)
        float q = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int at = first + c * kStep;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                v[c][e] = at < a.D ? v[c][e] - mean : 0.f;
                q = fmaf(v[c][e], v[c][e], q);
            }
        }
        const float r = 1.0f / sqrtf(row_sum<WPR>(q, red[group][1], wave_in_row) * a.inv_d + a.eps);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int at = first + c * kStep;
            if (at < a.D) {
                float wv[VE];
                load_weight<VE>(w, a.plus, at, wv);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    v[c][e] *= r;
                    if (on) {
                        dw[c][e] = fmaf(g[c][e], v[c][e], dw[c][e]);
                        db[c][e] += g[c][e];
                    }
                    g[c][e] *= wv[e];
                    s1 += g[c][e];
                    s2 = fmaf(g[c][e], v[c][e], s2);
                }
            }
        }
        const float m1 = row_sum<WPR>(s1, red[group][2], wave_in_row) * a.inv_d;
        const float m2 = row_sum<WPR>(s2, red[group][3], wave_in_row) * a.inv_d;
        if (on) {
            XT* dx = static_cast<XT*>(a.out) + row * a.D;
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int at = first + c * kStep;
                if (at >= a.D) continue;
                float o[VE];
#pragma unroll
                for (int e = 0; e < VE; ++e) o[e] = r * (g[c][e] - m1 - v[c][e] * m2);
                store_chunk<XT, VE>(dx + at, o);
            }
        }
    }
    if (gr.dw == nullptr) return;
    float* pw = chunks > 1 ? gr.part + static_cast<int64_t>(blockIdx.x) * 2 * a.D : gr.dw + static_cast<int64_t>(sample) * gr.stride;
    float* pb = chunks > 1 ? pw + a.D : gr.db + static_cast<int64_t>(sample) * gr.stride;
    // the groups' sums, one group after the other
    if constexpr (kGroups > 1) {
        for (int k = 0; k < kGroups; ++k) {
            __syncthreads();
            if (group != k) continue;
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int at = first + c * kStep;
                if (at >= a.D) continue;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    if (k > 0) {
                        dw[c][e] += cols[at + e];
                        db[c][e] += cols[a.D + at + e];
                    }
                    if (k < kGroups - 1) {
                        cols[at + e] = dw[c][e];
                        cols[a.D + at + e] = db[c][e];
                    }
                }
            }
        }
        if (group != kGroups - 1) return;
    }
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int at = first + c * kStep;
        if (at >= a.D) continue;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            pw[at + e] = dw[c][e];
            pb[at + e] = db[c][e];
        }
    }
}

// dw, db [sample] = the partial rows of its chunks, added: 64 columns x 16 threads per workgroup, each thread every 16th chunk.
constexpr int kJoinRows = 16;
__global__ __launch_bounds__(64 * kJoinRows) void norm_join_kernel(NormGrad gr, int32_t D) {
    __shared__ float red[kJoinRows][64];
    const int col = blockIdx.x * 64 + threadIdx.x % 64, k = threadIdx.x / 64, which = blockIdx.y;
    const int64_t sample = blockIdx.z;
    float s = 0.f;
    if (col < D)
        for (int c = k; c < gr.chunks; c += kJoinRows) s += gr.part[((sample * gr.chunks + c) * 2 + which) * D + col];
    red[k][threadIdx.x % 64] = s;
    __syncthreads();
    if (k != 0 || col >= D) return;
#pragma unroll
    for (int j = 1; j < kJoinRows; ++j) s += red[j][threadIdx.x];
    (which == 0 ? gr.dw : gr.db)[sample * gr.stride + col] = s;
}

__global__ __launch_bounds__(kThreads) void norm_zero_kernel(NormGrad gr, int32_t D) {
    const int col = blockIdx.x * kThreads + threadIdx.x;
    if (col < D) gr.dw[col] = gr.db[col] = 0.f;
}

// Values per lane: the smallest row layout that holds D.  A lane holds up to 32 values in the backward pass (x, dy and two column sums
// of each are 128 registers), so wider rows take more wavefronts.
struct Layout {
    int ve, nv, wpr;
};
Layout layout_of(int32_t D, bool vec) {
    const int per_wave = (D + 63) / 64;
    if (vec) {
        const int n = (D / 4 + 63) / 64;                              // 16-byte chunks per lane of one wavefront
        if (n <= 1) return {4, 1, 1};
        if (n <= 2) return {4, 2, 1};
        if (n <= 5) return {4, 5, 1};
        if (n <= 10) return {4, 5, 2};
        if (n <= 20) return {4, 5, 4};
        if (n <= 32) return {4, 8, 4};
        return {4, 8, 8};
    }
    if (per_wave <= 8) return {1, 8, 1};
    if (per_wave <= 32) return {1, 16, 2};
    if (per_wave <= 64) return {1, 16, 4};
    if (per_wave <= 128) return {1, 16, 8};
    return {1, 16, 16};
}
constexpr int kMaxWidth = 64 * 16 * 16;
constexpr int kMaxBlocks = 1 << 22;                                    // grids of less than 2^32 threads

#define FREE_NORM_LAYOUTS(CASE) \
    CASE(4, 1, 1) CASE(4, 2, 1) CASE(4, 5, 1) CASE(4, 5, 2) CASE(4, 5, 4) CASE(4, 8, 4) CASE(4, 8, 8) \
    CASE(1, 8, 1) CASE(1, 16, 2) CASE(1, 16, 4) CASE(1, 16, 8) CASE(1, 16, 16)

template <typename XT, typename OT>
int32_t forward_of(const NormArgs& a, const Layout& l, hipStream_t s) {
    const int groups = l.wpr > 4 ? 1 : 4 / l.wpr, threads = l.wpr > 4 ? l.wpr * 64 : kThreads;
    const int blocks = static_cast<int>(std::min<int64_t>((static_cast<int64_t>(a.M) + groups - 1) / groups, kMaxBlocks));
#define FREE_CASE(VE, NV, WPR)                                                                                              \
    if (l.ve == VE && l.nv == NV && l.wpr == WPR) {                                                                         \
        hipLaunchKernelGGL((norm_forward_kernel<XT, OT, VE, NV, WPR>), dim3(blocks), dim3(threads), 0, s, a);               \
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;                                                                        \
    }
    FREE_NORM_LAYOUTS(FREE_CASE)
#undef FREE_CASE
    return FREE_ERR_SHAPE;
}

template <typename XT, typename OT>
int32_t backward_of(const NormArgs& a, const NormGrad& gr, int samples, const Layout& l, hipStream_t s) {
    const int threads = l.wpr > 4 ? l.wpr * 64 : kThreads;
    const size_t lds = l.wpr >= 4 || gr.dw == nullptr ? 0 : static_cast<size_t>(2) * a.D * sizeof(float);
#define FREE_CASE(VE, NV, WPR)                                                                                              \
    if (l.ve == VE && l.nv == NV && l.wpr == WPR) {                                                                         \
        hipLaunchKernelGGL((norm_backward_kernel<XT, OT, VE, NV, WPR>), dim3(samples * gr.chunks), dim3(threads), lds, s, a, gr, \
                           gr.chunks);                                                                                      \
        return launch_ok() ? FREE_OK : FREE_ERR_HIP;                                                                        \
    }
    FREE_NORM_LAYOUTS(FREE_CASE)
#undef FREE_CASE
    return FREE_ERR_SHAPE;
}

bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// whether rows can be read and written four values at a time
bool vector_ok(const void* x, int xb, const void* o, int ob, const float* w, const float* b, int32_t stride, int32_t D) {
    return D % 4 == 0 && stride % 4 == 0 && aligned(x, 4 * xb) && aligned(o, 4 * ob) && aligned(w, 16) && aligned(b, 16);
}

// Workgroups per sample in the backward pass.  Each writes a partial row of the weight's gradient and adds to what the second launch
// reads, so no more than keep the chip busy, and none for fewer than eight rows of a group.
int chunks_of(int32_t M, int32_t D, int32_t rows_per_sample) {
    const int64_t samples = (static_cast<int64_t>(M) + rows_per_sample - 1) / rows_per_sample;
    const int groups = std::max(1, 4 / layout_of(D, D % 4 == 0).wpr);
    const int64_t rows = std::min<int64_t>(M, rows_per_sample);
    const int64_t most = (rows + 8 * groups - 1) / (8 * groups);
    const int64_t want = (1024 + samples - 1) / samples;
    return static_cast<int>(std::max<int64_t>(1, std::min(most, want)));
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
    const int xb = x_dtype == FREE_BF16 ? 2 : 4, ob = dtype == FREE_BF16 ? 2 : 4;
    const Layout l = layout_of(D, vector_ok(x, xb, out, ob, weight, bias, stride, D));
    if (xb == 4) return ob == 4 ? forward_of<float, float>(a, l, s) : forward_of<float, bf16_t>(a, l, s);
    return ob == 4 ? forward_of<bf16_t, float>(a, l, s) : forward_of<bf16_t, bf16_t>(a, l, s);
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
    const int xb = x_dtype == FREE_BF16 ? 2 : 4, ob = dtype == FREE_BF16 ? 2 : 4;
    const bool vec = vector_ok(x, xb, dout, ob, weight, nullptr, weight ? stride : 0, D) && aligned(dx, 4 * xb);
    const Layout l = layout_of(D, vec);
    int32_t st;
    if (xb == 4) st = ob == 4 ? backward_of<float, float>(a, gr, samples, l, s) : backward_of<float, bf16_t>(a, gr, samples, l, s);
    else st = ob == 4 ? backward_of<bf16_t, float>(a, gr, samples, l, s) : backward_of<bf16_t, bf16_t>(a, gr, samples, l, s);
    if (st != FREE_OK || gr.chunks == 1 || dweight == nullptr) return st;
    hipLaunchKernelGGL(norm_join_kernel, dim3((D + 63) / 64, 2, samples), dim3(64 * kJoinRows), 0, s, gr, D);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

}  // namespace freemi
