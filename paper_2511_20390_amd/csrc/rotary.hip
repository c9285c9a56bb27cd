// Rotary positions over several axes.  A head's values are cut into one section per axis (time, row, column, ...) and a rest; pair i of
// axis a's section of d_a values is turned by the angle pos_a theta^(-2 i / d_a):
//     (a, b) -> (a cos - b sin, a sin + b cos),
// the inverse (the gradient's way back) by the opposite angle; the rest is copied.
//
// Angles are kept in turns, as 64-bit fixed point: the frequency is F = round(2^64 theta^(-2 i / d) / 2 pi), at most 2^64 / 2 pi, and
// pos F modulo 2^64 is the angle modulo one turn, exactly but for F's own error, the rounding's and that of the product of factors it comes
// from (against 60 digits, theta from 1 to 1e9 and up to 256 values: 8 units at most).  So positions up to 2^31 are off by less than 2^-29
// turns, where an fp32 product of position and frequency is off by a turn from 2^24 on.  Of it the leading 32 bits go to sincospi, rounded
// to an fp32 number: up to 2^-26 turns, as for any fp32 angle of up to half a turn.
//
// Bound by HBM (every value read and written once).  A thread holds V pairs of a token and computes their sines and cosines once for
// up to kHeads heads, whose loads are all in flight before the first is turned.  32760 tokens of 48 heads of 128 in bf16: 154 us, 5.2 TB/s
// read and written (a copy of 1 GiB: 5.1); fp32, 15640 tokens of 24 heads of 64, halves of the sections 24 values apart, 37.5 us, 5.1 TB/s;
// 256 tokens of 32 heads of 72, 4.6 us, of which an empty launch takes half.
#include <algorithm>
#include <cmath>

#include "free_internal.h"

namespace freemi {

namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 4;                    // heads per thread
constexpr int kMaxPairs = 128;               // of a head

struct RopeTable {
    uint64_t turn[kMaxPairs];                // F of pair p, 0: not turned
    uint8_t axis[kMaxPairs];
    uint8_t first[kMaxPairs];                // where the pair's values stand in the head
    uint8_t second[kMaxPairs];
};

struct RopeArgs {
    const void* x;
    void* out;
    const int32_t* pos;
    int64_t x_stride, out_stride;
    int32_t rows, pos_rows, axes, heads, dh;
    int32_t units, slots;                    // units of V pairs per head; threads that share the heads of a token
    int32_t inverse;
};

template <typename T, int N>
__device__ __forceinline__ void load_run(const T* p, float* v) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float4 f = *reinterpret_cast<const float4*>(p + i);
                v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
            }
        } else if constexpr (N == 2) {
            const float2 f = *reinterpret_cast<const float2*>(p);
            v[0] = f.x; v[1] = f.y;
        } else {
            v[0] = p[0];
        }
    } else if constexpr (N == 1) {
        v[0] = load_f(p);
    } else {
        uint32_t u[N / 2];
        if constexpr (N == 8) {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            u[0] = q.x; u[1] = q.y; u[2] = q.z; u[3] = q.w;
        } else if constexpr (N == 4) {
            const uint2 q = *reinterpret_cast<const uint2*>(p);
            u[0] = q.x; u[1] = q.y;
        } else {
            u[0] = *reinterpret_cast<const uint32_t*>(p);
        }
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}

template <typename T, int N>
__device__ __forceinline__ void store_run(T* p, const float* v) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else if constexpr (N == 2) {
            *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
        } else {
            p[0] = v[0];
        }
    } else if constexpr (N == 1) {
        store_f(p, v[0]);
    } else if constexpr (N == 8) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16_pair(v[0], v[1]), pack_bf16_pair(v[2], v[3]),
                                                  pack_bf16_pair(v[4], v[5]), pack_bf16_pair(v[6], v[7]));
    } else if constexpr (N == 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16_pair(v[0], v[1]), pack_bf16_pair(v[2], v[3]));
    } else {
        *reinterpret_cast<uint32_t*>(p) = pack_bf16_pair(v[0], v[1]);
    }
}

// kAdjacent: the two values of a pair stand next to each other and a unit is 2 V values in a row; otherwise its first and its second
// values are two runs of V.
template <typename T, int V, bool kAdjacent>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, RopeTable tab) {
    const int per_row = a.units * a.slots;
    const uint64_t g0 = static_cast<uint64_t>(blockIdx.x) * kThreads;
    const int64_t row0 = static_cast<int64_t>(g0 / per_row);
    const int t = static_cast<int>(g0 - static_cast<uint64_t>(row0) * per_row) + threadIdx.x;
    const int64_t row = row0 + t / per_row;
    if (row >= a.rows) return;
    const int in_row = t % per_row;
    const int unit = in_row % a.units, slot = in_row / a.units;
    const int p0 = unit * V;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    T* out = static_cast<T*>(a.out) + row * a.out_stride;
    const int o1 = tab.first[p0], o2 = kAdjacent ? 0 : tab.second[p0];
    float v[kHeads][2 * V];
#pragma unroll
    for (int j = 0; j < kHeads; ++j) {
        const int h = slot + j * a.slots;
        if (h >= a.heads) continue;
        const T* src = x + static_cast<int64_t>(h) * a.dh;
        if constexpr (kAdjacent) {
            load_run<T, 2 * V>(src + o1, v[j]);
        } else {
            load_run<T, V>(src + o1, v[j]);
            load_run<T, V>(src + o2, v[j] + V);
        }
    }
    const int32_t* pos = a.pos + (row % a.pos_rows) * a.axes;
    float c[V], s[V];
    bool turned[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint64_t turn = tab.turn[p0 + i];
        turned[i] = turn != 0;
        const uint64_t angle = static_cast<uint64_t>(static_cast<int64_t>(pos[tab.axis[p0 + i]])) * turn;
        sincospif(static_cast<float>(static_cast<int32_t>(angle >> 32)) * 0x1p-31f, &s[i], &c[i]);
        if (a.inverse) s[i] = -s[i];
    }
#pragma unroll
    for (int j = 0; j < kHeads; ++j) {
        const int h = slot + j * a.slots;
        if (h >= a.heads) continue;
        float o[2 * V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            constexpr int kFirst = kAdjacent ? 2 : 1;
            const int i1 = kFirst * i, i2 = kAdjacent ? i1 + 1 : i + V;
            const float p = v[j][i1], q = v[j][i2];
            o[i1] = turned[i] ? p * c[i] - q * s[i] : p;
            o[i2] = turned[i] ? p * s[i] + q * c[i] : q;
        }
        T* dst = out + static_cast<int64_t>(h) * a.dh;
        if constexpr (kAdjacent) {
            store_run<T, 2 * V>(dst + o1, o);
        } else {
            store_run<T, V>(dst + o1, o);
            store_run<T, V>(dst + o2, o + V);
        }
    }
}

template <typename T, int V, bool kAdjacent>
int32_t launch_of(RopeArgs a, const RopeTable& tab, hipStream_t s) {
    a.units = a.dh / 2 / V;
    a.slots = a.heads / kHeads + (a.heads % kHeads != 0);
    const int64_t per_row = static_cast<int64_t>(a.units) * a.slots;
    if (per_row > (1 << 30)) return FREE_ERR_LIMIT;
    const int64_t blocks = (a.rows * per_row + kThreads - 1) / kThreads;
    if (blocks > (1 << 24) - 1) return FREE_ERR_LIMIT;             // a grid has less than 2^32 threads
    hipLaunchKernelGGL((rope_kernel<T, V, kAdjacent>), dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, s, a, tab);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <typename T>
int32_t launch_type(const RopeArgs& a, const RopeTable& tab, int adjacent, int width, hipStream_t s) {
    if (adjacent) return width >= 4 ? launch_of<T, 4, true>(a, tab, s) : width == 2 ? launch_of<T, 2, true>(a, tab, s) : launch_of<T, 1, true>(a, tab, s);
    return width >= 4 ? launch_of<T, 4, false>(a, tab, s) : width == 2 ? launch_of<T, 2, false>(a, tab, s) : launch_of<T, 1, false>(a, tab, s);
}

}  // namespace

bool rope_covers(int32_t dh, int32_t axes, const int32_t* dims) {
    if (dh < 2 || dh % 2 != 0 || dh > 2 * kMaxPairs || axes < 1 || axes > 4) return false;
    int64_t sum = 0;
    for (int a = 0; a < axes; ++a) {
        if (dims[a] < 0 || dims[a] % 2 != 0) return false;
        sum += dims[a];
    }
    return sum <= dh;
}

int32_t launch_rope(const void* x, int64_t x_stride, const int32_t* pos, int32_t pos_rows, int32_t rows, int32_t heads, int32_t dh,
                    int32_t axes, const int32_t* dims, double theta, bool adjacent, bool inverse, int32_t dtype, void* out,
                    int64_t out_stride, hipStream_t s) {
    RopeTable tab;
    int p = 0, at = 0, run = dh;                                    // run: what the lengths of all runs are multiples of
    const auto gcd = [](int u, int v) { while (v) { const int w = u % v; u = v; v = w; } return u; };
    for (int a = 0; a <= axes; ++a) {                               // the rest last, as a section that is not turned
        const int d = a < axes ? dims[a] : dh - at;
        if (d == 0) continue;
        // in long double (64 significant bits) and one factor after the other: off by at most 128 of 2^-64
        const long double ratio = a < axes ? powl(static_cast<long double>(theta), -2.0L / d) : 0.0L;
        long double f = 0x1p64L / (2.0L * 3.141592653589793238462643383279502884L);
        for (int i = 0; i < d / 2; ++i, ++p, f *= ratio) {
            tab.turn[p] = a < axes ? static_cast<uint64_t>(f + 0.5L) : 0;
            tab.axis[p] = static_cast<uint8_t>(a < axes ? a : 0);
            tab.first[p] = static_cast<uint8_t>(at + (adjacent ? 2 * i : i));
            tab.second[p] = static_cast<uint8_t>(at + (adjacent ? 2 * i + 1 : i + d / 2));
        }
        if (!adjacent) run = gcd(run, d / 2);
        at += d;
    }
    // Pairs per thread: what divides the runs (pairs: the head) and keeps every access aligned to its own size
    const int es = dtype == FREE_BF16 ? 2 : 4;
    int width = 4;
    const auto fits = [&](int w) {
        const int values = adjacent ? 2 * w : w, bytes = std::min(16, values * es);
        const int64_t mask = bytes / es - 1;
        return (adjacent ? (dh / 2) % w : run % w) == 0 && !((x_stride | out_stride | dh) & mask) &&
               !((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) & (bytes - 1));
    };
    while (width > 1 && !fits(width)) width /= 2;
    const RopeArgs a{x, out, pos, x_stride, out_stride, rows, pos_rows, axes, heads, dh, 0, 0, inverse};
    // (a single pair of two neighbours may still be on an odd address: one value at a time then)
    const bool pair_at_once = !adjacent || width > 1 || fits(1);
    if (dtype == FREE_BF16) return launch_type<bf16_t>(a, tab, adjacent && pair_at_once, width, s);
    return launch_type<float>(a, tab, adjacent && pair_at_once, width, s);
}

}  // namespace freemi
