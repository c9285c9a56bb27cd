// The products of the gated feed-forward block and of its gradient in bf16 on the matrix cores, fp32 accumulation:
//   C[m, n] = sum over k of X(m, k) W(n, k)
// with X and W each either row-major (k next to each other) or K-major (rows of k, m or n next to each other):
//   [g | u] = x w_in^T                          rows, rows       h = act(g) u in the epilogue, and g, u kept
//   y  = h w_out^T                              rows, rows
//   dh = dy w_out                               rows, K-major    [dg | du] in the epilogue, from the kept g, u
//   dx = [dg | du] w_in                         rows, K-major
//   dw_in = [dg | du]^T x,  dw_out = dy^T h     K-major, K-major both in one launch
// so that no operand is transposed in memory first: a transposed copy of every factor of the gradient would move 6 M D + 14 M F + 12 D F
// bytes more.
//
// The K loop is that of gemm_pipe.hip (slices of 64 k in two LDS stages, loads global -> LDS, quarter steps).  What a K-major operand
// changes: a slice is 64 rows of 128 or 256 values, and the fragments come through ds_read_b64_tr_b16, which gives lane i of 16 the i-th
// column of a 4 x 16 block whose 4-value pieces the 16 lanes address.  A read of 32 lanes covers 4 k x 32 columns, four rows of 64
// bytes at the same place of rows 256 or 512 bytes long; 16-byte chunk (b4 b3 b2 b1 b0) of row k is kept at place (b4, b1, b2 ^ k1, b3 ^
// k0, b0) instead, which puts the 32 lanes on 64 different banks.
// The last slice of a K-major operand ends where the tensor does: the buffer descriptor gives zeros from there on.  Columns past the
// end of a row hold the next row's values and end in columns of C that are not written.  Of a row-major operand whose rows are not whole
// slices the fragments past the end are cleared in registers, in the last slice.  So widths need to be multiples of 8 only (16-byte
// rows); the hidden values' own tensors (h, dg, du and what is kept) have rows of H values, F rounded up to whole slices, zeros at the end, and an
// index of [dg | du] past H is one of w_in's rows past F: `fold`.
//
// Bound by the matrix pipe at the clock that the power limit leaves (1.7 GHz in the long launches; busy 0.65 to 0.78 of the cycles; LDS bank
// conflicts 1 % of its cycles).  Medians: 12288 x 1152 x 4608, gate and up 230 us (1137 TFLOP/s), down 117 (1119); 4096 x 4096 x 10240, gate and up with
// both kept 550 (1250), down 276 (1244), gated gradient 389 (883: 0.5 GB of g, u, dg and du besides), dx 605 (1135), both weights 809 (1274).
// The library's product of 8192^3 reaches 1325 on that card.
#include <algorithm>

#include "ffn_act.h"
#include "ffn_mfma.h"
#include "free_internal.h"
#include "gemm_dma.h"

namespace freemi {

namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));

struct Problem {
    const bf16_t *X, *W;
    int64_t ldx, ldw;            // values from row to row (K-major: from k to k)
    int32_t M, N, K;             // N: of the hidden values for the gated epilogues
    int32_t cols, fold, fold_to; // see FfnProduct
    int32_t tiles_m, tiles_n, group_m;
    int32_t split_slices;        // slices of a part of K (all, or those of one of several)
    bf16_t* out;                 // [M, cols], ldo values from row to row; gated gradient: dg, du `cols` further
    float* part;                 // sums over a part of K: [part][32 x 32 block][4][lane][4]
    float* gu;                   // kept [g | u], in blocks likewise
    int64_t ldo;
    int32_t act;
};

struct Launch {
    Problem p[2];
    int32_t first1;              // tiles (and parts of K) of p[0]
    int32_t total;               // of both
};

// Whether a workgroup does several tiles (LDS for the stages and for the epilogue, one workgroup per compute unit): launches of one product
// in whole sums, the others having few tiles, whose epilogue is short of neither registers (the gated gradient would spill 150) nor
// patience: the next tile's first slice is counted as arrived only once the epilogue's stores are, so that keeping g and u would cost
// more (12288 x 1152 x 4608 forward and gradient 1274 -> 1284 us) than it saves.  Forward of these rows 342 -> 334 us, 4096 x 4096 x 10240 777 -> 767.
constexpr bool ffn_rounds(int bm, int bn, bool xk, int epi) { return bm * bn > 128 * 128 && !xk && (epi == FFN_GATE || epi == FFN_STORE); }

template <int EPI>
constexpr bool kGated = EPI == FFN_GATE || EPI == FFN_GATE_KEEP;

// kRagged: rows of a row-major operand are not whole slices of K, or `cols` is more than N (an instance of its own: what it does in the
// last slice and in the epilogue costs products of few slices 3 %)
template <int BM, int BN, int WGM, int WGN, bool XK, bool WK, int EPI, bool kRagged>
__global__ __launch_bounds__(512) void ffn_product_kernel(Launch la) {
    constexpr int NW = 8;
    static_assert(WGM * WGN == NW && BN / WGN == 64, "eight wavefronts of 64 columns");
    constexpr int TM = BM / WGM / 32, TN = 2, MF = TM * TN;
    constexpr int LA = BM / 64, NL = (BM + BN) / 64, D2 = NL / 2, D3 = NL - D2;
    constexpr int kStageBytes = (BM + BN) * kRowBytes;
    constexpr int XU = XK ? 2 : 1, WU = WK ? 2 : 1;              // reads per fragment
    constexpr int RU = XU * TM + WU * TN;                        // reads of a k-step
    static_assert(!XK || BM == 128 || BM == 256, "rows of a K-major slice");
    static_assert(!WK || BN == 128 || BN == 256, "rows of a K-major slice");
    static_assert(!kGated<EPI> || !WK, "gate and up rows are interleaved row by row");
    extern __shared__ __attribute__((aligned(16))) char lds[];

    constexpr int kCols = kGated<EPI> ? BN / 2 : BN;             // columns of C per tile
    // A tile that has its compute unit to itself is one of several that a workgroup does: the next one's first two slices are requested
    // before the epilogue, which has its own piece of LDS.
    constexpr bool kRounds = ffn_rounds(BM, BN, XK, EPI);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int kHalfN = WGN / 2;
    const int wm = (wave & 3) / kHalfN, wn = (wave >> 2) * kHalfN + (wave & 3) % kHalfN;
    const bool second = !kRounds && static_cast<int>(blockIdx.x) >= la.first1;
    const Problem& a = second ? la.p[1] : la.p[0];
    const int ldx2 = static_cast<int>(a.ldx) * 2, ldw2 = static_cast<int>(a.ldw) * 2;
    // the tile at work (its epilogue goes by copies)
    int m0, n0, split, kt0, nk;
    u32x4_t xsrd, wsrd;

    // ---- loads, blocks of 1 KB: w, w + 8, ... per wavefront.  Row-major: 8 rows of 64 k, chunks swizzled as in gemm_pipe.hip.  K-major:
    // 1024 / row bytes rows of k.
    const auto major_offset = [&](int row_bytes, int ld2) {
        const int per = 64 / (1024 / row_bytes);                 // lanes per row of k
        const int k = lane / per + (row_bytes == 512 ? 2 * (wave & 1) : 0), p = lane % per;
        const int c = (p & 0x11) | ((p >> 3 & 1) << 1) | ((p >> 2 & 1) ^ (k >> 1 & 1)) << 2 | ((p >> 1 & 1) ^ (k & 1)) << 3;
        return (lane / per) * ld2 + c * 16;
    };
    const auto minor_offset = [&](int ld2) { return (lane >> 3) * ld2 + (((lane & 7) ^ (((wave & 1) << 2) | (lane >> 4))) << 4); };
    constexpr int XB = XK ? 1024 / (BM * 2) : 8, WB = WK ? 1024 / (BN * 2) : 8;       // memory rows per block
    const uint32_t lds_base = lds_address(lds);
    // gated: tile row r holds a gate row of the hidden value n0 + 32 (r / 64) + r % 32 where r % 64 < 32, else the up row; wavefronts
    // 0 to 3 load the gate rows of a group of 64, 4 to 7 the up rows
    const int xoff = XK ? major_offset(BM * 2, ldx2) : minor_offset(ldx2);
    const int woff = WK ? major_offset(BN * 2, ldw2) : minor_offset(ldw2);
    const auto set_tile = [&](int id) {
        const int pid = second ? id - la.first1 : id;
        const int tiles = a.tiles_m * a.tiles_n;
        int tile_m, tile_n;
        split = pid / tiles;
        tile_coords(a.group_m, pid % tiles, a.tiles_m, a.tiles_n, &tile_m, &tile_n);
        m0 = tile_m * BM;
        n0 = tile_n * kCols;
        const int all_slices = (a.K + BK - 1) / BK;
        kt0 = split * a.split_slices;
        nk = (kt0 + a.split_slices < all_slices ? a.split_slices : all_slices - kt0);
        const RowRange w_rows = kGated<EPI> ? gated_rows(wave, a.N, n0) : RowRange{n0, a.N - n0};
        if constexpr (!XK) xsrd = make_rsrc(a.X + m0 * a.ldx, (a.M - m0) * a.ldx * 2);
        if constexpr (!WK) wsrd = make_rsrc(a.W + w_rows.first * a.ldw, w_rows.count * a.ldw * 2);
    };
    // descriptors of a slice of a K-major operand, from its first k on: the offsets inside stay small whatever K is
    const auto aim = [&](int kt) {
        const int64_t k = static_cast<int64_t>(kt) * BK;
        if constexpr (XK) xsrd = make_rsrc(a.X + k * a.ldx + m0, ((a.K - k) * a.ldx - m0) * 2);
        if constexpr (WK) {
            const bool folded = !XK && a.fold > 0 && k >= a.fold;         // (of two K-major operands it is X's rows that fold)
            const int64_t row = folded ? k - a.fold + a.fold_to : k;
            const int64_t end = XK || a.fold == 0 ? a.K : folded ? 2 * static_cast<int64_t>(a.fold_to) : a.fold_to;
            wsrd = make_rsrc(a.W + row * a.ldw + n0, ((end - row) * a.ldw - n0) * 2);
        }
    };
    const auto dma = [&](int kt, int stage, int i) {
        const uint32_t dst = lds_base + stage * kStageBytes + wave * 1024;
        if (i < LA) {
            dma_1k(dst + i * NW * 1024, xoff, xsrd, (wave + i * NW) * XB * ldx2 + (XK ? 0 : kt * kRowBytes));
        } else {
            const int j = i - LA;
            const int row = kGated<EPI> ? j * 32 : (wave + j * NW) * WB;
            dma_1k(dst + BM * kRowBytes + j * NW * 1024, woff, wsrd, row * ldw2 + (WK ? 0 : kt * kRowBytes));
        }
    };

    // ---- fragments of k-step ks
    const int l32 = lane & 31, lhi = lane >> 5;
    const int sw = (l32 >> 1) & 7;
    const int kq = (lane & 15) >> 2;                             // the row of k, of four, that this lane addresses
    const auto major_place = [&](int tile) {                     // of its 8 bytes, in a row of k: columns 32 tile + 16 (lane / 16 % 2) + 4 (lane % 4)
        const int t0 = tile & 1, t1 = tile >> 1 & 1, t2 = tile >> 2;
        const int p = (lane >> 1 & 1) | (t1 ^ (kq & 1)) << 1 | (t0 ^ (kq >> 1)) << 2 | (lane >> 4 & 1) << 3 | t2 << 4;
        return p * 16 + (lane & 1) * 8;
    };
    int xat[TM], wat[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
        xat[i] = XK ? (lhi * 8 + kq) * BM * 2 + major_place(wm * TM + i) : (wm * TM * 32 + l32 + i * 32) * kRowBytes;
#pragma unroll
    for (int j = 0; j < TN; ++j)
        wat[j] = BM * kRowBytes + (WK ? (lhi * 8 + kq) * BN * 2 + major_place(wn * TN + j) : (wn * TN * 32 + l32 + j * 32) * kRowBytes);
    u32x2_t f[4][TM + TN][2];
    const auto read_half = [&](const char* at) {
        return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)at));
    };
    const auto read = [&](int stage, int ks, int r) {            // r-th of the RU reads
        const char* base = lds + stage * kStageBytes;
        const int minor = (((ks << 1) | lhi) ^ sw) << 4;
        if (r < XU * TM) {
            const int i = r / XU;
            if constexpr (XK) {
                f[ks][i][r % 2] = read_half(base + xat[i] + (ks * 16 + (r % 2) * 4) * BM * 2);
            } else {
                const u32x4_t v = *reinterpret_cast<const u32x4_t*>(base + xat[i] + minor);
                f[ks][i][0] = u32x2_t{v[0], v[1]};
                f[ks][i][1] = u32x2_t{v[2], v[3]};
            }
        } else {
            const int q = r - XU * TM, j = q / WU;
            if constexpr (WK) {
                f[ks][TM + j][q % 2] = read_half(base + wat[j] + (ks * 16 + (q % 2) * 4) * BN * 2);
            } else {
                const u32x4_t v = *reinterpret_cast<const u32x4_t*>(base + wat[j] + minor);
                f[ks][TM + j][0] = u32x2_t{v[0], v[1]};
                f[ks][TM + j][1] = u32x2_t{v[2], v[3]};
            }
        }
    };
    f32x16_t acc[TM][TN];
    const auto frag = [&](int ks, int r) {
        return __builtin_bit_cast(bf16x8_t, u32x4_t{f[ks][r][0][0], f[ks][r][0][1], f[ks][r][1][0], f[ks][r][1][1]});
    };
    const auto mma = [&](int ks, int t) {
        const int i = t / TN, j = t % TN;
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(ks, TM + j), frag(ks, i), acc[i][j], 0, 0, 0);
    };
    // a quarter: the products of k-step ks with nd loads and nr fragment reads spread between them
    const auto quarter = [&](auto ks_c, auto nd_c, auto nr_c, auto&& load, auto&& fetch) {
        constexpr int ks = decltype(ks_c)::value, nd = decltype(nd_c)::value, nr = decltype(nr_c)::value;
#pragma unroll
        for (int t = 0; t < MF; ++t) {
#pragma unroll
            for (int d = t * nd / MF; d < (t + 1) * nd / MF; ++d) load(d);
#pragma unroll
            for (int r = t * nr / MF; r < (t + 1) * nr / MF; ++r) fetch(r);
            mma(ks, t);
            if constexpr (nd > 0) {
                if ((t + 1) * nd / MF != t * nd / MF) __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (nd == 0) {
#pragma unroll
            for (int t = 0; t < MF; ++t) {
                __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                if ((t + 1) * nr / MF != t * nr / MF) __builtin_amdgcn_sched_group_barrier(kDsRd, (nr + MF - 1) / MF, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // the last slice of K: fragments of row-major operands past the end of a row
    const auto clear = [&](int kt, int ks) {
        if constexpr (kRagged) {
            if ((a.K - (kt0 + kt) * BK) >= BK) return;
            const bool ok = ks * 16 + lhi * 8 < a.K - (kt0 + kt) * BK;
#pragma unroll
            for (int r = XK ? TM : 0; r < (WK ? TM : TM + TN); ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e) f[ks][r][h][e] = ok ? f[ks][r][h][e] : 0u;
        }
    };
    const auto slice = [&](int kt, auto on, auto more1, auto more2) {   // slices kt + 1, kt + 2 exist; kt counts from this part's first
        constexpr bool kOn = decltype(on)::value, m1 = decltype(more1)::value, m2 = decltype(more2)::value;
        constexpr int nd2 = m2 ? D2 : 0, nd3 = m2 ? D3 : 0;
        const int s = kt & 1, o = s ^ 1;
        if constexpr (m2) aim(kt0 + kt + 2);
        const auto load2 = [&](int d) { dma(kt0 + kt + 2, s, d); };
        const auto load3 = [&](int d) { dma(kt0 + kt + 2, s, D2 + d); };
        if constexpr (kOn) {
            const auto none = [](int) {};
            using std::integral_constant;
            if constexpr (!m1) clear(kt, 0);
            quarter(integral_constant<int, 0>{}, integral_constant<int, 0>{}, integral_constant<int, 2 * RU>{}, none,
                    [&](int r) { read(s, 1 + r / RU, r % RU); });
            if constexpr (!m1) clear(kt, 1);
            quarter(integral_constant<int, 1>{}, integral_constant<int, 0>{}, integral_constant<int, RU>{}, none,
                    [&](int r) { read(s, 3, r); });
            if constexpr (m2) wait_lds_barrier();
            if constexpr (!m1) clear(kt, 2);
            quarter(integral_constant<int, 2>{}, integral_constant<int, nd2>{}, integral_constant<int, 0>{}, load2, none);
            if constexpr (m1) wait_vm_barrier<nd2>();
            if constexpr (!m1) clear(kt, 3);
            quarter(integral_constant<int, 3>{}, integral_constant<int, nd3>{}, integral_constant<int, m1 ? RU : 0>{}, load3,
                    [&](int r) { read(o, 0, r); });
        } else {
            if constexpr (m2) wait_lds_barrier();
#pragma unroll
            for (int d = 0; d < nd2; ++d) load2(d);
            if constexpr (m1) wait_vm_barrier<nd2>();
#pragma unroll
            for (int d = 0; d < nd3; ++d) load3(d);
        }
    };
    const std::true_type yes{};
    const std::false_type no{};

    const auto first_slices = [&]() {
        aim(kt0);
#pragma unroll
        for (int i = 0; i < NL; ++i) dma(kt0, 0, i);
        if (nk > 1) {
            aim(kt0 + 1);
#pragma unroll
            for (int i = 0; i < NL; ++i) dma(kt0 + 1, 1, i);
        }
    };
    const auto k_loop = [&](auto on) {
        if constexpr (decltype(on)::value) {
#pragma unroll
            for (int r = 0; r < RU; ++r) read(0, 0, r);
            __builtin_amdgcn_sched_barrier(0);
        }
        int kt = 0;
        for (; kt + 2 < nk; ++kt) slice(kt, on, yes, yes);
        if (kt + 1 < nk) {
            slice(kt, on, yes, no);
            ++kt;
        }
        slice(kt, on, no, no);
    };
    int id = blockIdx.x;
    set_tile(id);
    first_slices();
    for (;;) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        // the first slice has arrived (loads return in order, and the epilogue's stores behind them only make this wait longer)
        if (nk > 1) wait_vm_barrier<NL>();
        else wait_vm_barrier<0>();
        const int e_m0 = m0, e_split = split, e_col = n0 + wn * (kGated<EPI> ? 32 : 64);       // first row; this wavefront's first column of C
        const bool mine = e_col < a.cols && e_m0 + wm * TM * 32 < a.M;
        if (mine) k_loop(yes);
        else k_loop(no);
        wait_lds_barrier();
        id += gridDim.x;
        const bool more = kRounds && id < la.total;
        if (more) {
            set_tile(id);
            first_slices();
        }

        // ---- epilogue: register e of acc[i][j] in lane l is row 32 i + l % 32, column 32 j + 8 (e / 4) + 4 (l / 32) + e % 4 of the
        // wavefront's part.  bf16 goes through a private piece of LDS, so that whole rows are written.
        if (mine) {
            constexpr int OC = kGated<EPI> ? 1 : TN;                     // 32-column blocks of an output row
            constexpr int CH = OC * 4;
            char* const stage = lds + (kRounds ? 2 * kStageBytes : 0) + wave * 32 * CH * 16;
            static_assert(kRounds || NW * 32 * CH * 16 <= 2 * kStageBytes, "output staging must fit in the K-loop stages");
            const auto place = [&](int row, int chunk) { return stage + (row * CH + (chunk ^ (row & (CH - 1)))) * 16; };
            // 16 values of a 32 x 32 block -> row l32 of the staging rows, chunks 4 j ..
            const auto put = [&](int j, const auto& v) {
#pragma unroll
                for (int e8 = 0; e8 < 2; ++e8) {
                    const uint32_t lo0 = pack2(v[8 * e8], v[8 * e8 + 1]), lo1 = pack2(v[8 * e8 + 2], v[8 * e8 + 3]);
                    const uint32_t hi0 = pack2(v[8 * e8 + 4], v[8 * e8 + 5]), hi1 = pack2(v[8 * e8 + 6], v[8 * e8 + 7]);
                    const u32x2_t s0 = __builtin_amdgcn_permlane32_swap(lo0, hi0, false, false);
                    const u32x2_t s1 = __builtin_amdgcn_permlane32_swap(lo1, hi1, false, false);
                    *reinterpret_cast<u32x4_t*>(place(l32, 4 * j + 2 * e8 + lhi)) = u32x4_t{s0[0], s1[0], s0[1], s1[1]};
                }
            };
            const auto flush = [&](int i, bf16_t* out) {                 // the staged 32 rows -> out[row][e_col ..]
                int gm0 = e_m0 + (wm * TM + i) * 32, rows = a.M;
                if constexpr (XK) {                                      // (a fold is at a multiple of 64)
                    if (a.fold > 0) {
                        rows = gm0 < a.fold ? a.fold_to : 2 * a.fold_to;
                        gm0 = gm0 < a.fold ? gm0 : gm0 - a.fold + a.fold_to;
                    }
                }
#pragma unroll
                for (int q = 0; q < 32 * CH / 64; ++q) {
                    const int c = q * 64 + lane, row = c / CH, ch = c % CH;
                    const u32x4_t o = *reinterpret_cast<const u32x4_t*>(place(row, ch));
                    if (gm0 + row < rows && e_col + ch * 8 < a.cols)
                        *reinterpret_cast<u32x4_t*>(out + static_cast<int64_t>(gm0 + row) * a.ldo + e_col + ch * 8) = o;
                }
            };
            const int blocks_n = (a.cols + 31) / 32;
            if constexpr (EPI == FFN_PART) {
                const int64_t blocks = static_cast<int64_t>((a.M + 31) / 32) * blocks_n;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const int mb = e_m0 / 32 + wm * TM + i, nb = e_col / 32 + j;
                        if (mb * 32 >= a.M || nb >= blocks_n) continue;
                        float* p = a.part + (e_split * blocks + static_cast<int64_t>(mb) * blocks_n + nb) * 1024 + lane * 4;
#pragma unroll
                        for (int e4 = 0; e4 < 4; ++e4)
                            *reinterpret_cast<f32x4_t*>(p + e4 * 256) = f32x4_t{acc[i][j][4 * e4], acc[i][j][4 * e4 + 1], acc[i][j][4 * e4 + 2], acc[i][j][4 * e4 + 3]};
                    }
            } else if constexpr (kGated<EPI>) {
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    if constexpr (EPI == FFN_GATE_KEEP) {
                        const int mb = e_m0 / 32 + wm * TM + i;
                        if (mb * 32 < a.M) {
                            float* p = a.gu + (static_cast<int64_t>(mb) * 2 * blocks_n + e_col / 32) * 1024 + lane * 4;
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int e4 = 0; e4 < 4; ++e4)
                                    // (read again by the gradient only, out of memory: passing by the L2 leaves it to the products,
                                    // 12288 x 1152 x 4608 forward and gradient 1293 -> 1261 us)
                                    __builtin_nontemporal_store(
                                        f32x4_t{acc[i][j][4 * e4], acc[i][j][4 * e4 + 1], acc[i][j][4 * e4 + 2], acc[i][j][4 * e4 + 3]},
                                        reinterpret_cast<f32x4_t*>(p + static_cast<int64_t>(j) * blocks_n * 1024 + e4 * 256));
                        }
                    }
                    float h[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float f, df;
                        act_fast(acc[i][0][e], a.act, &f, &df);
                        h[e] = !kRagged || e_col + 8 * (e / 4) < a.N ? f * acc[i][1][e] : 0.f;
                    }
                    put(0, h);
                    flush(i, a.out);
                }
            } else if constexpr (EPI == FFN_GATE_GRAD) {
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const int mb = e_m0 / 32 + wm * TM + i;
                    float du[TN][16];
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const int nb = e_col / 32 + j;
                        f32x4_t g[4], u[4];
                        if (mb * 32 < a.M && nb < blocks_n) {
                            const float* p = a.gu + (static_cast<int64_t>(mb) * 2 * blocks_n + nb) * 1024 + lane * 4;
#pragma unroll
                            for (int e4 = 0; e4 < 4; ++e4) {
                                g[e4] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p + e4 * 256));
                                u[e4] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p + static_cast<int64_t>(blocks_n) * 1024 + e4 * 256));
                            }
                        }
                        float dg[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float f, df;
                            act_fast(g[e / 4][e % 4], a.act, &f, &df);
                            const bool there = !kRagged || e_col + 32 * j + 8 * (e / 4) < a.N;
                            du[j][e] = there ? acc[i][j][e] * f : 0.f;
                            dg[e] = there ? acc[i][j][e] * u[e / 4][e % 4] * df : 0.f;
                        }
                        put(j, dg);
                    }
                    flush(i, a.out);
#pragma unroll
                    for (int j = 0; j < TN; ++j) put(j, du[j]);
                    flush(i, a.out + a.cols);
                }
            } else {
#pragma unroll
                for (int i = 0; i < TM; ++i) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) put(j, acc[i][j]);
                    flush(i, a.out);
                }
            }
        }
        if (!more) break;
    }
}

// The parts of a product's sums over K, added in order, and the epilogue they were left without; a wavefront per 32 x 32 block of the
// result
template <typename T>
struct Join {
    const float* part;               // [splits][M / 32][part_n], and u's blocks `up` floats behind g's
    int64_t up;
    int32_t part_n;
    float* gu;
    T* out;
    int64_t ldo;
    int32_t M, N, cols, fold, fold_to, splits, act;       // N: hidden values for the gated kinds
};

template <FfnKind kKind, typename T>
__global__ __launch_bounds__(256) void ffn_join_kernel(Join<T> a) {
    constexpr bool kGate = kKind == FFN_GATE || kKind == FFN_GATE_KEEP, kGrad = kKind == FFN_GATE_GRAD;
    const int blocks_n = (a.cols + 31) / 32;
    const int64_t rows = (a.M + 31) / 32, block = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (block >= rows * blocks_n) return;
    const int lane = threadIdx.x & 63;
    const int mb = static_cast<int>(block / blocks_n), nb = static_cast<int>(block % blocks_n);
    constexpr int B = kGate ? 2 : 1;
    f32x4_t s[B][4];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const float* p = a.part + b * a.up + (static_cast<int64_t>(mb) * a.part_n + nb) * 1024 + lane * 4;
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) s[b][e4] = *reinterpret_cast<const f32x4_t*>(p + e4 * 256);
#pragma unroll 3
        for (int k = 1; k < a.splits; ++k)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) s[b][e4] += *reinterpret_cast<const f32x4_t*>(p + k * rows * a.part_n * 1024 + e4 * 256);
    }
    float* const gu = a.gu + (static_cast<int64_t>(mb) * 2 * blocks_n + nb) * 1024 + lane * 4;
    float* const up = gu + static_cast<int64_t>(blocks_n) * 1024;
    int m = mb * 32 + (lane & 31), m_end = a.M;
    if (kKind == FFN_ROWS && a.fold > 0) {
        m_end = m < a.fold ? a.fold_to : 2 * a.fold_to;
        m = m < a.fold ? m : m - a.fold + a.fold_to;
    }
    T* const out = a.out + m * a.ldo + nb * 32 + 4 * (lane >> 5);
    const auto store = [&](T* p, const f32x4_t& v) {
        if (m >= m_end) return;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_t*>(p) = v;
        else *reinterpret_cast<u32x2_t*>(p) = u32x2_t{pack2(v[0], v[1]), pack2(v[2], v[3])};
    };
    const auto activate = [&](float v, float* f, float* df) {
        if constexpr (sizeof(T) == 4) act_exact(v, a.act, f, df);
        else act_fast(v, a.act, f, df);
    };
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
        const bool there = nb * 32 + 8 * e4 < a.N;               // (N: a multiple of 8)
        if constexpr (kGate) {
            if constexpr (kKind == FFN_GATE_KEEP) {
                *reinterpret_cast<f32x4_t*>(gu + e4 * 256) = s[0][e4];
                *reinterpret_cast<f32x4_t*>(up + e4 * 256) = s[1][e4];
            }
            f32x4_t h;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float f, df;
                activate(s[0][e4][c], &f, &df);
                h[c] = there ? f * s[1][e4][c] : 0.f;
            }
            store(out + 8 * e4, h);
        } else if constexpr (kGrad) {
            const f32x4_t g = *reinterpret_cast<const f32x4_t*>(gu + e4 * 256), u = *reinterpret_cast<const f32x4_t*>(up + e4 * 256);
            f32x4_t dg, du;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float f, df;
                activate(g[c], &f, &df);
                du[c] = there ? s[0][e4][c] * f : 0.f;
                dg[c] = there ? s[0][e4][c] * u[c] * df : 0.f;
            }
            store(out + 8 * e4, dg);
            store(out + 8 * e4 + a.cols, du);
        } else if (there) {
            store(out + 8 * e4, s[0][e4]);
        }
    }
}

struct Tile {
    int bm, bn;
};

template <int BM, int BN, int WGM, int WGN, bool XK, bool WK, int EPI, bool kRagged>
int32_t launch_kernel(const Launch& la, int blocks, hipStream_t s) {
    auto kern = ffn_product_kernel<BM, BN, WGM, WGN, XK, WK, EPI, kRagged>;
    constexpr bool rounds = ffn_rounds(BM, BN, XK, EPI);
    const size_t lds = 2 * static_cast<size_t>(BM + BN) * kRowBytes + (rounds ? 8 * 32 * (kGated<EPI> ? 64 : 128) : 0);
    static LdsLimit limit;
    if (!limit.allow(reinterpret_cast<const void*>(kern), lds)) return FREE_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3(rounds ? std::min(blocks, device_cus()) : blocks), dim3(512), lds, s, la);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <bool XK, bool WK, int EPI, bool kRagged>
int32_t launch_size(const Tile& t, const Launch& la, int blocks, hipStream_t s) {
    if (t.bm == 256) return launch_kernel<256, 256, 2, 4, XK, WK, EPI, kRagged>(la, blocks, s);
    if (t.bn == 256) return launch_kernel<128, 256, 2, 4, XK, WK, EPI, kRagged>(la, blocks, s);
    return launch_kernel<128, 128, 4, 2, XK, WK, EPI, kRagged>(la, blocks, s);
}

template <bool XK, bool WK, int EPI>
int32_t launch_tile(const Tile& t, const Launch& la, int blocks, hipStream_t s) {
    // (K-major X, and rows by K-major but for the gated gradient, whose K is D: their K is the token rows, or whole slices of [dg | du])
    if constexpr (!XK && !(WK && EPI == FFN_STORE)) {
        const Problem& q = la.p[0];
        if (q.K % BK != 0 || q.cols != q.N) return launch_size<XK, WK, EPI, true>(t, la, blocks, s);
    }
    return launch_size<XK, WK, EPI, false>(t, la, blocks, s);
}

// What a launch takes: tile, and per product the parts that its sums over K are cut in
struct Plan {
    Tile tile;
    int splits[2];
};

int slices_of(int32_t K) { return std::max(1, (K + BK - 1) / BK); }
int parts_of(int slices, int splits) { return (slices + (slices + splits - 1) / splits - 1) / ((slices + splits - 1) / splits); }

template <typename T>
int64_t tiles_of(const FfnProduct<T>& p, const Tile& t, bool parts) {
    // (in parts gate and up are two products that meet in the join)
    const int per = p.gated() && !parts ? t.bn / 2 : t.bn;
    return static_cast<int64_t>((p.M + t.bm - 1) / t.bm) * ((p.cols() + per - 1) / per) * (p.gated() && parts ? 2 : 1);
}

template <typename T>
size_t part_bytes(const FfnProduct<T>& p, int splits) {
    return splits == 0 ? 0 : static_cast<size_t>(splits) * ((p.M + 31) / 32) * ((p.cols() + 31) / 32) * (p.gated() ? 2 : 1) * 4096;
}

// Times of a workgroup, us: a launch; a slice of 64 k with all compute units at work, and with nothing in the way but its loads' latency;
// the epilogue by what it does; slices of K-major operands against those of rows.  Fitted to 930 launches (70 to 12288 rows, widths 384 /
// 768 / 1152 / 2048 / 4096 with 1536 to 10240 hidden values, the three tiles, K in 1 to 24 parts, every kind of product): the plan chosen
// by them takes 1.0 % longer than the fastest one on average, 14 % at most.  The gated gradient has a factor of its own for K-major slices: its
// two resident 128 x 128 tiles are slower in long launches than products without its reads (4096 x 4096 x 10240, backward pass 1802 us, with 256 x 256
// tiles 1755; 44 sizes of 300 to 12288 rows: 0.2 % longer than the fastest tile on average).  What it decides, us: 12288 x 1152 x 4608, gate and up, 256 x
// 256 tiles 257, 128 x 128 322; 4096 x 1152 x 4608, the gated gradient, 256 x 256 100, 128 x 128 - a workgroup's epilogue beside another's
// products - 79; 128 x 1152 x 4608, the down product, K whole 46, in 12 parts 9 and 7 for the join.
struct TileTime {
    Tile tile;
    double launch, slice, alone, store, gate, grad, part, one_k_major, grad_k_major, both_k_major;
    int resident;                    // workgroups per compute unit
};
constexpr TileTime kTileTimes[] = {{{256, 256}, 0.46, 1.15, 0.58, 7.6, 8.8, 16.0, 10.5, 1.05, 1.05, 1.06, 1},
                                   {{128, 256}, 1.35, 0.89, 0.53, 4.8, 3.6, 9.5, 6.3, 0.82, 0.82, 0.83, 1},
                                   {{128, 128}, 3.25, 0.58, 0.49, 1.9, 6.7, 6.9, 4.0, 0.64, 0.72, 1.01, 2}};
constexpr int kUnits = 256;          // compute units; not asked of the device, as a workspace's size must not depend on which is current
constexpr int kMinPart = 4;          // slices of a part of K

Plan plan_of(const FfnProduct<bf16_t>* p, int n) {
    Plan best{{128, 128}, {1, 1}};
    double best_time = 0.0;
    const FfnKind kind = p[0].kind;
    for (const int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24}) {
        Plan plan{{0, 0}, {1, 1}};
        double join = 0.0;
        int slices = 0;
        for (int i = 0; i < n; ++i) {
            const int all = slices_of(p[i].K);
            plan.splits[i] = parts_of(all, std::min(splits, all));
            slices = std::max(slices, (all + plan.splits[i] - 1) / plan.splits[i]);
            if (splits > 1) join += 4.8 + 0.27 * plan.splits[i] + 0.18e-6 * static_cast<double>(part_bytes(p[i], plan.splits[i]));
        }
        if (splits > 1 && slices < kMinPart) break;
        for (const TileTime& t : kTileTimes) {
            int64_t work = 0;
            for (int i = 0; i < n; ++i) work += tiles_of(p[i], t.tile, splits > 1) * plan.splits[i];
            const double slice = t.slice * (kind == FFN_K_BY_K ? t.both_k_major : kind == FFN_GATE_GRAD ? t.grad_k_major : kind == FFN_ROWS_BY_K ? t.one_k_major : 1.0);
            const double end = splits > 1 ? t.part : p[0].gated() ? t.gate : kind == FFN_GATE_GRAD ? t.grad : t.store;
            const int64_t rounds = work / (kUnits * t.resident), rest = work % (kUnits * t.resident), share = (rest + kUnits - 1) / kUnits;
            double time = t.launch + join + rounds * (slices * std::max(t.alone, slice * t.resident) + end);
            if (rest > 0) time += slices * std::max(t.alone, slice * share) + end * share / t.resident;
            if (best_time == 0.0 || time < best_time) {
                best_time = time;
                best = plan;
                best.tile = t.tile;
            }
        }
    }
    return best;
}

template <FfnKind kKind, typename T>
int32_t launch_join_kernel(const FfnProduct<T>& p, const float* part, int splits, hipStream_t s) {
    const int64_t rows = (p.M + 31) / 32, cols = (p.cols() + 31) / 32, blocks = rows * cols;
    // g's and u's parts: fp32 those of one matrix [g | u], bf16 all of g's, then all of u's
    const bool one = sizeof(T) == 4 && p.gated();
    const Join<T> j{part,  one ? cols * 1024 : splits * blocks * 1024, static_cast<int32_t>(one ? 2 * cols : cols),
                    p.gu,  p.out, p.ldo, p.M, p.N, p.cols(), p.kind == FFN_K_BY_K ? p.fold : 0, p.fold_to, splits, p.act};
    hipLaunchKernelGGL((ffn_join_kernel<kKind, T>), dim3(static_cast<uint32_t>((blocks + 3) / 4)), dim3(256), 0, s, j);
    return launch_ok() ? FREE_OK : FREE_ERR_HIP;
}

template <typename T>
int32_t launch_join(const FfnProduct<T>& p, FfnKind kind, const float* part, int splits, hipStream_t s) {
    switch (kind) {
        case FFN_GATE: return launch_join_kernel<FFN_GATE>(p, part, splits, s);
        case FFN_GATE_KEEP: return launch_join_kernel<FFN_GATE_KEEP>(p, part, splits, s);
        case FFN_GATE_GRAD: return launch_join_kernel<FFN_GATE_GRAD>(p, part, splits, s);
        default: return launch_join_kernel<FFN_ROWS>(p, part, splits, s);
    }
}

// fp32: tile and parts by the times of gemm_f32.hip's tiles
struct PlanF32 {
    bool large;
    int splits;
};
constexpr int kSliceF32 = 32, kMinPartF32 = 8;

// a second launch whatever the parts: gate and up are in different tiles
bool join_anyway(FfnKind k) { return k == FFN_GATE || k == FFN_GATE_KEEP; }

PlanF32 plan_of(const FfnProduct<float>* p, int n) {
    PlanF32 best{false, 1};
    double best_time = 0.0;
    const int all = std::max(1, (p[0].K + kSliceF32 - 1) / kSliceF32);
    for (const int want : {1, 2, 3, 4, 6, 8, 12, 16}) {
        const int splits = parts_of(all, std::min(want, all)), slices = (all + splits - 1) / splits;
        if (want > 1 && slices < kMinPartF32) break;
        for (const bool large : {false, true}) {
            const int b = large ? 128 : 64;
            int64_t work = 0;
            double join = 0.0;
            for (int i = 0; i < n; ++i) {
                const int64_t cols = p[i].gated() ? 2 * static_cast<int64_t>(p[i].N) : p[i].N;        // (N: multiples of 64)
                work += static_cast<int64_t>((p[i].M + b - 1) / b) * ((cols + b - 1) / b) * splits;
                if (splits > 1) join += (join_anyway(p[i].kind) ? 0.0 : 4.8) + 0.27 * splits + 0.18e-6 * static_cast<double>(part_bytes(p[i], splits));
            }
            const double time = product_f32_time(large, work, slices) + join;
            if (best_time == 0.0 || time < best_time) {
                best_time = time;
                best = PlanF32{large, splits};
            }
        }
    }
    return best;
}

// parts in `part`, not in the place of the result (one part of a kept [g | u] is what is kept)
bool needs_room(const FfnProduct<float>& p, int splits) { return splits > 1 || p.kind == FFN_GATE; }

}  // namespace

size_t ffn_products_part_bytes(const FfnProduct<bf16_t>* p, int n) {
    const Plan plan = plan_of(p, n);
    if (plan.splits[0] == 1 && (n == 1 || plan.splits[1] == 1)) return 0;
    return part_bytes(p[0], plan.splits[0]) + (n == 2 ? part_bytes(p[1], plan.splits[1]) : 0);
}

size_t ffn_products_part_bytes(const FfnProduct<float>* p, int n) {
    const int splits = plan_of(p, n).splits;
    size_t bytes = 0;
    for (int i = 0; i < n; ++i)
        if (needs_room(p[i], splits)) bytes += part_bytes(p[i], splits);
    return bytes;
}

int32_t launch_ffn_products(const FfnProduct<float>* p, int n, float* part, hipStream_t s) {
    const PlanF32 plan = plan_of(p, n);
    if (p[0].kind == FFN_GATE_GRAD && plan.splits == 1) {
        const ProductF32 q{p[0].X, p[0].W, p[0].ldx, p[0].ldw, p[0].M, p[0].N, p[0].K, p[0].out};
        return launch_gated_grad_f32(plan.large, q, p[0].gu, p[0].act, s);
    }
    const bool blocks = plan.splits > 1 || join_anyway(p[0].kind);
    const bool x_by_k = p[0].kind == FFN_K_BY_K, w_by_k = x_by_k || p[0].kind == FFN_ROWS_BY_K || p[0].kind == FFN_GATE_GRAD;
    ProductF32 q[2];
    for (int i = 0; i < n; ++i) {
        q[i] = ProductF32{p[i].X, p[i].W, p[i].ldx, p[i].ldw, p[i].M, p[i].gated() ? 2 * p[i].N : p[i].N, p[i].K, p[i].out};
        if (!blocks) continue;
        q[i].out = p[i].gu;
        if (needs_room(p[i], plan.splits)) {
            q[i].out = part;
            part += part_bytes(p[i], plan.splits) / sizeof(float);
        }
    }
    int32_t st = launch_products_f32(x_by_k, w_by_k, plan.large, q, n, plan.splits, blocks, s);
    // (what is kept already is not written again)
    for (int i = 0; i < n && st == FREE_OK && blocks; ++i)
        st = launch_join(p[i], q[i].out == p[i].gu ? FFN_GATE : p[i].kind, q[i].out, plan.splits, s);
    return st;
}

int32_t launch_ffn_products(const FfnProduct<bf16_t>* p, int n, float* part, hipStream_t s) {
    const Plan plan = plan_of(p, n);
    const Tile t = plan.tile;
    const bool parts = plan.splits[0] > 1 || (n == 2 && plan.splits[1] > 1);
    Launch la{};
    int64_t blocks = 0;
    int count = 0;
    const auto add = [&](const FfnProduct<bf16_t>& from, int splits, const bf16_t* W) {
        Problem& q = la.p[count];
        q.X = from.X;
        q.W = W;
        q.ldx = from.ldx;
        q.ldw = from.ldw;
        q.M = from.M;
        q.N = from.N;
        q.K = from.K;
        q.cols = from.cols();
        q.fold = from.fold;
        q.fold_to = from.fold_to;
        const int cols = from.gated() && !parts ? t.bn / 2 : t.bn;
        q.tiles_m = (q.M + t.bm - 1) / t.bm;
        q.tiles_n = (q.cols + cols - 1) / cols;
        q.group_m = 8;
        q.split_slices = (slices_of(q.K) + splits - 1) / splits;
        q.out = from.out;
        q.ldo = from.ldo;
        q.gu = from.gu;
        q.act = from.act;
        if (parts) {
            q.part = part;
            part += static_cast<int64_t>(splits) * ((q.M + 31) / 32) * ((q.cols + 31) / 32) * 1024;
        }
        if (count == 1) la.first1 = static_cast<int32_t>(blocks);
        blocks += static_cast<int64_t>(q.tiles_m) * q.tiles_n * splits;
        ++count;
    };
    for (int i = 0; i < n; ++i) {
        add(p[i], plan.splits[i], p[i].W);
        if (p[i].gated() && parts) add(p[i], plan.splits[i], p[i].W + static_cast<int64_t>(p[i].N) * p[i].ldw);
    }
    if (count == 1) la.first1 = 0x7fffffff;
    if (blocks > (1 << 22)) return FREE_ERR_LIMIT;
    const int b = la.total = static_cast<int>(blocks);
    if (!parts) {
        switch (p[0].kind) {
            case FFN_GATE: return launch_tile<false, false, FFN_GATE>(t, la, b, s);
            case FFN_GATE_KEEP: return launch_tile<false, false, FFN_GATE_KEEP>(t, la, b, s);
            case FFN_GATE_GRAD: return launch_tile<false, true, FFN_GATE_GRAD>(t, la, b, s);
            case FFN_ROWS: return launch_tile<false, false, FFN_STORE>(t, la, b, s);
            case FFN_ROWS_BY_K: return launch_tile<false, true, FFN_STORE>(t, la, b, s);
            case FFN_K_BY_K: return launch_tile<true, true, FFN_STORE>(t, la, b, s);
            default: return FREE_ERR_RANGE;
        }
    }
    int32_t st;
    switch (p[0].kind) {
        case FFN_GATE:
        case FFN_GATE_KEEP:
        case FFN_ROWS: st = launch_tile<false, false, FFN_PART>(t, la, b, s); break;
        case FFN_GATE_GRAD:
        case FFN_ROWS_BY_K: st = launch_tile<false, true, FFN_PART>(t, la, b, s); break;
        case FFN_K_BY_K: st = launch_tile<true, true, FFN_PART>(t, la, b, s); break;
        default: return FREE_ERR_RANGE;
    }
    for (int i = 0; i < n && st == FREE_OK; ++i) {
        st = launch_join(p[i], p[i].kind, la.p[i].part, plan.splits[i], s);
    }
    return st;
}

}  // namespace freemi
