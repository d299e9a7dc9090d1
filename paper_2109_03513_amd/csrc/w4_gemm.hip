// Products of float or 8-bit activations with 4-bit weights (w4.hip's layout):
//   y[m][n] = s_m sum_g alpha[n][g] sum_{k in g} x[m][k] q[n][k].
//
// The activations are the first operand of the MFMAs (rows m), the weights the second (columns n):
// a lane holds outputs of one n, so a group's scale is one value per lane.  E2M1 values are exact in
// bf16 and fp16, E4M3 activations in bf16, so a group's products are exact and its sum fp32; the
// group's scale multiplies that sum in fp32, and the sums of the groups are added in fp32.
//
// By how many rows share the weights:
//  * k_w4_token (few rows): 16 outputs per workgroup, the reduction split over its waves; the weights
//    are read once from HBM and are all that costs: one row, 18432 outputs, K = 4096, G = 128 11.0 us
//    (3.5 TB/s of 39 MB; a copy reaches 5.1, and a launch alone is 2.5 us), 4096 outputs, K = 9216,
//    E4M3 rows 7.1 us.
//  * k_w4_tile: tiles of 32 to 128 rows, everything through a ring in LDS; with few tiles the
//    reduction is split over workgroups and k_w4_sum adds the parts.  Few rows are bound by the chain of
//    a step (64 fp16 rows of 9216 x 4096, G = 32: 16.9 us), many by power and by MFMA and VALU issue:
//    4096 E4M3 rows of 18432 x 4096, G = 128 490 to 514 us by card, 1.20 to 1.26 PFLOP/s, MFMA busy
//    56 % and VALU 61 % of cycles (bf16 rows 517 to 527); 1999 bf16 rows of 4096 x 9216, G = 64 146 us,
//    1.03 PFLOP/s, MFMA 43 %, VALU 44 %.
//    With bf16 rows of zeros the same products take 20 to 25 % less; tiles of 128 x 512 and 256 x 256, which
//    bring a quarter to a third fewer bytes per product into a CU, and an fma after every MFMA instead
//    of in groups all came out within 4 % or slower.
#include <math.h>

#include <type_traits>

#include "float_rows.h"

namespace esb {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Four pairs of 16-bit values as one fragment.
template <typename F, typename P>
__device__ __forceinline__ F join(P a, P b, P c, P d) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(F, u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                       __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)});
}

struct Bf16 {
    typedef bf16x8 frag;
    static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mma(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    // Eight E2M1 nibbles, lowest first.
    static __device__ __forceinline__ frag decode(uint32_t d) {
        return join<frag>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, 0),
                          __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, 2),
                          __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, 3));
    }
};
struct F16 {
    typedef f16x8 frag;
    static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mma(frag a, frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ frag decode(uint32_t d) {
        return join<frag>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 0),
                          __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 2),
                          __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 3));
    }
};

// Activations: `raw` is what one lane loads of eight elements, zeros past the row's end.
template <typename X> struct Act;
template <> struct Act<__bf16> {
    typedef Bf16 M;
    typedef bf16x8 raw;
    static __device__ __forceinline__ raw load(const __bf16* p, int n) { return load8(p, n); }
    static __device__ __forceinline__ bf16x8 frag(raw r) { return r; }
};
template <> struct Act<_Float16> {
    typedef F16 M;
    typedef f16x8 raw;
    static __device__ __forceinline__ raw load(const _Float16* p, int n) { return load8(p, n); }
    static __device__ __forceinline__ f16x8 frag(raw r) { return r; }
};
template <> struct Act<uint8_t> {
    typedef Bf16 M;
    typedef uint2 raw;
    static __device__ __forceinline__ raw load(const uint8_t* p, int n) {
        if (n >= 8) return ((const Loose<uint2, uint8_t>*)p)->v;
        uint32_t v[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) v[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
        return uint2{v[0], v[1]};
    }
    // E4M3 values are exact in bf16.
    static __device__ __forceinline__ bf16x8 frag(raw v) {
        return join<bf16x8>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.x, 1.0f, false),
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.x, 1.0f, true),
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.y, 1.0f, false),
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.y, 1.0f, true));
    }
};

__device__ __forceinline__ float scale_value(uint16_t s) { return __uint_as_float((uint32_t)s << 16); }

// Stores with the output type picked once: f(pointer of the type).
template <typename F>
__device__ __forceinline__ void with_y(const W4GemmParams& p, F f) {
    if (p.y_type == kBF16) f((__bf16*)p.y);
    else if (p.y_type == kF16) f((_Float16*)p.y);
    else f((float*)p.y);
}

// 16 outputs n x up to 16 rows m per workgroup, the column chunks dealt to its NW waves and their sums
// added in LDS in wave order.
template <typename X, int G, int NW, int U>
__global__ __launch_bounds__(64 * NW) void k_w4_token(W4GemmParams p) {
    typedef typename Act<X>::M M;
    __shared__ f32x4 red[NW][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, s = lane >> 4;
    const int nt = blockIdx.x >> 1, row = 16 * (blockIdx.x & 1) + r;
    if (32 * nt + 16 * (int)(blockIdx.x & 1) >= p.L.N) return;
    const bool live = r < p.M;
    const X* x = (const X*)p.x + (live ? r : 0) * p.ldx;
    const int h = s >> 1, e = s & 1;
    const uint8_t* w = p.w4 + (int64_t)nt * p.L.chunks * 1024 + 16 * (32 * h + row) + 8 * e;
    const uint16_t* sc = (const uint16_t*)(p.w4 + p.L.scale_offset) + (int64_t)nt * p.L.groups * 32 + row;
    f32x4 acc = {0, 0, 0, 0};
    constexpr int NG = G == 32 ? 2 : 1;
    // U chunks at a time, every load in flight before the first product
    auto go = [&](int k0, auto full) {
        constexpr int n = decltype(full)::value;
        uint2 q[n];
        uint16_t a[n][NG];
        typename Act<X>::raw raw[n][2];
#pragma unroll
        for (int u = 0; u < n; u++) {
            const int kc = k0 + u * NW;
            q[u] = *(const uint2*)(w + (int64_t)kc * 1024);
#pragma unroll
            for (int g = 0; g < NG; g++) a[u][g] = sc[(int64_t)(G == 128 ? kc >> 1 : NG * kc + g) * 32];
        }
#pragma unroll
        for (int u = 0; u < n; u++) {
            raw[u][0] = raw[u][1] = typename Act<X>::raw{};
            const int k = 64 * (k0 + u * NW) + 16 * h + 8 * e;
            if (live) {
                raw[u][0] = Act<X>::load(x + k, p.L.K - k);
                raw[u][1] = Act<X>::load(x + k + 32, p.L.K - k - 32);
            }
        }
#pragma unroll
        for (int u = 0; u < n; u++) {
            const f32x4 p0 = M::mma(Act<X>::frag(raw[u][0]), M::decode(q[u].x), f32x4{0, 0, 0, 0});
            const f32x4 p1 = M::mma(Act<X>::frag(raw[u][1]), M::decode(q[u].y), NG == 2 ? f32x4{0, 0, 0, 0} : p0);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (NG == 2) acc[i] = fmaf(scale_value(a[u][0]), p0[i], acc[i]);
                acc[i] = fmaf(scale_value(a[u][NG - 1]), p1[i], acc[i]);
            }
        }
    };
    int kc = wave;
    for (; kc + (U - 1) * NW < p.L.chunks; kc += U * NW) go(kc, std::integral_constant<int, U>{});
    for (; kc < p.L.chunks; kc += NW) go(kc, std::integral_constant<int, 1>{});
    red[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    for (int u = 1; u < NW; u++) acc += red[u][lane];
    const int n = 32 * nt + row;
    if (n >= p.L.N) return;
    with_y(p, [&](auto* y) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t m = 4 * s + i;
            if (m < p.M) y[m * p.ldy + n] = p.x_scale ? acc[i] * p.x_scale[m] : acc[i];
        }
    });
}

// Workgroup `id` of `total` to a tile: each XCD (every eighth id) gets a contiguous run.
__device__ __forceinline__ int xcd_run(int id, int total) {
    const int x = id & 7, q = total >> 3, rem = total & 7;
    return x * q + min(x, rem) + (id >> 3);
}

// Tiles of BM = 32 TM WM rows m x BN = 64 WN outputs n, a wave of the workgroup 32 TM x 64 of it.
// A step is 128 bytes of every row of the tile: 64 columns of 16-bit values (F8 == 0; E4M3 activations
// become bf16 on their way) or 128 columns of E4M3 (F8 == 1: fragments become bf16 when they are read,
// 64 columns at a time), and the weights and scales of these columns.  All of it lies in a ring of R stages in LDS, fetched R - 1 steps ahead by DMA, which holds
// no registers; activations that DMA cannot take (DMA == 0: rows that are not 16-byte aligned, or that
// need the conversion) go through registers one step ahead.
//
// 16-byte piece c of row i is at c ^ ((i / 2) % 8) of its row, so that the 16 rows which one quarter of
// a wave reads at a time lie in different banks.  One barrier per step.  A step's products go group by
// group and tile by tile: the MFMAs of one (tile, group) are issued, then the sums of an earlier one
// are scaled and added under them.
//
// KW parts of WM x WN waves, each with a ring of its own, take every KW-th step of the tile, and the first
// part adds their sums: a step's chain of barrier, LDS reads, decoding and dependent MFMAs is about
// 1000 cycles that only other waves can fill (32 x 256, 64 steps, one workgroup per CU: 28 us with
// one part, 21 with two, 17 with four; 64 bf16 rows of 9216 x 4096: 18.7 us in 32 x 256 tiles of two
// parts, 16.8 in 32 x 128 of four; 128 of 4096 x 4096: 17.5 there, 13.2 in 32 x 64 of eight).
//
// 8-bit rows take the bf16 MFMAs too.  Those on 8-bit operands, with 4-bit weights or with weights as
// E4M3, drop what lies 13 binades below the largest product of an instruction: of E4M3 times E2M1, whose
// products span 21, sums of 16 or 64 with both signs came out wrong by up to 95 times their value.
// The bf16 form gave the exact sum of every one (2^18 random sums, and two products that cancel beside
// a third).
__device__ __align__(16) const uint8_t kZeros[1024] = {0};

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

__device__ __forceinline__ void dma16(const void* g, uint8_t* wave_base) {
    __builtin_amdgcn_global_load_lds((global_void*)g, (lds_void*)wave_base, 16, 0, 0);
}
__device__ __forceinline__ void dma4(const void* g, uint8_t* wave_base) {
    __builtin_amdgcn_global_load_lds((global_void*)g, (lds_void*)wave_base, 4, 0, 0);
}
// s_waitcnt vmcnt(N), the other counters at their maxima.
template <int N>
__device__ __forceinline__ void vm_wait() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
// Barrier for LDS alone: DMAs stay in flight.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0), seen by the compiler's own tracking
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <typename X, int F8, int G, int TM, int WM, int WN, int KW, int R, int DMA>
__global__ __launch_bounds__(64 * WM * WN * KW, KW == 4 ? 4 : 2) void k_w4_tile(W4GemmParams p, int tiles_m, int tiles, int per_split) {
    typedef typename Act<X>::M M;
    typedef typename Act<X>::raw Raw;
    typedef typename M::frag Frag;
    constexpr int NW = WM * WN, BM = 32 * TM * WM;            // waves and rows of one part
    constexpr int BK = F8 ? 128 : 64, EP = F8 ? 16 : 8;       // columns of a step, of a piece
    constexpr int NC = F8 ? 2 : 1;                            // column chunks of a step
    constexpr int NG = F8 ? 128 / G : G == 32 ? 2 : 1;        // scales of a step
    constexpr int NX = BM / (8 * NW), NT = 2 * WN * NC / NW;  // DMAs of a wave: rows, weight tiles
    static_assert(NX * 8 * NW == BM && NT * NW == 2 * WN * NC, "whole DMAs per wave");
    constexpr int PER = (DMA ? NX : 0) + NT + 1;
    constexpr int XB = BM * 128, WB = 2 * WN * NC * 1024, STAGE = XB + WB + 256 * NW;
    constexpr int GM = 4;                                     // tiles of rows in a band
    constexpr int SLAB = 68;                                  // floats of a slab's row
    static_assert(NW * 32 * SLAB * 4 <= R * STAGE, "the slabs fit the ring");
    static_assert((KW - 1) * NW * TM * 8192 <= KW * R * STAGE, "the other parts' sums fit the rings");
    __shared__ __align__(16) uint8_t rings[KW * R * STAGE];

    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, h = lane >> 5;
    const int part_k = __builtin_amdgcn_readfirstlane(tid >> 6) / NW;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) % NW;
    const int wm = wave / WN, wn = wave % WN;
    uint8_t* ring = rings + part_k * (R * STAGE);
    // A run of tiles goes through bands of up to GM tiles of rows, n by n: the workgroups of an XCD that
    // run together then share few rows and few columns, and its L2 fetches each once.
    const int id = xcd_run(blockIdx.x, gridDim.x), z = id / tiles, t = id - z * tiles, tiles_n = tiles / tiles_m;
    const int band = t / (GM * tiles_n), in_band = t - band * GM * tiles_n, high = min(GM, tiles_m - band * GM);
    const int64_t m0 = (int64_t)(band * GM + in_band % high) * BM;
    const int nt0 = in_band / high * (2 * WN);
    const int K = p.L.K, chunks = p.L.chunks, steps = (chunks + NC - 1) / NC;
    const int first = z * per_split, end = min(first + per_split, steps);

    // Rows: DMA i of the wave serves rows 8 (wave + i NW) + lane / 8 and writes slot lane % 8 of each,
    // so it fetches piece (lane % 8) ^ (row / 2 % 8).  Through registers, the same rows and pieces.
    const X* xb = (const X*)p.x + m0 * p.ldx;
    int64_t xo[NX];
    int pc[NX];
#pragma unroll
    for (int i = 0; i < NX; i++) {
        const int64_t m = m0 + 8 * (wave + i * NW) + (lane >> 3);
        pc[i] = (lane & 7) ^ (((8 * (wave + i * NW) + (lane >> 3)) >> 1) & 7);
        xo[i] = ((m < p.M ? m : p.M - 1) - m0) * p.ldx + EP * pc[i];
    }
    // Weight tiles wave + i NW of the stage's [row tile][chunk]; rows of tiles past N read the last.
    const uint8_t* wp[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) {
        const int q = wave + i * NW;
        wp[i] = p.w4 + ((int64_t)min(nt0 + q / NC, p.L.tiles - 1) * chunks + q % NC) * 1024;
    }
    // The wave's own scales, [row tile j][group g of the step][32 rows], 16 lanes each.
    const int sj = (lane >> 4) / NG & 1, sg = (lane >> 4) % NG, snt = min(nt0 + 2 * wn, p.L.tiles - 1);
    const uint8_t* sp = p.w4 + p.L.scale_offset + (int64_t)snt * p.L.groups * 64;
    const uint32_t so = (sj && snt + 1 < p.L.tiles ? (uint32_t)p.L.groups * 64 : 0) + 4 * (lane & 15);

    // Every stage issues the same number of DMAs, also past the last step.  What differs between lanes fits
    // 32 bits (rows closer than 2^24 elements), so a whole step's addresses are scalar but for one sum.
    const int whole = p.ldx < 1 << 24 ? min(end, K / BK) : 0;
    auto fetch = [&](int s, uint8_t* slot) {
        if constexpr (DMA) {
            if (s < whole) {
                const char* base = (const char*)(xb + (int64_t)s * BK);
#pragma unroll
                for (int i = 0; i < NX; i++) dma16(base + (uint32_t)xo[i] * (uint32_t)sizeof(X), slot + 1024 * (wave + i * NW));
            } else {
#pragma unroll
                for (int i = 0; i < NX; i++)
                    dma16(s * BK + EP * pc[i] < K && s < end ? (const void*)(xb + xo[i] + s * BK) : (const void*)kZeros,
                          slot + 1024 * (wave + i * NW));
            }
        }
#pragma unroll
        for (int i = 0; i < NT; i++) {
            const bool in = s * NC + (wave + i * NW) % NC < chunks;
            dma16((in ? wp[i] + (int64_t)s * (NC * 1024) : kZeros) + (uint32_t)(16 * lane), slot + XB + 1024 * (wave + i * NW));
        }
        // steps past the end and groups past the last one get scales of 0: an infinite one of another
        // step would make NaN of their sums of 0
        const int gi = F8 || G < 128 ? NG * s + sg : s >> 1;
        dma4(s < end && gi < p.L.groups ? sp + ((uint32_t)gi * 64 + so) : kZeros, slot + XB + WB + 256 * wave);
    };
    Raw st[DMA ? 1 : NX][F8 ? 2 : 1];
    auto load = [&](int s) {
        const int k = s < end ? s * BK : K;
        if (k + BK <= K) {
#pragma unroll
            for (int i = 0; i < NX; i++)
#pragma unroll
                for (int u = 0; u < (F8 ? 2 : 1); u++) st[i][u] = Act<X>::load(xb + xo[i] + k + 8 * u, 8);
        } else {
#pragma unroll
            for (int i = 0; i < NX; i++)
#pragma unroll
                for (int u = 0; u < (F8 ? 2 : 1); u++)
                    st[i][u] = Act<X>::load(xb + xo[i] + k + 8 * u, K - k - EP * pc[i] - 8 * u);
        }
    };
    auto put = [&](uint8_t* slot) {
#pragma unroll
        for (int i = 0; i < NX; i++) {
            uint8_t* d = slot + 1024 * (wave + i * NW) + 16 * lane;
            if constexpr (F8) {
                *(Raw*)d = st[i][0];
                *(Raw*)(d + 8) = st[i][1];
            } else {
                *(typename M::frag*)d = Act<X>::frag(st[i][0]);
            }
        }
    };

    f32x16 acc[TM][2] = {};
    const uint32_t arow = (uint32_t)(wm * 32 * TM + r) * 128;
    const int swz = (r >> 1) & 7;
    constexpr int NF = 4, NGH = G == 32 ? 2 : 1;      // MFMAs and scales of a tile's 64 columns
    // two behind where the registers allow, so that no sum is waited for
    constexpr int U = TM * 2 * NGH, LAG = TM == 4 || (KW >= 4 && WN == 2 && !F8 && G == 32) ? 1 : 2;
    // 64 columns, the half-th of the step
    auto columns = [&](const uint8_t* slot, int half) {
        float a[2][NGH];
        Frag wf[2][NF], x[NF];
        uint4 raw[2];
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const i32x4 q = *(const i32x4*)(slot + XB + ((2 * wn + j) * NC + half) * 1024 + 16 * lane);
            wf[j][0] = M::decode(q[0]);
            wf[j][1] = M::decode(q[2]);
            wf[j][2] = M::decode(q[1]);
            wf[j][3] = M::decode(q[3]);
#pragma unroll
            for (int g = 0; g < NGH; g++)
                a[j][g] = scale_value(*(const uint16_t*)(slot + XB + WB + 256 * wave + 64 * (j * NG + (F8 ? half * (NG - 1) : g)) + 2 * r));
        }
        auto rows = [&](int i) {
            const uint8_t* base = slot + arow + i * 32 * 128;
            if constexpr (F8) {
#pragma unroll
                for (int c = 0; c < 2; c++) raw[c] = *(const uint4*)(base + 16 * ((4 * half + h + 2 * c) ^ swz));
            } else {
#pragma unroll
                for (int c = 0; c < NF; c++) x[c] = *(const Frag*)(base + 16 * ((2 * h + (c & 1) + 4 * (c >> 1)) ^ swz));
            }
        };
        rows(0);
        f32x16 part[LAG + 1];
#pragma unroll
        for (int u = 0; u < U + LAG; u++) {
            if (u < U) {
                const int j = u / NGH % 2, g = u % NGH;
                if constexpr (F8) {
                    if (u % (2 * NGH) == 0) {
#pragma unroll
                        for (int c = 0; c < NF; c++)
                            x[c] = Act<X>::frag(c & 1 ? uint2{raw[c / 2].z, raw[c / 2].w} : uint2{raw[c / 2].x, raw[c / 2].y});
                    }
                }
                f32x16 d = {};
#pragma unroll
                for (int c = NF / NGH * g; c < NF / NGH * (g + 1); c++) d = M::mma(x[c], wf[j][c], d);
                part[u % (LAG + 1)] = d;
                // the next rows, once the registers that they go to are free
                if ((F8 ? u : u + 1) % (2 * NGH) == 0 && u / (2 * NGH) + 1 < TM) rows(u / (2 * NGH) + 1);
            }
            if (u >= LAG) {
                const int v = u - LAG, i = v / (2 * NGH), j = v / NGH % 2, g = v % NGH;
#pragma unroll
                for (int q = 0; q < 16; q++) acc[i][j][q] = fmaf(a[j][g], part[v % (LAG + 1)][q], acc[i][j][q]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto step = [&](const uint8_t* slot) {
#pragma unroll
        for (int half = 0; half < NC; half++) columns(slot, half);
    };

    // step first + i KW + part_k in slot i % R; a part's steps past the end add zeros
    const int begin = first + part_k, turns = (end - first + KW - 1) / KW;
    if constexpr (!DMA) {
        load(begin);
        put(ring);
        load(begin + KW);
    }
#pragma unroll
    for (int q = 0; q < R - 1; q++) fetch(begin + q * KW, ring + q * STAGE);
    int cur = 0, last = R - 1;           // slots of this turn and of the one before it
    for (int i = 0; i < turns; i++) {
        const int s = begin + i * KW;
        vm_wait<(R - 2) * PER>();        // this wave's part of step s has landed
        lds_barrier();                   // all of it; every read of the last turn is done
        __builtin_amdgcn_sched_barrier(0);
        fetch(s + (R - 1) * KW, ring + last * STAGE);
        if constexpr (!DMA) {
            put(ring + (cur + 1 == R ? 0 : cur + 1) * STAGE);
            load(s + 2 * KW);
        }
        __builtin_amdgcn_sched_barrier(0);
        step(ring + cur * STAGE);
        last = cur;
        cur = cur + 1 == R ? 0 : cur + 1;
    }
    vm_wait<0>();                            // no DMA outlives its workgroup
    __syncthreads();
    if constexpr (KW > 1) {
        // the first part adds the sums of the others, in order
        f32x4* red = (f32x4*)rings + wave * (TM * 512) + lane;
        if (part_k > 0)
#pragma unroll
            for (int q = 0; q < TM * 8; q++) {
                const f32x16& v = acc[q / 8][q / 4 % 2];
                red[(part_k - 1) * (NW * TM * 512) + 64 * q] = f32x4{v[4 * (q % 4)], v[4 * (q % 4) + 1], v[4 * (q % 4) + 2], v[4 * (q % 4) + 3]};
            }
        __syncthreads();
        if (part_k == 0)
#pragma unroll
            for (int k = 0; k < KW - 1; k++)
#pragma unroll
                for (int q = 0; q < TM * 8; q++) {
                    const f32x4 o = red[k * (NW * TM * 512) + 64 * q];
#pragma unroll
                    for (int c = 0; c < 4; c++) acc[q / 8][q / 4 % 2][4 * (q % 4) + c] += o[c];
                }
        __syncthreads();
        if (part_k > 0) return;
    }

    // Outputs, 32 rows at a time through a slab of LDS of each wave's own: lanes hold columns, stores
    // want rows of 16-byte pieces.
    float* slab = (float*)(ring + wave * (32 * SLAB * 4));
    // f(row m, first column n, eight values): every lane, column n may lie past the last
    auto outputs = [&](auto f) {
#pragma unroll
        for (int i = 0; i < TM; i++) {
#pragma unroll
            for (int q = 0; q < 16; q++)
#pragma unroll
                for (int j = 0; j < 2; j++)
                    slab[(8 * (q >> 2) + 4 * h + (q & 3)) * SLAB + 32 * j + r] = acc[i][j][q];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int row = 8 * e + (lane >> 3);
                const f32x4 lo = *(const f32x4*)(slab + row * SLAB + 8 * (lane & 7));
                const f32x4 hi = *(const f32x4*)(slab + row * SLAB + 8 * (lane & 7) + 4);
                const int64_t m = m0 + wm * 32 * TM + 32 * i + row;
                if (m < p.M) f(m, 32 * (nt0 + 2 * wn) + 8 * (lane & 7), f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (p.part) {
        const int64_t np = 32 * (int64_t)p.L.tiles;
        outputs([&](int64_t m, int n, f32x8 v) {
            if (n < np) *(f32x8*)(p.part + ((int64_t)z * p.M + m) * np + n) = v;
        });
        return;
    }
    with_y(p, [&](auto* y) {
        typedef std::remove_reference_t<decltype(*y)> Y;
        outputs([&](int64_t m, int n, f32x8 v) {
            if (p.x_scale) v *= p.x_scale[m];
            if (n < p.L.N) store8(y + m * p.ldy + n, __builtin_convertvector(v, typename Vec8<Y>::type), p.L.N - n);
        });
    });
}

// Rows that DMA cannot take, once into aligned ones with whole 64-column pieces (zeros past K); E4M3 rows
// for the bf16 MFMAs (TO == 2) are converted.
template <typename X, int TO>
__global__ __launch_bounds__(256) void k_w4_align(W4GemmParams p, uint8_t* __restrict__ out, int pieces) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = i / pieces;
    if (m >= p.M) return;
    constexpr int EP = 16 / TO;
    const int k = EP * (int)(i - m * pieces);
    const X* x = (const X*)p.x + m * p.ldx + k;
    if constexpr (EP == 16) {
        const uint2 lo = Act<X>::load(x, p.L.K - k), hi = Act<X>::load(x + 8, p.L.K - k - 8);
        *(uint4*)(out + 16 * i) = uint4{lo.x, lo.y, hi.x, hi.y};
    } else {
        *(typename Act<X>::M::frag*)(out + 16 * i) = Act<X>::frag(Act<X>::load(x, p.L.K - k));
    }
}

// y from the sums of the column ranges, added in order.
__global__ __launch_bounds__(256) void k_w4_sum(W4GemmParams p, int splits) {
    const int64_t np = 32 * (int64_t)p.L.tiles, cols = np / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.M * cols) return;
    const int64_t m = i / cols;
    const int n = 8 * (int)(i - m * cols);
    const float* q = p.part + m * np + n;
    f32x8 v = *(const f32x8*)q;
    for (int z = 1; z < splits; z++) v += *(const f32x8*)(q + z * p.M * np);
    if (p.x_scale) v *= p.x_scale[m];
    if (n >= p.L.N) return;
    with_y(p, [&](auto* y) {
        typedef std::remove_reference_t<decltype(*y)> Y;
        store8(y + m * p.ldy + n, __builtin_convertvector(v, typename Vec8<Y>::type), p.L.N - n);
    });
}

// No columns: zeros, whatever x_scale holds.
__global__ __launch_bounds__(256) void k_w4_zero(W4GemmParams p) {
    const int64_t cols = (p.L.N + 7) / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.M * cols) return;
    const int64_t m = i / cols;
    const int n = 8 * (int)(i - m * cols);
    with_y(p, [&](auto* y) {
        typedef std::remove_reference_t<decltype(*y)> Y;
        store8(y + m * p.ldy + n, typename Vec8<Y>::type{}, p.L.N - n);
    });
}

// The shapes of k_w4_tile and what they cost, us: of a workgroup beyond a launch, of each further round of
// workgroups, and of a step on one CU holding 1 .. slots of them (fitted to sizes of 16 to 1024 rows,
// 1024 to 18432 outputs, K = 4096 and 9216, G = 128, each with every shape and number of splits: 24 for
// 16-bit rows, 40 for 8-bit ones).  Small
// tiles spread few rows over the chip, large ones read less per product; 32 x 64 tiles split their steps
// over 8 parts of a workgroup, 32 x 128 over 4, and over 8 where a CU gets only one (64 fp16 rows of
// 9216 x 4096, G = 32: 18.9 us with 4, 17.4 with 8; 128 rows: 25.9 and 33.2).
struct TileShape {
    int bm, bn, slots;
    float fix, again, step[2];
};
constexpr TileShape kShapes16[] = {{32, 64, 1, 0.5f, 4.0f, {0.105f}},
                                   {64, 256, 2, 0.0f, 0.0f, {0.615f, 1.025f}},
                                   {32, 128, 2, 0.0f, 1.0f, {0.185f, 0.285f}},
                                   {32, 128, 1, 1.3f, 4.0f, {0.16f}},
                                   {64, 256, 1, 2.2f, 1.5f, {0.50f}},
                                   {128, 256, 1, 0.0f, 0.0f, {1.00f}},
                                   {128, 256, 2, 0.0f, 0.0f, {1.10f, 1.96f}}};
constexpr TileShape kShapes8[] = {{32, 64, 1, 0.7f, 3.7f, {0.22f}},
                                  {64, 128, 2, 0.0f, 0.0f, {0.98f, 1.21f}},
                                  {32, 128, 1, 1.0f, 3.3f, {0.39f}},
                                  {64, 128, 1, 1.5f, 4.9f, {0.54f}},
                                  {128, 128, 1, 0.8f, 5.4f, {1.05f}},
                                  {128, 256, 1, 0.0f, 7.0f, {1.92f}},
                                  {128, 256, 2, 1.2f, 0.0f, {2.06f, 3.04f}}};
// rows through registers: a step of small tiles costs more, 64 x 256 tiles lose to 32 x 256 at every size
// (1024 rows of 4096 x 4096: 60.9 us against 50.0)
constexpr TileShape kLoose16[] = {{32, 64, 1, 0.5f, 4.0f, {0.16f}}, {32, 256, 2, 0.0f, 0.0f, {0.53f, 0.66f}}};
constexpr TileShape kLoose8[] = {{32, 64, 1, 0.5f, 3.6f, {0.41f}},
                                 {64, 128, 1, 0.1f, 3.8f, {0.72f}},
                                 {64, 128, 2, 2.2f, 0.0f, {1.00f, 1.32f}}};

// The shape and the ranges of columns (splits) that should take the least time: rounds of full CUs,
// then one of what is left; splits write and read fp32 sums at about 4 TB/s and launch one more kernel.
// room: bytes for the sums.
struct TilePlan {
    int shape, splits;
};
size_t sums_bytes(int64_t M, const W4Layout& L, int splits) {
    return splits > 1 ? (size_t)splits * M * L.tiles * 32 * 4 : 0;
}
TilePlan tile_plan(int64_t M, const W4Layout& L, bool f8, bool dma, size_t room) {
    const int steps = f8 ? (L.chunks + 1) / 2 : L.chunks;
    const double cus = num_cus();
    TilePlan best = {0, 1};
    double least = 1e30;
    const int shapes = dma ? 7 : f8 ? 3 : 2;
    for (int v = 0; v < shapes; v++) {
        // the last shape's registers do not hold the two scales that a step of groups of 32 has
        if (L.group == 32 && v == 6) continue;
        const TileShape& s = dma ? (f8 ? kShapes8[v] : kShapes16[v]) : f8 ? kLoose8[v] : kLoose16[v];
        const double tiles = (double)((M + s.bm - 1) / s.bm) * ((L.N + s.bn - 1) / s.bn);
        for (int z : {1, 2, 3, 4, 6, 8}) {
            if (steps < 4 * z && z > 1) break;
            if (sums_bytes(M, L, z) > room) break;
            const double held = ceil(tiles * z / cus), rounds = floor((held - 1) / s.slots);
            const int rest = (int)(held - rounds * s.slots);
            double us = s.fix + rounds * s.again +
                        (rounds * s.step[s.slots - 1] + s.step[rest - 1]) * ceil((double)steps / z);
            if (z > 1) us += 4.5 + z * (double)M * L.tiles * 32 * 8 / 4e6;
            if (us < least) {
                least = us;
                best = {v, z};
            }
        }
    }
    return best;
}

constexpr int64_t kRowsOfALaunch = 1 << 17;     // tiles of one launch stay below 2^31

// Whether E4M3 rows come to LDS in 8 bits (F8): the scales that a step of 128 columns has with groups of
// 32 would not fit a wave's DMA.
bool takes_f8(int x_type, int group) { return x_type == kE4M3 && group >= 64; }
// Whether the rows can be fetched by DMA, 16-byte pieces in place; E4M3 rows that LDS holds as bf16 are
// converted on their way.
bool takes_dma(const W4GemmParams& p, int x_type, bool f8) {
    const int es = x_type == kE4M3 ? 1 : 2;
    if (p.aligned) return true;
    return (f8 || es == 2) && (uintptr_t)p.x % 16 == 0 && p.ldx * es % 16 == 0 && (int64_t)p.L.K * es % 16 == 0;
}

template <typename X, int F8, int G, int TM, int WM, int WN, int KW, int R, int DMA>
hipError_t launch_tile(const W4GemmParams& p, int splits, hipStream_t s) {
    const int tm = (int)((p.M + 32 * TM * WM - 1) / (32 * TM * WM)), tn = (p.L.tiles + 2 * WN - 1) / (2 * WN);
    const int steps = F8 ? (p.L.chunks + 1) / 2 : p.L.chunks, per = (steps + splits - 1) / splits;
    splits = (steps + per - 1) / per;            // none without steps
    W4GemmParams q = p;
    q.part = splits > 1 ? (float*)p.ws : nullptr;
    k_w4_tile<X, F8, G, TM, WM, WN, KW, R, DMA><<<(unsigned)(tm * tn * splits), 64 * WM * WN * KW, 0, s>>>(q, tm, tm * tn, per);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && splits > 1) {
        k_w4_sum<<<(unsigned)((p.M * p.L.tiles * 4 + 255) / 256), 256, 0, s>>>(q, splits);
        e = hipGetLastError();
    }
    return e;
}

// From so many rows on, rows that DMA cannot take are aligned first, where there is room for them (4000
// outputs of K = 4001, us aligned first and not: bf16 128 rows 15.8 / 16.8, 512 rows 29.9 / 35.8, 4000
// rows 130 / 178; E4M3 128 rows 15.6 / 18.8, 512 rows 28.7 / 28.1, 4000 rows 124 / 181).  With fewer rows
// it takes a workspace of the rows' size to save 1.5 to 4 us (64 rows: 15.1 / 16.6, E4M3 14.9 / 18.7).
constexpr int64_t kAlignRows = 128;
int64_t aligned_pitch(const W4Layout& L) { return 64 * (int64_t)L.chunks; }      // elements
size_t aligned_bytes(int64_t M, const W4Layout& L, bool f8) { return (size_t)M * aligned_pitch(L) * (f8 ? 1 : 2); }

template <typename X, int F8, int G>
hipError_t launch_shape(const W4GemmParams& p, int x_type, hipStream_t s) {
    const bool dma = takes_dma(p, x_type, F8);
    const size_t copy = aligned_bytes(p.M, p.L, F8);
    if (!dma && p.M >= kAlignRows && p.ws_bytes >= copy) {
        constexpr int to = F8 ? 1 : 2;
        W4GemmParams q = p;
        q.x = p.ws;
        q.ldx = aligned_pitch(p.L);
        q.aligned = true;                    // pieces that K cuts hold zeros past it
        q.ws = p.ws + copy;
        q.ws_bytes = p.ws_bytes - copy;
        const int pieces = (int)(q.ldx * to / 16);
        k_w4_align<X, to><<<(unsigned)((p.M * pieces + 255) / 256), 256, 0, s>>>(p, p.ws, pieces);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if constexpr (sizeof(X) == 1 && !F8) return launch_shape<__bf16, 0, G>(q, kBF16, s);
        else return launch_shape<X, F8, G>(q, x_type, s);
    }
    const TilePlan t = tile_plan(p.M, p.L, F8, dma, p.ws_bytes);
    if constexpr (F8) {
        if (!dma) {
            if (t.shape == 0) return launch_tile<X, 1, G, 1, 1, 1, 8, 2, 0>(p, t.splits, s);
            if (t.shape == 1) return launch_tile<X, 1, G, 1, 2, 2, 4, 2, 0>(p, t.splits, s);
            return launch_tile<X, 1, G, 1, 2, 2, 1, 4, 0>(p, t.splits, s);
        }
        if (t.shape == 0) return launch_tile<X, 1, G, 1, 1, 1, 8, 2, 1>(p, t.splits, s);
        if (t.shape == 1) return launch_tile<X, 1, G, 1, 2, 2, 1, 4, 1>(p, t.splits, s);
        if (t.shape == 2) return launch_tile<X, 1, G, 1, 1, 2, 4, 2, 1>(p, t.splits, s);
        if (t.shape == 3) return launch_tile<X, 1, G, 1, 2, 2, 4, 2, 1>(p, t.splits, s);
        if (t.shape == 4) return launch_tile<X, 1, G, 2, 2, 2, 2, 2, 1>(p, t.splits, s);
        if (t.shape == 5) return launch_tile<X, 1, G, 2, 2, 4, 1, 4, 1>(p, t.splits, s);
        return launch_tile<X, 1, G, 4, 1, 4, 1, 2, 1>(p, t.splits, s);
    } else {
        if constexpr (sizeof(X) == 2) {
            if (dma) {
                if (t.shape == 0) return launch_tile<X, 0, G, 1, 1, 1, 8, 2, 1>(p, t.splits, s);
                if (t.shape == 1) return launch_tile<X, 0, G, 2, 1, 4, 1, 4, 1>(p, t.splits, s);
                if (t.shape == 2) return launch_tile<X, 0, G, 1, 1, 2, 4, 2, 1>(p, t.splits, s);
                if (t.shape == 3) return launch_tile<X, 0, G, 1, 1, 2, 8, 2, 1>(p, t.splits, s);
                if (t.shape == 4) return launch_tile<X, 0, G, 2, 1, 4, 2, 4, 1>(p, t.splits, s);
                if (t.shape == 5) return launch_tile<X, 0, G, 2, 2, 4, 1, 4, 1>(p, t.splits, s);
                if constexpr (G > 32) return launch_tile<X, 0, G, 4, 1, 4, 1, 3, 1>(p, t.splits, s);
            }
        }
        if (t.shape == 0) return launch_tile<X, 0, G, 1, 1, 1, 8, 2, 0>(p, t.splits, s);
        return launch_tile<X, 0, G, 1, 1, 4, 2, 3, 0>(p, t.splits, s);
    }
}

// A token's kernel reads the weights once, without LDS, but every row in pieces and the weights' decoding
// once per wave: with more than a few rows it wins only while its workgroups come at about one per CU or
// the weights are few.  us here against tiles, 16-bit / E4M3 rows: 16 rows of 4096 x 4096 7.2 : 11.1 / 7.9 :
// 10.5, of 4096 x 9216 12.7 : 13.8 / 12.7 : 14.4, of 9216 x 1024 5.7 : 6.7 / 7.8 : 7.8, of 9216 x 4096
// 15.5 : 12.1 / 15.4 : 12.6; 18432 x 4096 with 6 rows 15.3 : 15.9 / 15.5 : 17.2, 8 rows 17.3 : 15.7 /
// 17.4 : 17.2.
bool takes_token(int64_t M, const W4Layout& L) {
    const int64_t few = (2 * (int64_t)L.tiles <= num_cus() * 3 / 2 ? 40 : 12) << 20;
    return M <= 6 || (M <= 16 && (int64_t)L.N * L.K <= few);
}

template <typename X, int G>
hipError_t launch_g(const W4GemmParams& p, int x_type, hipStream_t s) {
    if (takes_token(p.M, p.L)) {
        // 16 waves where the CUs get about one workgroup each, else 8 (one row, K = 9216, 4096 outputs:
        // 7.2 us against 9.0; K = 4096, 18432 outputs: 14.0 against 11.7)
        const unsigned grid = 2 * p.L.tiles;
        if ((int)grid <= num_cus() * 3 / 2) k_w4_token<X, G, 16, 2><<<grid, 1024, 0, s>>>(p);
        else k_w4_token<X, G, 8, 2><<<grid, 512, 0, s>>>(p);
        return hipGetLastError();
    }
    if constexpr (sizeof(X) == 1 && G >= 64) {
        if (takes_f8(x_type, G)) return launch_shape<X, 1, G>(p, x_type, s);
    }
    return launch_shape<X, 0, G>(p, x_type, s);
}

template <typename X>
hipError_t launch_x(const W4GemmParams& p, int x_type, hipStream_t s) {
    if (p.L.group == 32) return launch_g<X, 32>(p, x_type, s);
    if (p.L.group == 64) return launch_g<X, 64>(p, x_type, s);
    return launch_g<X, 128>(p, x_type, s);
}

hipError_t launch_zero(const W4GemmParams& p, hipStream_t s) {
    k_w4_zero<<<(unsigned)((p.M * ((p.L.N + 7) / 8) + 255) / 256), 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace

size_t w4_gemm_workspace(int64_t M, const W4Layout& L, int x_type) {
    M = M < kRowsOfALaunch ? M : kRowsOfALaunch;
    const bool f8 = takes_f8(x_type, L.group);
    if (L.K == 0 || takes_token(M, L)) return 0;
    // rows of whole 16-byte pieces are expected to be aligned; others cannot be
    const int es = x_type == kE4M3 ? 1 : 2;
    const bool dma = (f8 || es == 2) && (int64_t)L.K * es % 16 == 0, copy = !dma && M >= kAlignRows;
    return (copy ? aligned_bytes(M, L, f8) : 0) + sums_bytes(M, L, tile_plan(M, L, f8, dma || copy, SIZE_MAX).splits);
}

hipError_t launch_w4_gemm(const W4GemmParams& p, int x_type, hipStream_t s) {
    const int xs = x_type == kE4M3 ? 1 : 2, ys = p.y_type == kF32 ? 4 : 2;
    for (int64_t m = 0; m < p.M; m += kRowsOfALaunch) {
        W4GemmParams q = p;
        q.M = p.M - m < kRowsOfALaunch ? p.M - m : kRowsOfALaunch;
        q.x = (const char*)p.x + m * p.ldx * xs;
        if (p.x_scale) q.x_scale = p.x_scale + m;
        q.y = (char*)p.y + m * p.ldy * ys;
        const hipError_t e = p.L.K == 0        ? launch_zero(q, s)
                             : x_type == kBF16 ? launch_x<__bf16>(q, x_type, s)
                             : x_type == kF16  ? launch_x<_Float16>(q, x_type, s)
                                               : launch_x<uint8_t>(q, x_type, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace esb
