// Products of float or 8-bit activations with 4-bit weights (w4.hip's layout):
//   y[m][n] = s_m sum_g alpha[n][g] sum_{k in g} x[m][k] q[n][k].
//
// The activations are the first operand of the MFMAs (rows m), the weights the second (columns n):
// a lane holds outputs of one n, so a group's scale is one value per lane.  E2M1 values are exact in
// bf16 and fp16, E4M3 activations in bf16, so a group's products are exact and its sum fp32; the
// group's scale multiplies that sum in fp32, and the sums of the groups are added in fp32.
//
// Three kernels, by how many rows share the weights:
//  * k_w4_token (M <= 16): 16 outputs per workgroup, the reduction split over its waves; the weights
//    are read once from HBM and are all that costs.
//  * k_w4_batch: 32 outputs x up to 64 rows per workgroup, split the same way.
//  * k_w4_tile: large tiles, the activations through LDS, the weights straight into registers.
#include "float_rows.h"

namespace esb {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

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

// 16 outputs n x 16 rows m per workgroup, the column chunks dealt to its NW waves and their sums
// added in LDS in wave order.
template <typename X, int G, int NW>
__global__ __launch_bounds__(64 * NW) void k_w4_token(W4GemmParams p) {
    typedef typename Act<X>::M M;
    __shared__ f32x4 red[NW][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, s = lane >> 4;
    const int nt = blockIdx.x >> 1, row = 16 * (blockIdx.x & 1) + r;
    if (32 * nt + 16 * (int)(blockIdx.x & 1) >= p.L.N) return;
    const int64_t m0 = (int64_t)blockIdx.y * 16;
    const bool live = m0 + r < p.M;
    const X* x = (const X*)p.x + (live ? m0 + r : 0) * p.ldx;
    const int h = s >> 1, e = s & 1;
    const uint8_t* w = p.w4 + (int64_t)nt * p.L.chunks * 1024 + 16 * (32 * h + row) + 8 * e;
    const uint16_t* sc = (const uint16_t*)(p.w4 + p.L.scale_offset) + (int64_t)nt * p.L.groups * 32 + row;
    f32x4 acc = {0, 0, 0, 0};
    for (int kc = wave; kc < p.L.chunks; kc += NW) {
        const uint2 q = *(const uint2*)(w + (int64_t)kc * 1024);
        typename Act<X>::raw raw[2] = {};
        const int k = 64 * kc + 16 * e + 8 * h;
        if (live) {
            raw[0] = Act<X>::load(x + k, p.L.K - k);
            raw[1] = Act<X>::load(x + k + 32, p.L.K - k - 32);
        }
        const f32x4 zero = {0, 0, 0, 0};
        if (G == 32) {
            const f32x4 p0 = M::mma(Act<X>::frag(raw[0]), M::decode(q.x), zero);
            const f32x4 p1 = M::mma(Act<X>::frag(raw[1]), M::decode(q.y), zero);
            const float a0 = scale_value(sc[(int64_t)kc * 64]), a1 = scale_value(sc[(int64_t)kc * 64 + 32]);
#pragma unroll
            for (int i = 0; i < 4; i++) acc[i] = fmaf(a1, p1[i], fmaf(a0, p0[i], acc[i]));
        } else {
            const f32x4 p0 = M::mma(Act<X>::frag(raw[0]), M::decode(q.x), zero);
            const f32x4 p1 = M::mma(Act<X>::frag(raw[1]), M::decode(q.y), p0);
            const float a = scale_value(sc[(int64_t)(G == 64 ? kc : kc >> 1) * 32]);
#pragma unroll
            for (int i = 0; i < 4; i++) acc[i] = fmaf(a, p1[i], acc[i]);
        }
    }
    red[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    for (int u = 1; u < NW; u++) acc += red[u][lane];
    const int n = 32 * nt + row;
    if (n >= p.L.N) return;
    with_y(p, [&](auto* y) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t m = m0 + 4 * s + i;
            if (m < p.M) y[m * p.ldy + n] = p.x_scale ? acc[i] * p.x_scale[m] : acc[i];
        }
    });
}

// 32 outputs n x 32 MT rows m per workgroup, the column chunks dealt to its NW waves; each wave then
// adds its share of the sums of all, in wave order.
template <typename X, int G, int MT, int NW>
__global__ __launch_bounds__(64 * NW) void k_w4_batch(W4GemmParams p) {
    typedef typename Act<X>::M M;
    __shared__ float red[NW][MT * 16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
    const int nt = blockIdx.x;
    const int64_t m0 = (int64_t)blockIdx.y * 32 * MT;
    const X* x[MT];
    bool live[MT];
#pragma unroll
    for (int i = 0; i < MT; i++) {
        live[i] = m0 + 32 * i + r < p.M;
        x[i] = (const X*)p.x + (live[i] ? m0 + 32 * i + r : 0) * p.ldx;
    }
    const uint8_t* w = p.w4 + (int64_t)nt * p.L.chunks * 1024 + 16 * lane;
    const uint16_t* sc = (const uint16_t*)(p.w4 + p.L.scale_offset) + (int64_t)nt * p.L.groups * 32 + r;
    f32x16 acc[MT] = {};
    for (int kc = wave; kc < p.L.chunks; kc += NW) {
        const uint4 q = *(const uint4*)(w + (int64_t)kc * 1024);
        typename Act<X>::raw raw[MT][4] = {};
        const int k = 64 * kc + 8 * h;
#pragma unroll
        for (int i = 0; i < MT; i++)
            if (live[i])
#pragma unroll
                for (int t = 0; t < 4; t++) raw[i][t] = Act<X>::load(x[i] + k + 16 * t, p.L.K - k - 16 * t);
        const typename M::frag wf[4] = {M::decode(q.x), M::decode(q.z), M::decode(q.y), M::decode(q.w)};
        constexpr int NG = G == 32 ? 2 : 1;
        float a[NG];
#pragma unroll
        for (int g = 0; g < NG; g++) a[g] = scale_value(sc[(int64_t)(G == 128 ? kc >> 1 : NG * kc + g) * 32]);
#pragma unroll
        for (int i = 0; i < MT; i++)
#pragma unroll
            for (int g = 0; g < NG; g++) {
                f32x16 part = {};
#pragma unroll
                for (int t = 0; t < 4 / NG; t++)
                    part = M::mma(Act<X>::frag(raw[i][4 / NG * g + t]), wf[4 / NG * g + t], part);
#pragma unroll
                for (int j = 0; j < 16; j++) acc[i][j] = fmaf(a[g], part[j], acc[i][j]);
            }
    }
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < 16; j++) red[wave][16 * i + j][lane] = acc[i][j];
    __syncthreads();
    const int n = 32 * nt + r;
    if (n >= p.L.N) return;
    with_y(p, [&](auto* y) {
        for (int j = wave; j < 16 * MT; j += NW) {
            const int64_t m = m0 + 32 * (j >> 4) + 8 * ((j >> 2) & 3) + 4 * h + (j & 3);
            if (m >= p.M) continue;
            float v = red[0][j][lane];
#pragma unroll
            for (int u = 1; u < NW; u++) v += red[u][j][lane];
            y[m * p.ldy + n] = p.x_scale ? v * p.x_scale[m] : v;
        }
    });
}

template <int F8, typename F> struct FragOf { typedef F type; };
template <typename F> struct FragOf<1, F> { typedef i32x8 type; };

// Workgroup `id` of `total` to a tile: each XCD (every eighth id) gets a contiguous run.
__device__ __forceinline__ int xcd_run(int id, int total) {
    const int x = id & 7, q = total >> 3, rem = total & 7;
    return x * q + min(x, rem) + (id >> 3);
}

// Tiles of BM = 32 TM WM rows m x BN = 64 WN outputs n, a wave of the workgroup 32 TM x 64 of it.
// A step is 128 bytes of every row of the tile in LDS: 64 columns of 16-bit values (F8 == 0; E4M3
// activations become bf16 on their way) or 128 columns of E4M3 (F8 == 1).  16-byte piece c of row i
// is at c ^ ((i / 2) % 8) of its row, so that the 16 rows which one quarter of a wave reads at a time
// lie in different banks.  While a step's MFMAs run, the next step's weights and the activations of
// the one after it are on their way to registers.
template <typename X, int F8, int G, int TM, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_w4_tile(W4GemmParams p, int tiles_m, int tiles) {
    typedef typename Act<X>::M M;
    constexpr int T = 64 * WM * WN, BM = 32 * TM * WM;
    constexpr int BK = F8 ? 128 : 64, EP = F8 ? 16 : 8;       // columns of a step, of a piece
    constexpr int P = BM * 8 / T;                             // pieces of a thread
    constexpr int NC = F8 ? 2 : 1;                            // column chunks of a step
    constexpr int NG = F8 ? 128 / G : G == 32 ? 2 : 1;        // scales of a step
    __shared__ __align__(16) uint8_t lds[2][BM * 128];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, h = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    const int t = xcd_run(blockIdx.x, tiles);
    const int64_t m0 = (int64_t)(t % tiles_m) * BM;
    const int nt0 = (t / tiles_m) * (2 * WN) + 2 * wn;
    const int K = p.L.K, chunks = p.L.chunks, steps = (chunks + NC - 1) / NC;

    // this thread's pieces: piece tid % 8 of rows tid / 8 + i T / 8
    const int pc = tid & 7, pr = tid >> 3;
    const X* xp[P];
    uint32_t at[P];
#pragma unroll
    for (int i = 0; i < P; i++) {
        const int row = pr + i * (T / 8);
        const int64_t m = m0 + row < p.M ? m0 + row : p.M - 1;
        xp[i] = (const X*)p.x + m * p.ldx + EP * pc;
        at[i] = row * 128;
    }
    typedef typename Act<X>::raw Raw;
    Raw st[P][F8 ? 2 : 1];
    auto fetch = [&](int s) {
        const int k = s * BK;
        if (k + BK <= K) {
#pragma unroll
            for (int i = 0; i < P; i++)
#pragma unroll
                for (int u = 0; u < (F8 ? 2 : 1); u++) st[i][u] = Act<X>::load(xp[i] + k + 8 * u, 8);
        } else {
#pragma unroll
            for (int i = 0; i < P; i++)
#pragma unroll
                for (int u = 0; u < (F8 ? 2 : 1); u++)
                    st[i][u] = Act<X>::load(xp[i] + k + 8 * u, K - k - EP * pc - 8 * u);
        }
    };
    auto put = [&](int b) {
#pragma unroll
        for (int i = 0; i < P; i++) {
            const int sw = ((pr + i * (T / 8)) >> 1) & 7;
            if constexpr (F8) {
                // The instruction pairs 8-bit lane half h, 16-byte piece c with 4-bit lane half c, words
                // 2h and 2h + 1, which hold columns 16t + 8c .. + 7 of t = h and h + 2.
                const int u = pc >> 2, tt = pc & 3;
#pragma unroll
                for (int c = 0; c < 2; c++)
                    *(Raw*)(lds[b] + at[i] + 16 * ((4 * u + 2 * (tt & 1) + c) ^ sw) + 8 * (tt >> 1)) = st[i][c];
            } else {
                *(typename M::frag*)(lds[b] + at[i] + 16 * (pc ^ sw)) = Act<X>::frag(st[i][0]);
            }
        }
    };

    const uint8_t* wp[2];
    const uint16_t* sp[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
        const int nt = min(nt0 + j, p.L.tiles - 1);
        wp[j] = p.w4 + (int64_t)nt * chunks * 1024 + 16 * lane;
        sp[j] = (const uint16_t*)(p.w4 + p.L.scale_offset) + (int64_t)nt * p.L.groups * 32 + r;
    }
    uint4 wq[2][NC];
    uint16_t ws[2][NG];
    auto weights = [&](int s) {
#pragma unroll
        for (int j = 0; j < 2; j++) {
#pragma unroll
            for (int c = 0; c < NC; c++)
                wq[j][c] = NC == 1 || NC * s + c < chunks ? *(const uint4*)(wp[j] + (int64_t)(NC * s + c) * 1024)
                                                          : uint4{0, 0, 0, 0};
#pragma unroll
            for (int g = 0; g < NG; g++) {
                const int gi = F8 ? min(NG * s + g, p.L.groups - 1) : G == 128 ? s >> 1 : NG * s + g;
                ws[j][g] = sp[j][(int64_t)gi * 32];
            }
        }
    };

    // A step's products go group by group and tile by tile: the MFMAs of one (tile, group) are issued,
    // then the sums of the one before it are scaled and added under them.
    f32x16 acc[TM][2] = {};
    const uint32_t arow = (uint32_t)(wm * 32 * TM + r) * 128;
    const int swz = (r >> 1) & 7;
    constexpr int NF = F8 ? 2 : 4;      // MFMAs of a tile in a step
    constexpr int U = TM * 2 * NG;
    auto step = [&](int b, int next) {
        typedef typename FragOf<F8, typename M::frag>::type Frag;
        float a[2][NG];
        Frag wf[2][NF], x[NF];
#pragma unroll
        for (int j = 0; j < 2; j++) {
#pragma unroll
            for (int g = 0; g < NG; g++) a[j][g] = scale_value(ws[j][g]);
            if constexpr (F8) {
#pragma unroll
                for (int c = 0; c < NC; c++)
                    wf[j][c] = i32x8{(int)wq[j][c].x, (int)wq[j][c].y, (int)wq[j][c].z, (int)wq[j][c].w, 0, 0, 0, 0};
            } else {
                wf[j][0] = M::decode(wq[j][0].x);
                wf[j][1] = M::decode(wq[j][0].z);
                wf[j][2] = M::decode(wq[j][0].y);
                wf[j][3] = M::decode(wq[j][0].w);
            }
        }
        if (next < steps) weights(next);
        f32x16 part[2];
#pragma unroll
        for (int u = 0; u <= U; u++) {
            if (u < U) {
                const int i = u / (2 * NG), j = u / NG % 2, g = u % NG;
                if (u % (2 * NG) == 0) {
                    const uint8_t* base = lds[b] + arow + i * 32 * 128;
#pragma unroll
                    for (int c = 0; c < NF; c++) {
                        if constexpr (F8) {
                            const uint4 lo = *(const uint4*)(base + 16 * ((4 * c + 2 * h) ^ swz));
                            const uint4 hi = *(const uint4*)(base + 16 * ((4 * c + 2 * h + 1) ^ swz));
                            x[c] = i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w,
                                         (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
                        } else {
                            x[c] = *(const Frag*)(base + 16 * ((2 * c + h) ^ swz));
                        }
                    }
                }
                f32x16 d = {};
#pragma unroll
                for (int c = NF / NG * g; c < NF / NG * (g + 1); c++) {
                    if constexpr (F8) d = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x[c], wf[j][c], d, 0, 4, 0, 127, 0, 127);
                    else d = M::mma(x[c], wf[j][c], d);
                }
                part[u & 1] = d;
            }
            if (u > 0) {
                const int v = u - 1, i = v / (2 * NG), j = v / NG % 2, g = v % NG;
#pragma unroll
                for (int q = 0; q < 16; q++) acc[i][j][q] = fmaf(a[j][g], part[v & 1][q], acc[i][j][q]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (steps > 0) {
        fetch(0);
        put(0);
        fetch(1);
        weights(0);
        __syncthreads();
        for (int s = 0; s < steps; s++) {
            if (s + 1 < steps) put((s + 1) & 1);
            if (s + 2 < steps) fetch(s + 2);
            step(s & 1, s + 1);
            __syncthreads();
        }
    }

    with_y(p, [&](auto* y) {
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int q = 0; q < 16; q++) {
                const int64_t m = m0 + wm * 32 * TM + 32 * i + 8 * (q >> 2) + 4 * h + (q & 3);
                if (m >= p.M) continue;
                const float s = p.x_scale ? p.x_scale[m] : 1.0f;
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const int n = 32 * (nt0 + j) + r;
                    if (n < p.L.N) y[m * p.ldy + n] = s * acc[i][j][q];
                }
            }
    });
}

template <typename X, int F8, int G, int TM, int WM, int WN>
hipError_t launch_tile(const W4GemmParams& p, hipStream_t s) {
    const int tm = (int)((p.M + 32 * TM * WM - 1) / (32 * TM * WM)), tn = (p.L.tiles + 2 * WN - 1) / (2 * WN);
    k_w4_tile<X, F8, G, TM, WM, WN><<<tm * tn, 64 * WM * WN, 0, s>>>(p, tm, tm * tn);
    return hipGetLastError();
}

template <typename X, int G>
hipError_t launch_g(const W4GemmParams& p, hipStream_t s) {
    if (p.M <= 16) {
        const dim3 grid(2 * p.L.tiles, (unsigned)((p.M + 15) / 16));
        k_w4_token<X, G, 8><<<grid, 512, 0, s>>>(p);
        return hipGetLastError();
    }
    const int64_t t128 = (p.M + 127) / 128 * ((p.L.N + 127) / 128);
    if (p.M <= 64 || t128 < num_cus() / 2) {
        if (p.M <= 32) {
            const dim3 grid(p.L.tiles, (unsigned)((p.M + 31) / 32));
            k_w4_batch<X, G, 1, 8><<<grid, 512, 0, s>>>(p);
        } else {
            const dim3 grid(p.L.tiles, (unsigned)((p.M + 63) / 64));
            k_w4_batch<X, G, 2, 8><<<grid, 512, 0, s>>>(p);
        }
        return hipGetLastError();
    }
    // dropped small products (k_w4_tile) stay below the rounding of a 16-bit output, not of fp32
    if constexpr (sizeof(X) == 1 && G >= 64) {
        if (p.y_type != kF32) return launch_tile<X, 1, G, 2, 2, 2>(p, s);
    }
    return launch_tile<X, 0, G, 2, 2, 2>(p, s);
}

template <typename X>
hipError_t launch_x(const W4GemmParams& p, hipStream_t s) {
    if (p.L.group == 32) return launch_g<X, 32>(p, s);
    if (p.L.group == 64) return launch_g<X, 64>(p, s);
    return launch_g<X, 128>(p, s);
}

}  // namespace

hipError_t launch_w4_gemm(const W4GemmParams& p, int x_type, hipStream_t s) {
    const int64_t most = 1 << 19;      // rows of one launch: the grid's second dimension
    const int xs = x_type == kE4M3 ? 1 : 2, ys = p.y_type == kF32 ? 4 : 2;
    for (int64_t m = 0; m < p.M; m += most) {
        W4GemmParams q = p;
        q.M = p.M - m < most ? p.M - m : most;
        q.x = (const char*)p.x + m * p.ldx * xs;
        if (p.x_scale) q.x_scale = p.x_scale + m;
        q.y = (char*)p.y + m * p.ldy * ys;
        const hipError_t e = x_type == kBF16  ? launch_x<__bf16>(q, s)
                             : x_type == kF16 ? launch_x<_Float16>(q, s)
                                              : launch_x<uint8_t>(q, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace esb
