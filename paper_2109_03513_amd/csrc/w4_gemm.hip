// Products of float or 8-bit activations with 4-bit weights (w4.hip's layout):
//   y[m][n] = s_m sum_g alpha[n][g] sum_{k in g} x[m][k] q[n][k].
//
// The weights are the first operand of the MFMAs, 16 rows n of a tile, the activations the second,
// 16 rows m: a lane holds four consecutive outputs n of one row m.  E2M1 values are exact in bf16
// and fp16, E4M3 activations in bf16, so a group's products are exact and its sum fp32; the group's
// scale multiplies that sum in fp32, and the sums of the groups are added in fp32.
#include "float_rows.h"

namespace esb {

namespace {

typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));

// Four pairs of 16-bit values as one fragment.
template <typename F, typename P>
__device__ __forceinline__ F join(P a, P b, P c, P d) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(F, u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                       __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)});
}

struct Bf16 {
    typedef bf16x8 frag;
    typedef __bf16 elem;
    static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
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
    typedef _Float16 elem;
    static __device__ __forceinline__ f32x4 mma(frag a, frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ frag decode(uint32_t d) {
        return join<frag>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 0),
                          __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 2),
                          __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 3));
    }
};

// Eight E4M3 bytes to bf16 (exact).
__device__ __forceinline__ bf16x8 e4m3_to_bf16(uint2 v) {
    return join<bf16x8>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.x, 1.0f, false),
                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.x, 1.0f, true),
                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.y, 1.0f, false),
                        __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v.y, 1.0f, true));
}

// Eight activations of one row, zeros past the row's end.
template <typename X> struct Act;
template <> struct Act<__bf16> {
    typedef Bf16 M;
    static __device__ __forceinline__ bf16x8 load(const __bf16* p, int n) { return load8(p, n); }
};
template <> struct Act<_Float16> {
    typedef F16 M;
    static __device__ __forceinline__ f16x8 load(const _Float16* p, int n) { return load8(p, n); }
};
template <> struct Act<uint8_t> {
    typedef Bf16 M;
    static __device__ __forceinline__ bf16x8 load(const uint8_t* p, int n) {
        uint2 v = {0, 0};
        if (n >= 8) {
            v = ((const Loose<uint2, uint8_t>*)p)->v;
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < n) (i < 4 ? v.x : v.y) |= (uint32_t)p[i] << (8 * (i & 3));
        }
        return e4m3_to_bf16(v);
    }
};

__device__ __forceinline__ f32x4 scales4(u16x4 s) {
    f32x4 r;
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = __uint_as_float((uint32_t)s[i] << 16);
    return r;
}

// Outputs n .. n+3 of row m.
__device__ __forceinline__ void store4(const W4GemmParams& p, int64_t m, int n, f32x4 v) {
    const int left = p.L.N - n;
    const int64_t o = m * p.ldy + n;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (i >= left) break;
        if (p.y_type == kF32) ((float*)p.y)[o + i] = v[i];
        else if (p.y_type == kBF16) ((__bf16*)p.y)[o + i] = (__bf16)v[i];
        else ((_Float16*)p.y)[o + i] = (_Float16)v[i];
    }
}

// 16 outputs n x 16 rows m per workgroup, the column chunks dealt to its waves and their sums
// added in LDS in wave order.
template <typename X, int G>
__global__ __launch_bounds__(256) void k_w4_skinny(W4GemmParams p) {
    typedef typename Act<X>::M M;
    __shared__ f32x4 red[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, j = lane >> 4;
    const int nt = blockIdx.x;
    const int64_t m = (int64_t)blockIdx.y * 16 + r;
    const X* x = (const X*)p.x + (m < p.M ? m : p.M - 1) * p.ldx;
    const uint8_t* w = p.w4 + (int64_t)nt * p.L.chunks * 1024;
    const uint16_t* sc = (const uint16_t*)(p.w4 + p.L.scale_offset) + (int64_t)nt * p.L.groups * 16;
    constexpr int TG = G / 32;
    f32x4 acc = {0, 0, 0, 0};
    for (int kc = wave; kc < p.L.chunks; kc += 4) {
        const uint4 q = *(const uint4*)(w + (int64_t)kc * 1024 + 16 * lane);
        const uint32_t qd[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int g = 0; g < 4 / TG; g++) {
            f32x4 part = {0, 0, 0, 0};
#pragma unroll
            for (int t = g * TG; t < (g + 1) * TG; t++) {
                const int k = 128 * kc + 32 * t + 8 * j;
                part = M::mma(M::decode(qd[t]), Act<X>::load(x + k, p.L.K - k), part);
            }
            const f32x4 a = scales4(*(const u16x4*)(sc + ((int64_t)kc * (4 / TG) + g) * 16 + 4 * j));
#pragma unroll
            for (int i = 0; i < 4; i++) acc[i] = fmaf(a[i], part[i], acc[i]);
        }
    }
    red[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    for (int u = 1; u < 4; u++) acc += red[u][lane];
    if (m >= p.M) return;
    if (p.x_scale) acc *= p.x_scale[m];
    store4(p, m, 16 * nt + 4 * j, acc);
}

template <typename X>
hipError_t launch_x(const W4GemmParams& p, hipStream_t s) {
    const dim3 grid((unsigned)p.L.tiles, (unsigned)((p.M + 15) / 16));
    if (p.L.group == 32) k_w4_skinny<X, 32><<<grid, 256, 0, s>>>(p);
    else if (p.L.group == 64) k_w4_skinny<X, 64><<<grid, 256, 0, s>>>(p);
    else k_w4_skinny<X, 128><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
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
