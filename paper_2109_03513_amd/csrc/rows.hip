// Row operators between a decoder's products, each one pass over its rows with 8-bit outputs:
//
//  * the root-mean-square norm with the residual's addition: z = x + r, y = z rstd w,
//    rstd = 1 / sqrt(mean z^2 + eps);
//  * the gated activation h = gate / (1 + exp(-gate)) * up.
//
// Outputs are the rows in the inputs' type and / or OCP E4M3 bytes under one scale per row,
// s = max(max|y| / 448, 2^-126), byte = y (1/s) rounded to nearest even: the operand of
// esb_w4_gemm.  A row stays in registers between its two reductions (the sum of squares, the
// maximum), so HBM sees each input and output once; that bounds them: 4096 rows of 4096 bf16 with a
// residual 22.6 us (5.2 TB/s), gated activations of 4096 x 9216 bf16 36.5 us (5.2 TB/s), 1999 fp32 rows
// of 1000 6.7 us; one row of 4096 3.2 us, which is a launch and one round trip to memory.
//
// The sum of squares is held in fp64: squares of fp32 values up to the largest do not overflow,
// and rstd is the fp32 value next to the exact one (of rows above 2^126, a subnormal one of 22 bits).  Everything else is fp32,
// rounded once to the output's type.
#include "float_rows.h"

namespace esb {

namespace {

constexpr float kE4M3Max = 448.0f;
constexpr float kTiny = 0x1p-126f;

// exp(c) = 2^hi (1 + lo ln 2): hi the rounded product c log2(e), lo what the product lost.
struct Exp2Parts {
    float hi, lo;
};
__device__ __forceinline__ Exp2Parts exp2_parts(float c) {
    const float hi = c * 0x1.715476p+0f;
    return {hi, fmaf(c, 0x1.4ae0cp-26f, fmaf(c, 0x1.715476p+0f, -hi))};
}
// g / (1 + exp(-g)) within 9 roundings for g >= kFar (and NaN): exp by the hardware's exp2, the quotient by
// its reciprocal, whose results end at 2^-126, so at g = -87.
constexpr float kFar = -64.0f;
__device__ __forceinline__ float silu(float g) {
    const Exp2Parts p = exp2_parts(__builtin_amdgcn_fmed3f(-g, -104.0f, 104.0f));   // exp is 0 beyond
    const float e = __builtin_amdgcn_exp2f(p.hi) * fmaf(p.lo, 0x1.62e43p-1f, 1.0f);
    return g * __builtin_amdgcn_rcpf(1.0f + e);
}
// g / (1 + exp(-g)) * u for g < kFar, where it is g exp(g) u to fp32: the exponential's power of two is
// applied last, so that only the result may leave the range of normal numbers (u 2^-16 does so only
// under a result of 2^-190).  Below -256 it is 0 for every finite u; a gate of -infinity gives NaN.
__device__ __forceinline__ float silu_far(float g, float u) {
    const float c = fmaxf(g, -256.0f);
    const Exp2Parts p = exp2_parts(c);
    const float n = rintf(p.hi), m = __builtin_amdgcn_exp2f(p.hi - n) * fmaf(p.lo, 0x1.62e43p-1f, 1.0f);
    return __builtin_amdgcn_ldexpf(c * m * (u * 0x1p-16f), (int)n + 16) + (g - c) * 0.0f;
}

// TPR threads to a row, NV vectors of eight elements to a thread (d <= 8 TPR NV).  With 64 threads a wave
// works alone, four of them to a workgroup; else a row has a workgroup.
template <int OP, typename T, int TPR, int NV>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_rows(RowsParams p) {
    typedef typename Vec8<T>::type V;
    constexpr int W = TPR / 64;
    __shared__ double red[W];
    __shared__ uint32_t redm[W];
    const int tid = threadIdx.x % TPR, lane = tid & 63, wave = tid >> 6;
    const int64_t row = W > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (row >= p.rows) return;
    const int d = p.d;
    const T* a = (const T*)p.a + row * p.lda;
    const T* b = p.b ? (const T*)p.b + row * p.ldb : nullptr;

    // Outputs may lie over the inputs: a thread reads an element before it writes it.  With few vectors
    // to a thread every load is issued before the first store; many would not fit its registers.
    constexpr int AHEAD = NV <= 2 ? NV : 1;
    f32x8 v[NV];
    double ss = 0.0;
#pragma unroll
    for (int u0 = 0; u0 < NV; u0 += AHEAD) {
        V ra[AHEAD], rb[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int e = 8 * ((u0 + u) * TPR + tid);
            ra[u] = rb[u] = V{};
            if (e < d) {
                ra[u] = load8(a + e, d - e);
                if (b) rb[u] = load8(b + e, d - e);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int e = 8 * ((u0 + u) * TPR + tid);
            v[u0 + u] = f32x8{};
            if (e >= d) continue;
            f32x8 x = __builtin_convertvector(ra[u], f32x8);
            const f32x8 y = __builtin_convertvector(rb[u], f32x8);
            if (OP == kRowsNorm) {
                if (b) x += y;
                if (p.sum) store8((T*)p.sum + row * p.lds + e, __builtin_convertvector(x, V), d - e);
#pragma unroll
                for (int i = 0; i < 8; i++) ss = fma((double)x[i], (double)x[i], ss);
            } else {
                const f32x8 g = x;
                float least = g[0];
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    x[i] = silu(g[i]) * y[i];
                    least = fminf(least, g[i]);
                }
                if (least < kFar)
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        if (g[i] < kFar) x[i] = silu_far(g[i], y[i]);
            }
            v[u0 + u] = x;
        }
        if (AHEAD < NV) __builtin_amdgcn_sched_barrier(0);
    }
    if (OP == kRowsNorm) {
        f32x8 w[AHEAD];
        auto weights = [&](int u) {
            const int e = 8 * (u * TPR + tid);
            return p.w && e < d ? load8(p.w + e, d - e) : f32x8{1, 1, 1, 1, 1, 1, 1, 1};
        };
        if (AHEAD == NV)
#pragma unroll
            for (int u = 0; u < AHEAD; u++) w[u] = weights(u);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) ss += __shfl_xor(ss, o);
        if (W > 1) {
            if (lane == 0) red[wave] = ss;
            __syncthreads();
            ss = 0.0;
#pragma unroll
            for (int i = 0; i < W; i++) ss += red[i];
        }
        const float rstd = (float)(1.0 / sqrt(ss / (double)d + (double)p.eps));
#pragma unroll
        for (int u = 0; u < NV; u++) {
            v[u] = v[u] * rstd * (AHEAD == NV ? w[u % AHEAD] : weights(u));
            if (AHEAD < NV) __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (p.y) {
#pragma unroll
        for (int u = 0; u < NV; u++) {
            const int e = 8 * (u * TPR + tid);
            if (e < d) store8((T*)p.y + row * p.ldy + e, __builtin_convertvector(v[u], V), d - e);
        }
    }
    if (!p.y8) return;
    // max |y|, on bit patterns: a NaN is above every number
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < NV; u++)
        if (8 * (u * TPR + tid) < d)
#pragma unroll
            for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[u][i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    if (W > 1) {
        if (lane == 0) redm[wave] = m;
        __syncthreads();
        m = 0;
#pragma unroll
        for (int i = 0; i < W; i++) m = max(m, redm[i]);
    }
    // a NaN or an infinity in the row: no scale fits it
    const float s = m < 0x7f800000u ? fmaxf(__uint_as_float(m) / kE4M3Max, kTiny) : __builtin_nanf("");
    const float inv = 1.0f / s;
    if (tid == 0) p.scale[row] = s;
#pragma unroll
    for (int u = 0; u < NV; u++) {
        const int e = 8 * (u * TPR + tid);
        if (e >= d) continue;
        const uint2 q = to_e4m3(v[u] * inv);
        uint8_t* o = p.y8 + row * p.ld8 + e;
        if (d - e >= 8) {
            ((Loose<uint2, uint8_t>*)o)->v = q;
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < d - e) o[i] = (uint8_t)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
        }
    }
}

template <int OP, typename T, int TPR, int NV>
hipError_t launch_n(const RowsParams& p, hipStream_t s) {
    const int64_t most = 1 << 21;      // rows of one launch
    for (int64_t r = 0; r < p.rows; r += most) {
        RowsParams q = p;
        q.rows = p.rows - r < most ? p.rows - r : most;
        q.a = (const T*)p.a + r * p.lda;
        if (p.b) q.b = (const T*)p.b + r * p.ldb;
        if (p.sum) q.sum = (T*)p.sum + r * p.lds;
        if (p.y) q.y = (T*)p.y + r * p.ldy;
        if (p.y8) q.y8 = p.y8 + r * p.ld8, q.scale = p.scale + r;
        k_rows<OP, T, TPR, NV><<<(unsigned)(TPR > 64 ? q.rows : (q.rows + 3) / 4), TPR > 64 ? TPR : 256, 0, s>>>(q);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int OP, typename T>
hipError_t launch_t(const RowsParams& p, hipStream_t s) {
    // Measured over 1 to 4096 rows of 512 to 16384 (bf16, us, norm / gate): one vector to a thread as far
    // as 512 threads go, a wave to a row only for many short ones (4096 x 1024: 8.9 / 7.5 against 10.6 /
    // 8.3; 4096 x 4096: 31.6 / 25.8 against 26.5 / 18.8 with 512 threads).
    const int d = p.d;
    if (d <= 1024 && p.rows >= 4 * num_cus()) return launch_n<OP, T, 64, 2>(p, s);
    if (d <= 2048) return launch_n<OP, T, 256, 1>(p, s);
    if (d <= 4096) return launch_n<OP, T, 512, 1>(p, s);
    if (d <= 8192) return launch_n<OP, T, 512, 2>(p, s);
    if (d <= 16384) return launch_n<OP, T, 1024, 2>(p, s);
    if (d <= 32768) return launch_n<OP, T, 1024, 4>(p, s);
    return launch_n<OP, T, 1024, 8>(p, s);
}

}  // namespace

hipError_t launch_rows(int op, int type, const RowsParams& p, hipStream_t s) {
    if (op == kRowsNorm) {
        if (type == kF32) return launch_t<kRowsNorm, float>(p, s);
        if (type == kBF16) return launch_t<kRowsNorm, __bf16>(p, s);
        return launch_t<kRowsNorm, _Float16>(p, s);
    }
    if (type == kF32) return launch_t<kRowsGated, float>(p, s);
    if (type == kBF16) return launch_t<kRowsGated, __bf16>(p, s);
    return launch_t<kRowsGated, _Float16>(p, s);
}

}  // namespace esb
