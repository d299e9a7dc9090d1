// What the attention kernels share: one pass of softmax attention over tiles of keys in LDS (attention.hip, kv4_prompt.hip),
// 32 rows (queries x heads) to a wave, on 32x32x16 MFMAs, with a running maximum and sum; the decoding of the 4-bit
// cache, and the fallback over it for numbers that lie too far apart for the usual passes.
#pragma once

#include <type_traits>

#include "kv4.h"

namespace esb {

constexpr float kLazy = 8.0f;      // how far a score may pass the maximum (log2)
// A maximum m from which on scores are rounded before it is taken from them: x scale - m in one rounding is off by the
// rounding of m itself, 2^-24 of it, which soon is more than exp2 may be given.
constexpr float kFar = 0x1p20f;
constexpr float kNegInf = -__builtin_inff();

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename F, typename P>
__device__ __forceinline__ F join4(P a, P b, P c, P d) {
    return __builtin_bit_cast(F, u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                       __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)});
}
// Eight nibbles, lowest first.
__device__ __forceinline__ bf16x8 decode(uint32_t w, __bf16) {
    return join4<bf16x8>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
}
__device__ __forceinline__ f16x8 decode(uint32_t w, _Float16) {
    return join4<f16x8>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2),
                        __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3));
}
// Four bf16 scales as fp32.
__device__ __forceinline__ f32x4 four(uint2 s) {
    return f32x4{__uint_as_float(s.x << 16), __uint_as_float(s.x & 0xffff0000u), __uint_as_float(s.y << 16),
                 __uint_as_float(s.y & 0xffff0000u)};
}

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f16x8 a, f16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// Whether a maximum has to move from `top` for a score of `most`.
__device__ __forceinline__ bool passes(float most, float top, float lazy = kLazy) {
    return most > top + lazy || (top == kNegInf && most > kNegInf);
}
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// Keys of a tile are rows of DP / 8 16-byte pieces, piece c of a row at c ^ key_turn(row), so that 16 rows of one
// piece lie in distinct banks.
template <int DP> __device__ __forceinline__ int key_turn(int row) { return DP == 64 ? (row >> 1) & 7 : row & 15; }

// A lane holds one row (lane % 32): of the scores S^T = K Q^T of a 32-key block keys 8 (i / 4) + 4 (lane / 32) + i % 4,
// which are those that the second product O^T = V^T P^T wants of its operand, eight at a time; of O^T the
// elements 32 d + 8 (i / 4) + 4 (lane / 32) + i % 4.
template <typename T, int DP, int KT> struct Attend {
    typedef typename Vec8<T>::type V;
    static constexpr int P = DP / 8, DB = DP / 32, KB = KT / 32;
    // How far `top` is set above the maximum: weights of bf16 values are then at most 1, as their sums might leave fp32; fp16
    // needs its whole range for the weights, and its values have none to speak of.
    static constexpr float kLift = std::is_same<T, __bf16>::value ? kLazy : 0.0f;
    V qf[DP / 16];       // elements 16 s + 8 (lane / 32) .. + 7 of the row
    f32x16 acc[DB], x[KB];
    float top, sum;      // the running maximum (times scale, and lifted), and the lane's part of the sum

    __device__ __forceinline__ void start() {
#pragma unroll
        for (int d = 0; d < DB; d++) acc[d] = f32x16{};
        top = kNegInf, sum = 0.0f;
    }

    // Scores of a tile.
    __device__ __forceinline__ void scores(const V* kt) {
        const int col = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
#pragma unroll
        for (int b = 0; b < KB; b++) x[b] = f32x16{};
#pragma unroll
        for (int s = 0; s < DP / 16; s++)
#pragma unroll
            for (int b = 0; b < KB; b++) {
                const int r = 32 * b + col;
                x[b] = mma(kt[r * P + ((2 * s + half) ^ key_turn<DP>(r))], qf[s], x[b]);
            }
    }

    // What exp makes of them.  masks: keys after `end`, counted from 4 (lane / 32), are not seen.
    __device__ __forceinline__ void weights(float scale, bool masks, int end, float lazy = kLazy) {
        if (masks) {
#pragma unroll
            for (int b = 0; b < KB; b++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (32 * b + 8 * (i >> 2) + (i & 3) > end) x[b][i] = kNegInf;
        }
        float most = kNegInf;
#pragma unroll
        for (int b = 0; b < KB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) most = fmaxf(most, x[b][i]);
        most *= scale;
        if (__ballot(passes(most, top, lazy - kLift))) {
            // row by row: what a row gives does not depend on its neighbours
            const float all = fmaxf(most, other_half(most)), now = !passes(all, top, lazy - kLift) ? top : kLift > 0.0f ? all + kLift : all;
            const float f = now == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(top - now);
            top = now;
            sum *= f;
#pragma unroll
            for (int d = 0; d < DB; d++) acc[d] *= f;
        }
        const float m = top == kNegInf ? 0.0f : top;
        if (__builtin_expect(__ballot(fabsf(m) > kFar) != 0, 0)) {      // those rows only
            const float by = fabsf(m) > kFar ? scale : 1.0f;
#pragma unroll
            for (int b = 0; b < KB; b++) x[b] *= by;
            scale = fabsf(m) > kFar ? 1.0f : scale;
        }
#pragma unroll
        for (int b = 0; b < KB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                x[b][i] = __builtin_amdgcn_exp2f(fmaf(x[b][i], scale, -m));
                sum += x[b][i];
            }
    }

    // values(r, d): keys r + 0 .. 3 and r + 8 .. 11 of element 32 d + lane % 32.
    template <typename F> __device__ __forceinline__ void products(F values) {
        const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
        for (int b = 0; b < KB; b++)
#pragma unroll
            for (int s = 0; s < 2; s++) {
                f32x8 w;
#pragma unroll
                for (int i = 0; i < 8; i++) w[i] = x[b][8 * s + i];
                const V pf = __builtin_convertvector(w, V);
#pragma unroll
                for (int d = 0; d < DB; d++) acc[d] = mma(values(32 * b + 16 * s + 4 * half, d), pf, acc[d]);
            }
    }
};

// Whether some value's scale among keys k0 .. k1 - 1 is finite and so large (from 2^56 on) that sums of values under weights
// of up to 2^kLazy can near the end of fp32: what is not finite for another reason stays so.
__device__ __forceinline__ bool large_values(const Kv4AttentionParams& p, const Rows& rw, int h, int k0, int k1) {
    const int32_t* table = p.table + rw.seq * p.table_pitch;
    bool found = false;
    k1 = min(k1, rw.len);
#pragma unroll 1
    for (int j = k0 + 4 * (threadIdx.x & 63); j < k1; j += 256) {
        const int pid = table[j >> p.cache.shift], t = j & (p.cache.page - 1);
        if (pid < 0 || pid >= p.cache.pages) continue;
        const uint8_t* run = p.cache.block(pid, h) + p.cache.value_scales_at() + p.cache.scale_run(t);
#pragma unroll 1
        for (int k = 0; k < 4 * p.cache.groups; k++) {
            const uint32_t e = ((const uint16_t*)run)[k] >> 7 & 0xff;
            found |= e >= 127 + 56 && e < 255;
        }
    }
    return __any(found);
}

// The fallback for an item over the 4-bit cache, which usual data never takes: keys k0 .. k1 - 1 for the rows from `row0` on
// that `mask` has, by one wave, in fp32 but for codes and queries: a key's scale is on the sum of its group, a value's on the
// probability, which enters as two bf16.  Maxima move at once, so that no weight is above 1.  It leaves the outputs
// (to < 0) or the item's part: the first row's place among the parts (EVEN), or the part's number.  Operands come straight
// from the cache, and the scores are formed again for every 32 elements of the output, so that a kernel's registers are
// those of its usual pass (with all accumulators at once that of kv4_prompt.hip spilled, for 8 % of its time).
template <typename T, bool EVEN>
__device__ __forceinline__ void wide_pass(const Kv4AttentionParams& p, const Rows& rw, int h, int k0, int k1, int row0, uint32_t mask, int64_t to,
                                          int chunks, float* part, float2* stats) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));      // nothing is kept from before the usual pass
    const int col = lane & 31, half = lane >> 5, C = p.cache.groups, page = p.cache.page;
    const int row = row0 + col, last = rw.len - rw.n + row / p.group, head = h * p.group + row % p.group;
    const int64_t token = rw.begin + row / p.group;
    const bool live = row < rw.rows && mask >> col & 1, whole = to < 0;
    k1 = min(k1, rw.len - rw.n + (min(row0 + 32, rw.rows) - 1) / p.group + 1);
    const int32_t* table = p.table + rw.seq * p.table_pitch;
    const T* q = (const T*)p.q.p + token * p.q.token + head * p.q.head + 8 * half;
    // key j's place in its page, from the last key on that key's; a token's run of four shares it
    struct Place {
        const uint8_t* block;
        int t;
        bool bad;
    };
    auto place = [&](int j) {
        j = min(j, k1 - 1);
        const int pid = table[j >> p.cache.shift];
        const bool bad = pid < 0 || pid >= p.cache.pages;
        return Place{p.cache.block(bad ? 0 : pid, h), j & (page - 1), bad};
    };
#pragma unroll 1
    for (int d = 0; d < C; d++) {
        Attend<_Float16, 32, 32> fl;
        fl.start();
#pragma unroll 1
        for (int j0 = k0; j0 < k1; j0 += 32) {
            fl.x[0] = f32x16{};
#pragma unroll 1
            for (int g = 0; g < C; g++) {
                const Place mine = place(j0 + col);
                const uint8_t* words = mine.block + mine.t * 16 * C + half * 4 * C + 4 * g;
                typename Vec8<T>::type q0 = {}, q1 = {};
                if (live) q0 = load8(q + 32 * g, 8), q1 = load8(q + 32 * g + 16, 8);
                f32x16 z = mma(decode(*(const uint32_t*)words, T{}), q0, f32x16{});
                z = mma(decode(*(const uint32_t*)(words + 8 * C), T{}), q1, z);
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const Place run = place(j0 + 8 * r + 4 * half);
                    f32x4 a = four(*(const uint2*)(run.block + p.cache.key_scales_at() + p.cache.scale_run(run.t) + 8 * g));
                    if (run.bad) a = f32x4{} + __builtin_nanf("");
#pragma unroll
                    for (int i = 0; i < 4; i++) fl.x[0][4 * r + i] = fmaf(a[i], z[4 * r + i], fl.x[0][4 * r + i]);
                }
            }
            fl.weights(p.scale, true, last - j0 - 4 * half, 0.0f);
#pragma unroll
            for (int s = 0; s < 2; s++) {
                // keys `at` .. + 3 and `at` + 8 .. + 11 in turn; a byte has elements 2 a and 2 a + 1 of a key
                const int at = j0 + 16 * s + 4 * half;
                uint32_t w[2];
                f32x8 pa;
#pragma unroll
                for (int r = 0; r < 2; r++) {
                    const Place run = place(at + 8 * r);
                    const uint8_t* v = run.block + p.cache.values_at() + ((run.t >> 2) * 16 + (col >> 1)) * 4 * C;
                    w[r] = *(const uint32_t*)(v + 4 * d) >> 4 * (col & 1) & 0x0f0f0f0fu;
                    const f32x4 a = four(*(const uint2*)(run.block + p.cache.value_scales_at() + p.cache.scale_run(run.t) + 8 * d));
#pragma unroll
                    for (int i = 0; i < 4; i++)      // scales behind the last key may be anything
                        pa[2 * i + r] = at + 8 * r + i > last ? 0.0f : fl.x[0][8 * s + 4 * r + i] * a[i];
                }
                const bf16x8 v = decode(w[0] | w[1] << 4, __bf16{});
                const bf16x8 hi = __builtin_convertvector(pa, bf16x8);
                const bf16x8 lo = __builtin_convertvector(pa - __builtin_convertvector(hi, f32x8), bf16x8);
                fl.acc[0] = mma(v, hi, fl.acc[0]);
                fl.acc[0] = mma(v, lo, fl.acc[0]);
            }
        }
        const float sum = fl.sum + other_half(fl.sum);
        if (!live) continue;
        const int64_t at = EVEN ? to + col : (token * p.q.heads + head) * chunks + to;
        const float f = !whole ? 1.0f : last >= 0 ? 1.0f / sum : 0.0f;
        if (!whole && half == 0 && d == 0) stats[at] = make_float2(fl.top, sum);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int e = 32 * d + 8 * k + 4 * half;
            f32x4 w;
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = fl.acc[0][4 * k + i] * f;
            if (!whole) {
                *(f32x4*)(part + at * p.d + e) = w;
            } else {
                if (rw.bad) w = f32x4{} + __builtin_nanf("");
                typedef T t4 __attribute__((ext_vector_type(4)));
                ((Loose<t4, T>*)((T*)p.o.p + token * p.o.token + head * p.o.head + e))->v = __builtin_convertvector(w, t4);
            }
        }
    }
}

}  // namespace esb
