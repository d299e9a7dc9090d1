// One pass of softmax attention over tiles of keys in LDS, as attention.hip and kv4_prompt.hip share it: 32 rows
// (queries x heads) to a wave, on 32x32x16 MFMAs, with a running maximum and sum.
#pragma once

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
    V qf[DP / 16];       // elements 16 s + 8 (lane / 32) .. + 7 of the row
    f32x16 acc[DB], x[KB];
    float top, sum;      // the running maximum (times scale), and the lane's part of the sum

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
        if (__ballot(passes(most, top, lazy))) {
            // row by row: what a row gives does not depend on its neighbours
            const float all = fmaxf(most, other_half(most)), now = passes(all, top, lazy) ? all : top;
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

}  // namespace esb
