// 4-bit weights with a scale per group: quantization, packing and unpacking.
//
// A row's reduction is cut into groups of G = 32, 64 or 128 weights, each with its own bf16 scale.
// The codes are ESB(4,1), which is OCP E2M1: value q in {0, .5, 1, 1.5, 2, 3, 4, 6} and a sign.
// The scale of a group is the aligner's search (eq. (9), (13)) on that group: candidates
//   alpha_j = bf16(max(fl32(max|w| f_j) / 6, 2^-126)),
// the one of the least sum of (w - alpha_j q)^2, the lowest index on ties.  A bf16 scale makes the
// cell bounds mid * alpha exact in fp32 (3 + 8 bits), so codes are the exact nearest values of
// w / alpha, ties to the larger magnitude, with no division.
//
// Layout (w4_layout): what a wave of the products reads per step is contiguous.  Tiles of 32 rows x
// 64 columns, 1 KB each, [row tile][column chunk]; lane 32h + r of a tile owns row r and 16 bytes,
// words i of eight columns 8b .. 8b+7, b = 2h + i % 2 + 4 (i / 2) (lowest nibble first), in the order
// i = 0, 2, 1, 3.
//  * Word i of the 64 lanes is the operand of one 32x32x16 MFMA, words 0 and 1 (2 and 3) of the two
//    over columns 0 .. 31 (32 .. 63);
//  * the low or high half of the 16 bytes of 16 rows, lane 16(2h + e) + r, are words e and 2 + e:
//    operands of two 16x16x32 MFMAs over columns 0 .. 31 and 32 .. 63.
// So every MFMA stays within one group of 32, 64 or 128.  The scales follow, [row tile][group][32
// rows].  Rows and columns beyond N and K hold codes and scales of 0.
#include <type_traits>

#include "float_rows.h"

namespace esb {

namespace {

constexpr float kTiny = 0x1p-126f;

__device__ __forceinline__ float bf16_round(float x) { return (float)(__bf16)x; }

// Number of cell bounds of alpha at or below |w|: the E2M1 code of the magnitude.
__device__ __forceinline__ int magnitude_code(float aw, float alpha) {
    return (aw >= 0.25f * alpha) + (aw >= 0.75f * alpha) + (aw >= 1.25f * alpha) +
           (aw >= 1.75f * alpha) + (aw >= 2.5f * alpha) + (aw >= 3.5f * alpha) + (aw >= 5.0f * alpha);
}
__device__ __forceinline__ float code_value(int c) {
    return c < 2 ? 0.5f * (float)c : __uint_as_float(((uint32_t)(126 + (c >> 1)) << 23) | ((uint32_t)(c & 1) << 22));
}

// Owner of the weights in the kernels below: a wave takes two adjacent tiles (128 columns, one
// group of 128), lane 32h + r of it words i of both tiles (word 4u + i) of row r.
struct Owner {
    int r, h, nt, kc;    // row and half in the tile, row tile, first chunk
    int64_t n;
};
__device__ __forceinline__ bool own(const W4Layout& L, Owner* o) {
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int pairs = (L.chunks + 1) / 2;
    if (wave >= (int64_t)L.tiles * pairs) return false;
    o->r = lane & 31;
    o->h = lane >> 5;
    o->nt = (int)(wave / pairs);
    o->kc = 2 * (int)(wave % pairs);
    o->n = 32 * (int64_t)o->nt + o->r;
    return true;
}
__device__ __forceinline__ int column(const Owner& o, int word) {
    return 64 * (o.kc + (word >> 2)) + 8 * (2 * o.h + (word & 1) + 4 * ((word >> 1) & 1));
}
// The lane's eight words into the two tiles.
__device__ __forceinline__ void put_tiles(const W4Layout& L, const Owner& o, const uint32_t (&w)[8], uint8_t* out) {
#pragma unroll
    for (int u = 0; u < 2; u++)
        if (o.kc + u < L.chunks)
            *(uint4*)(out + 1024 * ((int64_t)o.nt * L.chunks + o.kc + u) + 16 * (32 * o.h + o.r)) =
                uint4{w[4 * u], w[4 * u + 2], w[4 * u + 1], w[4 * u + 3]};
}
__device__ __forceinline__ int64_t scale_index(const W4Layout& L, const Owner& o, int g) {
    return ((int64_t)o.nt * L.groups + g) * 32 + o.r;
}

// The quantizer's lanes hold one group's words of a row and half h: two for groups of 32 and four (32
// weights) else; two lanes to a group, four for groups of 128.  For groups of 64 a wave takes a tile,
// else half of the rows (blockIdx.y) of a tile's two groups or of two tiles.
template <int G>
struct Share {
    static constexpr int words = G == 32 ? 2 : 4;
    int r, h, nt, kc, gi;    // row and half in the tile, row tile, chunk and group of this lane
    int64_t n;
    static __host__ __device__ int across(const W4Layout& L) { return G == 128 ? (L.chunks + 1) / 2 : L.chunks; }
    __device__ __forceinline__ bool own(const W4Layout& L) {
        const int lane = threadIdx.x & 63;
        const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
        const int per = across(L), e = lane >> 4 & 1;
        if (wave >= (int64_t)L.tiles * per) return false;
        const int q = (int)(wave % per);
        nt = (int)(wave / per);
        r = G == 64 ? lane & 31 : 16 * (int)blockIdx.y + (lane & 15);
        kc = G == 128 ? 2 * q + e : q;
        gi = G == 32 ? 2 * q + e : q;
        h = lane >> 5;
        n = 32 * (int64_t)nt + r;
        return true;
    }
    __device__ __forceinline__ int column(int i) const {
        return 64 * kc + 8 * (2 * h + (i & 1) + 4 * (G == 32 ? gi & 1 : i >> 1));
    }
    __device__ __forceinline__ void put(const W4Layout& L, const uint32_t (&w)[words], uint8_t* out) const {
        if (kc >= L.chunks) return;
        uint8_t* d = out + 1024 * ((int64_t)nt * L.chunks + kc) + 16 * (32 * h + r);
        if constexpr (G == 32) {
            *(uint32_t*)(d + 4 * (gi & 1)) = w[0];
            *(uint32_t*)(d + 4 * (gi & 1) + 8) = w[1];
        } else {
            *(uint4*)d = uint4{w[0], w[2], w[1], w[3]};
        }
    }
};
// Over the lanes of a row.
template <int G, typename F>
__device__ __forceinline__ uint32_t over_row(uint32_t v, F f) {
    auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = f(s[0], s[1]);
    if (G == 128) {
        s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = f(s[0], s[1]);
    }
    return v;
}
template <int G>
__device__ __forceinline__ float row_sum(float v) {
    return __uint_as_float(over_row<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

template <int G>
__device__ __forceinline__ double row_sum(double v) {
    v += __shfl_xor(v, 32);
    if (G == 128) v += __shfl_xor(v, 16);
    return v;
}

// One group of a row's lanes, in any range of values: errors in fp64 from exact cell bounds.  Rare: it
// reads the group's weights again rather than keep them.
template <typename T, int G>
__device__ __forceinline__ float search_exact(const Share<G>& o, const T* row, int K, float top,
                                              const float* factors, int nf) {
    float alpha = __builtin_nanf("");
    double least = __builtin_inf();
    for (int c = 0; c < nf; c++) {
        const float f = factors ? factors[c] : 1.0f;
        const float a = bf16_round(fmaxf(top * f / 6.0f, kTiny));
        if (!(f > 0.0f) || !(f < __builtin_inff())) continue;
        double err = 0.0;
#pragma unroll 1
        for (int t = 0; t < o.words; t++) {
            const int k = o.column(t);
            const f32x8 x = __builtin_convertvector(load8(row + k, K - k), f32x8);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float aw = fabsf(x[i]);
                const double e = (double)aw - (double)a * (double)code_value(magnitude_code(aw, a));
                err += e * e;
            }
        }
        err = row_sum<G>(err);
        if (a < __builtin_inff() && err < least) {
            least = err;
            alpha = a;
        }
    }
    return alpha;
}

// Squared error of one lane's weights n under scale a, fp64 from exact cell bounds.
template <int WG>
__device__ __forceinline__ double exact_error(const float* n, float a) {
    double err = 0.0;
#pragma unroll
    for (int i = 0; i < 8 * WG; i++) {
        const float aw = fabsf(n[i]);
        const double e = (double)aw - (double)a * (double)code_value(magnitude_code(aw, a));
        err += e * e;
    }
    return err;
}
// Eight values to E2M1 nibbles, rounded to nearest even, at most 6.
__device__ __forceinline__ uint32_t to_e2m1(const float* x, float by) {
    uint32_t q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0] * by, x[1] * by, 1.0f, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[2] * by, x[3] * by, 1.0f, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[4] * by, x[5] * by, 1.0f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[6] * by, x[7] * by, 1.0f, 3);
}

// The search needs no exact codes: the error is continuous where a code changes, so a candidate's q is
// the conversion to fp4 of w (1/alpha), and e = w - alpha q one fma.  The group is scaled by a power of
// two that brings its largest weight into [1, 2), which keeps e^2 in range.  An error's sum is off by
//  * 11 roundings of 2^-24: two in the square of a rounded e, nine sums on a square's way (four in its
//    lane's part, three over the parts, two over the lanes of a row);
//  * for 32-bit weights, q on the wrong side of a bound: 1/alpha is within 2^-23 and the product rounded,
//    so |w| is then within 1.5 2^-23 of mid alpha (relative), and its square above the least one by up to
//    28 times that (8 mid / gap, the most at 1.75 and 3.5), 2^-17.6.  16-bit weights are on a bound, where
//    both squares are equal, or 2^-11 away.
// So where the second least is within kNear of the least (a few groups in ten thousand, in a thousand for
// 32-bit weights), the two are compared in fp64: kNear is above twice the first part plus the second.
// Three candidates so close, or candidates far below the weights, are left to search_exact.
//
// Codes: for 16-bit weights w / alpha is a tie or at least 2^-11 from one, so w (1/alpha) (1 + 2^-22)
// rounds to the nearest value with ties up; 32-bit weights are compared with the exact bounds.
//
// Bound by VALU issue (97 % of all cycles busy): for two weights and a candidate two products with 1/alpha,
// a conversion to fp4 (a quarter of the fp32 rate), one back, two remainders and two squares, some 22
// cycles of a SIMD per 64 weights.  4096 x 9216 bf16 weights, G = 128, 16 candidates: 101-110 us (the
// bytes alone: 18), fp32 weights 114 (bytes: 33); 1000 x 1999 fp16, G = 32, 8 candidates: 9 us (11 with both groups in a lane).
// Dot products of 16-bit pairs would halve the sums but lose seven bits to cancellation, and fp4 from
// 16-bit products moves the cell bounds: both would send groups by the percent, not by the
// ten-thousand, to the fp64 comparison.
template <typename T> constexpr float kNear = sizeof(T) == 4 ? 0x1p-17f : 0x1p-19f;

template <typename T, int G>
__global__ __launch_bounds__(256) void k_w4_quantize(W4Layout L, const T* __restrict__ w, int64_t ldw,
                                                     const float* __restrict__ factors, int nf,
                                                     uint8_t* __restrict__ out) {
    Share<G> o;
    if (!o.own(L)) return;
    constexpr int WG = Share<G>::words;
    const int lane = threadIdx.x & 63;
    const float fs = factors && lane < nf ? factors[lane] : 1.0f;
    float n[8 * WG];
#pragma unroll
    for (int t = 0; t < WG; t++) {
        const int k = o.column(t);
        const f32x8 x = __builtin_convertvector(load8(w + o.n * ldw + k, o.n < L.N ? L.K - k : 0), f32x8);
#pragma unroll
        for (int i = 0; i < 8; i++) n[8 * t + i] = x[i];
    }
    uint32_t packed[WG];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8 * WG; i++) m = max(m, __float_as_uint(n[i]) & 0x7fffffffu);
    m = over_row<G>(m, [](uint32_t a, uint32_t b) { return max(a, b); });
    const float top = __uint_as_float(m);
    const bool finite = m < 0x7f800000u;

    // 2^-shift brings the largest weight into [1, 2)
    const int shift = finite && m ? __builtin_amdgcn_frexp_expf(top) - 1 : 0;
#pragma unroll
    for (int i = 0; i < 8 * WG; i++) n[i] = finite ? __builtin_amdgcn_ldexpf(n[i], -shift) : 0.0f;
    const float inf = __builtin_inff();
    float alpha = __builtin_nanf(""), other = alpha, least = inf, second = inf, third = inf;
    bool far = false, other_first = false;
    for (int c = 0; c < nf; c++) {
        const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(fs), c));
        if (!(f > 0.0f) || !(f < __builtin_inff())) continue;
        // x / 6 rounded correctly: the product with the reciprocal, corrected by its exact remainder
        const float x6 = top * f, q6 = x6 * (1.0f / 6.0f), d6 = fmaf(fmaf(-6.0f, q6, x6), 1.0f / 6.0f, q6);
        const float a = bf16_round(fmaxf(d6, kTiny));
        const float as = m ? __builtin_amdgcn_ldexpf(a, -shift) : 1.0f;
        const float inv = __builtin_amdgcn_rcpf(as);
        far |= as < 0x1p-100f;
        float sum[8] = {};
#pragma unroll
        for (int t = 0; t < WG; t++) {
            const float* x = n + 8 * t;
            const uint32_t q = to_e2m1(x, inv);
            const auto d0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0);
            const auto d1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1);
            const auto d2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2);
            const auto d3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3);
            const float d[8] = {d0[0], d0[1], d1[0], d1[1], d2[0], d2[1], d3[0], d3[1]};
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float e = fmaf(-as, d[i], x[i]);
                sum[i] = fmaf(e, e, sum[i]);
            }
        }
        float err = row_sum<G>(((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7])));
        // a candidate that overflows is passed over; one equal to a kept one adds nothing
        err = x6 < inf && a != alpha && a != other ? err : inf;
        const bool first = err < least, next = err < second;
        other = first ? alpha : next ? a : other;
        other_first = first || (other_first && !next);
        alpha = first ? a : alpha;
        third = fminf(third, fmaxf(second, err));
        second = __builtin_amdgcn_fmed3f(least, second, err);
        least = fminf(least, err);
    }
    const float near = least * (1.0f + kNear<T>);
    if (__any(finite && m && (far || third <= near))) {
        const float exact = search_exact<T, G>(o, w + (o.n < L.N ? o.n : 0) * ldw, o.n < L.N ? L.K : 0, top, factors, nf);
        if (finite) alpha = exact;
    } else if (__any(finite && m && second <= near)) {
        const double e0 = row_sum<G>(exact_error<WG>(n, __builtin_amdgcn_ldexpf(alpha, -shift)));
        const double e1 = row_sum<G>(exact_error<WG>(n, __builtin_amdgcn_ldexpf(other, -shift)));
        if (second <= near && (other_first ? e1 <= e0 : e1 < e0)) alpha = other;
    }
    if (!finite) alpha = __builtin_nanf("");
    const float as = __builtin_amdgcn_ldexpf(alpha, -shift);

    // (1/as) of a scale far below the weights may be infinite
    if (sizeof(T) == 2 && !__any(finite && m && as < 0x1p-100f)) {
        const float inv = m && alpha == alpha ? 1.0f / as * (1.0f + 0x1p-22f) : 0.0f;
#pragma unroll
        for (int t = 0; t < WG; t++) {
            const uint32_t q = to_e2m1(n + 8 * t, inv);
            // zeros without a sign: bit 3 stays where a magnitude bit is set
            packed[t] = q & (0x77777777u | ((q & 0x77777777u) + 0x77777777u));
        }
    } else {
#pragma unroll
        for (int t = 0; t < WG; t++) {
            uint32_t d = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float x = __builtin_amdgcn_ldexpf(n[8 * t + i], shift);
                const uint32_t c = (uint32_t)magnitude_code(fabsf(x), alpha);
                d |= (c | (c && x < 0.0f ? 8u : 0u)) << (4 * i);
            }
            packed[t] = d;
        }
    }
    if (o.h == 0 && (G < 128 || o.kc % 2 == 0))
        ((__bf16*)(out + L.scale_offset))[((int64_t)o.nt * L.groups + o.gi) * 32 + o.r] =
            o.n < L.N && (int64_t)o.gi * G < L.K ? (__bf16)alpha : (__bf16)0.0f;
    o.put(L, packed, out);
}

// Four ESB(4,1) codes, one a byte, to E2M1 nibbles in the bytes 0 and 2: one more in the exponent field,
// modulo 4, takes the all-ones (subnormal) binade to 0; zero has no sign.
__device__ __forceinline__ uint32_t code_nibbles(uint32_t c) {
    const uint32_t m = ((c & 0x07070707u) + 0x02020202u) & 0x07070707u;
    const uint32_t n = m | (c & (m + 0x07070707u) & 0x08080808u);
    return n | (n >> 4);
}

// ESB(4,1) codes and row-major scales into the layout: a byte in, half a byte out, bound by HBM (18432 x
// 4096: 27 us, 4.3 TB/s; loading and packing byte by byte took 190).
__global__ __launch_bounds__(256) void k_w4_pack(W4Layout L, const uint8_t* __restrict__ codes, int64_t ldc,
                                                 const __bf16* __restrict__ alpha, int64_t lda,
                                                 uint8_t* __restrict__ out) {
    Owner o;
    if (!own(L, &o)) return;
    uint32_t packed[8];
#pragma unroll
    for (int t = 0; t < 8; t++) {
        const int k = column(o, t);
        uint2 c = {0x06060606u, 0x06060606u};            // codes of zero
        const uint8_t* src = codes + o.n * ldc + k;
        if (o.n < L.N && k + 8 <= L.K) {
            c = ((const Loose<uint2, uint8_t>*)src)->v;
        } else if (o.n < L.N) {
            uint32_t v[2] = {c.x, c.y};
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (k + i < L.K) v[i >> 2] ^= (uint32_t)(src[i] ^ 6) << (8 * (i & 3));
            c = uint2{v[0], v[1]};
        }
        packed[t] = __builtin_amdgcn_perm(code_nibbles(c.y), code_nibbles(c.x), 0x06040200u);
    }
    put_tiles(L, o, packed, out);
    __bf16* scales = (__bf16*)(out + L.scale_offset);
    if (o.h) return;
    const int g0 = 64 * o.kc / L.group, per = 128 / L.group;
    for (int g = g0; g < g0 + per && g < L.groups; g++)
        scales[scale_index(L, o, g)] = o.n < L.N && (int64_t)g * L.group < L.K ? alpha[o.n * lda + g] : (__bf16)0.0f;
}

// Unscaled values as E4M3 bytes, and row-major scales; bound by HBM (18432 x 4096: 22.6 us, 5.1 TB/s).
__global__ __launch_bounds__(256) void k_w4_unpack(W4Layout L, const uint8_t* __restrict__ in,
                                                   uint8_t* __restrict__ values, int64_t ldv,
                                                   __bf16* __restrict__ alpha, int64_t lda) {
    Owner o;
    if (!own(L, &o) || o.n >= L.N) return;
    if (values) {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            if (o.kc + u >= L.chunks) break;
            const uint4 p = *(const uint4*)(in + 1024 * ((int64_t)o.nt * L.chunks + o.kc + u) + 16 * (32 * o.h + o.r));
            const uint32_t packed[4] = {p.x, p.z, p.y, p.w};
#pragma unroll
            for (int t = 0; t < 4; t += 2) {        // two words are 16 adjacent columns
                uint32_t q[4];
#pragma unroll
                for (int d = 0; d < 2; d++) {
                    // the eight magnitudes as E4M3 bytes, picked by v_perm_b32
                    const uint32_t ev = packed[t + d] & 0x0f0f0f0fu, od = (packed[t + d] >> 4) & 0x0f0f0f0fu;
                    const uint32_t be = __builtin_amdgcn_perm(0x4c484440u, 0x3c383000u, ev & 0x07070707u) | ((ev & 0x08080808u) << 4);
                    const uint32_t bo = __builtin_amdgcn_perm(0x4c484440u, 0x3c383000u, od & 0x07070707u) | ((od & 0x08080808u) << 4);
                    q[2 * d] = __builtin_amdgcn_perm(bo, be, 0x05010400u);
                    q[2 * d + 1] = __builtin_amdgcn_perm(bo, be, 0x07030602u);
                }
                const int k = column(o, 4 * u + t);
                uint8_t* dst = values + o.n * ldv + k;
                if (L.K - k >= 16) {
                    ((Loose<uint4, uint8_t>*)dst)->v = uint4{q[0], q[1], q[2], q[3]};
                } else {
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        if (k + i < L.K) dst[i] = (uint8_t)(q[i >> 2] >> (8 * (i & 3)));
                }
            }
        }
    }
    if (!alpha || o.h) return;
    const __bf16* scales = (const __bf16*)(in + L.scale_offset);
    const int g0 = 64 * o.kc / L.group, per = 128 / L.group;
    for (int g = g0; g < g0 + per && (int64_t)g * L.group < L.K; g++) alpha[o.n * lda + g] = scales[scale_index(L, o, g)];
}

unsigned tile_blocks(const W4Layout& L) {   // a wave per two chunks
    return (unsigned)(((int64_t)L.tiles * ((L.chunks + 1) / 2) + 3) / 4);
}

template <typename T>
hipError_t quantize_t(const W4Layout& L, const void* w, int64_t ldw, const float* f, int nf, void* out,
                      hipStream_t s) {
    auto go = [&](auto group, auto kernel) {
        constexpr int G = decltype(group)::value;
        const int64_t waves = (int64_t)L.tiles * Share<G>::across(L);
        kernel<<<dim3((unsigned)((waves + 3) / 4), G == 64 ? 1 : 2), 256, 0, s>>>(L, (const T*)w, ldw, f, nf, (uint8_t*)out);
    };
    if (L.group == 32) go(std::integral_constant<int, 32>(), k_w4_quantize<T, 32>);
    else if (L.group == 64) go(std::integral_constant<int, 64>(), k_w4_quantize<T, 64>);
    else go(std::integral_constant<int, 128>(), k_w4_quantize<T, 128>);
    return hipGetLastError();
}

}  // namespace

W4Layout w4_layout(int N, int K, int group) {
    W4Layout L;
    L.N = N;
    L.K = K;
    L.group = group;
    L.tiles = (int)(((int64_t)N + 31) / 32);
    L.chunks = (int)(((int64_t)K + 63) / 64);
    L.groups = (int)((64 * (int64_t)L.chunks + group - 1) / group);
    L.scale_offset = (int64_t)L.tiles * L.chunks * 1024;
    L.bytes = L.scale_offset + (int64_t)L.tiles * L.groups * 64;
    return L;
}

hipError_t launch_w4_quantize(const W4Layout& L, int type, const void* w, int64_t ldw, const float* factors,
                              int nf, void* out, hipStream_t s) {
    if (type == kF32) return quantize_t<float>(L, w, ldw, factors, nf, out, s);
    if (type == kBF16) return quantize_t<__bf16>(L, w, ldw, factors, nf, out, s);
    return quantize_t<_Float16>(L, w, ldw, factors, nf, out, s);
}

hipError_t launch_w4_pack(const W4Layout& L, const uint8_t* codes, int64_t ldc, const void* alpha, int64_t lda,
                          void* out, hipStream_t s) {
    k_w4_pack<<<tile_blocks(L), 256, 0, s>>>(L, codes, ldc, (const __bf16*)alpha, lda, (uint8_t*)out);
    return hipGetLastError();
}

hipError_t launch_w4_unpack(const W4Layout& L, const void* in, uint8_t* values, int64_t ldv, void* alpha,
                            int64_t lda, hipStream_t s) {
    k_w4_unpack<<<tile_blocks(L), 256, 0, s>>>(L, (const uint8_t*)in, values, ldv, (__bf16*)alpha, lda);
    return hipGetLastError();
}

}  // namespace esb
