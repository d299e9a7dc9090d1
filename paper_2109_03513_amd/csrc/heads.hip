// Heads of queries, keys and values on their way into attention, one pass over each:
//
//  * the norm over a head and the rotation of its first `rot` elements: y = x rstd w,
//    rstd = 1 / sqrt(mean x^2 + eps); pairs (a, b) become (a c - b s, b c + a s), c and s from the
//    table's row of the token's position;
//  * keys (normed and rotated so) and values into the 4-bit cache, with alpha = bf16(max|y| / 6) per
//    32 elements and the nearest of the eight magnitudes to |y| / alpha, ties to the larger.
//
// A head has d / 8 lanes (8, 16, 32 or 64 by d), eight elements each; the partners of a rotation are
// read from the head again, which its cache lines still hold, so nothing crosses lanes but
// the sum of squares and the group's maximum.
//
// Keys for the cache are computed in fp64 and rounded once to fp32 before they get their codes: the
// same call gives the same codes wherever the borders lie.  esb_rope computes in fp32 around an fp64
// sum of squares, which does not overflow.
#include "kv4.h"

namespace esb {

namespace {

constexpr float kTiny = 0x1p-126f;

__device__ __forceinline__ float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

__device__ __forceinline__ float root(float x) { return sqrtf(x); }
__device__ __forceinline__ double root(double x) { return sqrt(x); }

// Where elements e .. e + 7 of a token of a block are.
__device__ __forceinline__ uint32_t* key_word(const Kv4Layout& L, uint8_t* b, int t, int e) {
    return (uint32_t*)(b + (int64_t)t * 16 * L.groups + ((e >> 3) & 3) * 4 * L.groups + (e >> 5) * 4);
}
// Byte of elements e, e + 1; the next pairs' are 4 groups bytes apart.
__device__ __forceinline__ uint8_t* value_byte(const Kv4Layout& L, uint8_t* b, int t, int e) {
    return b + L.values_at() + (int64_t)(t >> 2) * 64 * L.groups + ((e >> 1) & 15) * 4 * L.groups + (e >> 5) * 4 +
           (t & 3);
}
__device__ __forceinline__ uint16_t* scale_at(const Kv4Layout& L, uint8_t* b, int region, int t, int g) {
    return (uint16_t*)(b + region + L.scale_run(t) + g * 8 + (t & 3) * 2);
}

// Eight nibbles (and, by the first lane of four, the group's scale) of one token into its block.
template <bool KEY>
__device__ __forceinline__ void store_codes(const Kv4Layout& L, uint8_t* b, int t, int e, uint32_t w, uint16_t alpha) {
    if (KEY) {
        *key_word(L, b, t, e) = w;
    } else {
        uint8_t* o = value_byte(L, b, t, e);
#pragma unroll
        for (int i = 0; i < 4; i++) o[i * 4 * L.groups] = (uint8_t)(w >> (8 * i));
    }
    if ((e & 31) == 0) *scale_at(L, b, KEY ? L.key_scales_at() : L.value_scales_at(), t, e >> 5) = alpha;
}

// Codes of eight elements of a group that four neighbouring lanes share.
struct Codes {
    uint32_t nibbles;
    uint16_t alpha;
};
__device__ __forceinline__ Codes quantize(f32x8 y) {
    uint32_t m = 0;      // max |y| on bit patterns: a NaN is above every number
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(y[i]) & 0x7fffffffu);
    m = max(m, (uint32_t)__shfl_xor((int)m, 1));
    m = max(m, (uint32_t)__shfl_xor((int)m, 2));
    if (m >= 0x7f800000u) return {0, 0x7fc0};
    const __bf16 a16 = (__bf16)fmaxf(__uint_as_float(m) / 6.0f, kTiny);
    const float a = (float)a16;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float v = fabsf(y[i]);
        // the borders are exact in fp32: three bits times eight
        const uint32_t c = (v >= 0.25f * a) + (v >= 0.75f * a) + (v >= 1.25f * a) + (v >= 1.75f * a) +
                           (v >= 2.5f * a) + (v >= 3.5f * a) + (v >= 5.0f * a);
        w |= (c | (y[i] < 0.0f && c ? 8u : 0u)) << (4 * i);
    }
    return {w, __builtin_bit_cast(uint16_t, a16)};
}

template <typename T>
__device__ __forceinline__ const T* head_at(const HeadsView& v, int64_t t, int h) {
    return (const T*)v.p + t * v.token + h * v.head;
}

template <typename T, typename A, int LPR, bool CACHE>
__global__ __launch_bounds__(256) void k_heads(HeadsParams p, int64_t token0, uint32_t rows) {
    typedef A a8 __attribute__((ext_vector_type(8)));
    typedef typename Vec8<T>::type V;
    const uint32_t row = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    if (row >= rows) return;
    const uint32_t nq = p.q.heads, nk = p.k.heads, all = nq + nk + (CACHE ? p.v.heads : 0);
    const int64_t t = token0 + row / all;
    int h = row % all;
    const int kind = h < (int)nq ? 0 : h < (int)(nq + nk) ? 1 : 2;
    h -= kind == 0 ? 0 : kind == 1 ? nq : nq + nk;
    const T* x = head_at<T>(kind == 0 ? p.q : kind == 1 ? p.k : p.v, t, h);
    const int d = p.d, e = 8 * (threadIdx.x % LPR), n = d - e;
    const bool in = n > 0;
    a8 y = in ? __builtin_convertvector(load8(x + e, n), a8) : a8{};
    if (kind < 2) {
        const float* w = p.eps > 0.0f ? (kind == 0 ? p.qw : p.kw) : nullptr;
        A rstd = 1;
        if (p.eps > 0.0f) {
            double ss = 0.0;
#pragma unroll
            for (int i = 0; i < 8; i++) ss = fma((double)y[i], (double)y[i], ss);
#pragma unroll
            for (int o = 1; o < LPR; o <<= 1) ss += __shfl_xor(ss, o);
            rstd = (A)(1.0 / sqrt(ss / (double)d + (double)p.eps));
            y *= rstd;
            if (w && in) y *= __builtin_convertvector(load8(w + e, n), a8);
        }
        if (p.rot) {
            const int64_t pos = p.positions[t];
            const int rot = p.rot, half = rot >> 1;
            if (pos < 0 || pos >= p.rows) {
                y = a8{} + (A)__builtin_nan("");
            } else if (in && e < rot) {
                const float* c = p.table + pos * rot;
                if (p.adjacent) {
#pragma unroll
                    for (int i = 0; i < 8; i += 2)
                        if (e + i < rot) {
                            const A co = c[(e + i) >> 1], si = c[half + ((e + i) >> 1)], a = y[i], b = y[i + 1];
                            y[i] = fma(a, co, -(b * si));
                            y[i + 1] = fma(b, co, a * si);
                        }
                } else if ((half & 7) == 0) {
                    const bool low = e < half;
                    const int at = low ? e : e - half, other = low ? e + half : at;
                    a8 z = __builtin_convertvector(load8(x + other, 8), a8) * rstd;
                    if (w) z *= __builtin_convertvector(load8(w + other, 8), a8);
                    const f32x8 co = load8(c + at, 8), si = load8(c + half + at, 8);
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const A s = low ? -(A)si[i] : (A)si[i];
                        y[i] = fma(y[i], (A)co[i], z[i] * s);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        if (e + i < rot) {
                            const bool low = e + i < half;
                            const int at = low ? e + i : e + i - half, other = low ? e + i + half : at;
                            A z = (A)x[other] * rstd;
                            if (w) z *= (A)w[other];
                            const A s = low ? -(A)c[half + at] : (A)c[half + at];
                            y[i] = fma(y[i], (A)c[at], z * s);
                        }
                }
            }
        }
    }
    const f32x8 r = __builtin_convertvector(y, f32x8);
    if (!CACHE || kind == 0) {
        const HeadsView& o = kind == 0 ? p.qo : p.ko;
        if (in) store8((T*)head_at<T>(o, t, h) + e, __builtin_convertvector(r, V), n);
        return;
    }
    const Codes q = quantize(r);
    const int64_t slot = p.slots[t];
    if (!in || slot < 0 || (slot >> p.cache.shift) >= p.cache.pages) return;
    uint8_t* b = p.cache.block(slot >> p.cache.shift, h);
    const int at = (int)slot & (p.cache.page - 1);
    if (kind == 1) store_codes<true>(p.cache, b, at, e, q.nibbles, q.alpha);
    else store_codes<false>(p.cache, b, at, e, q.nibbles, q.alpha);
}

// ESB(4,1) codes 0 .. 7 are 1, 1.5, 2, 3, 4, 6, 0, 0.5: E2M1's order turned by two.
__global__ __launch_bounds__(256) void k_pack(Kv4Layout L, int64_t items, const int64_t* slots, const uint8_t* k,
                                              const uint16_t* ka, const uint8_t* v, const uint16_t* va) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= items) return;
    const int pieces = 4 * L.groups, e = 8 * (int)(id % pieces);
    const int64_t row = id / pieces;      // token and head
    const int h = (int)(row % L.heads);
    const int64_t slot = slots[row / L.heads];
    if (slot < 0 || (slot >> L.shift) >= L.pages) return;
    uint8_t* b = L.block(slot >> L.shift, h);
    const int at = (int)slot & (L.page - 1);
    auto word = [&](const uint8_t* codes) {
        const uint8_t* c = codes + row * 32 * L.groups + e;
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t m = (c[i] + 2u) & 7u;
            w |= (m | (m ? c[i] & 8u : 0u)) << (4 * i);
        }
        return w;
    };
    const int64_t s = row * L.groups + (e >> 5);
    store_codes<true>(L, b, at, e, word(k), ka[s]);
    store_codes<false>(L, b, at, e, word(v), va[s]);
}

__global__ __launch_bounds__(256) void k_unpack(Kv4Layout L, int64_t items, const int64_t* slots, uint8_t* k,
                                                uint16_t* ka, uint8_t* v, uint16_t* va) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= items) return;
    const int pieces = 4 * L.groups, e = 8 * (int)(id % pieces);
    const int64_t row = id / pieces, s = row * L.groups + (e >> 5);
    const int64_t slot = slots[row / L.heads];
    const bool there = slot >= 0 && (slot >> L.shift) < L.pages;
    uint8_t* b = there ? L.block(slot >> L.shift, (int)(row % L.heads)) : nullptr;
    const int at = (int)slot & (L.page - 1);
    auto bytes = [](uint32_t w) {       // eight nibbles to eight E4M3 bytes
        f32x8 f;
        const auto put = [&](int i, auto pair) { f[i] = pair[0], f[i + 1] = pair[1]; };
        put(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0));
        put(2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1));
        put(4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2));
        put(6, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3));
        return to_e4m3(f);
    };
    if (k) ((Loose<uint2, uint8_t>*)(k + row * 32 * L.groups + e))->v = bytes(there ? *key_word(L, b, at, e) : 0u);
    if (v) {
        uint32_t w = 0;
        if (there) {
            const uint8_t* c = value_byte(L, b, at, e);
#pragma unroll
            for (int i = 0; i < 4; i++) w |= (uint32_t)c[i * 4 * L.groups] << (8 * i);
        }
        ((Loose<uint2, uint8_t>*)(v + row * 32 * L.groups + e))->v = bytes(w);
    }
    if (e & 31) return;
    if (ka) ka[s] = there ? *scale_at(L, b, L.key_scales_at(), at, e >> 5) : (uint16_t)0x7fc0;
    if (va) va[s] = there ? *scale_at(L, b, L.value_scales_at(), at, e >> 5) : (uint16_t)0x7fc0;
}

template <typename T, typename A, int LPR, bool CACHE>
hipError_t launch_n(const HeadsParams& p, hipStream_t s) {
    const int64_t all = (int64_t)p.q.heads + p.k.heads + (CACHE ? p.v.heads : 0);
    const int64_t most = ((int64_t)1 << 28) / all;      // tokens of one launch
    for (int64_t t = 0; t < p.tokens; t += most) {
        const uint32_t rows = (uint32_t)((p.tokens - t < most ? p.tokens - t : most) * all);
        constexpr int per = 256 / LPR;
        k_heads<T, A, LPR, CACHE><<<(rows + per - 1) / per, 256, 0, s>>>(p, t, rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, typename A, bool CACHE>
hipError_t launch_t(const HeadsParams& p, hipStream_t s) {
    if (p.d <= 64) return launch_n<T, A, 8, CACHE>(p, s);
    if (p.d <= 128) return launch_n<T, A, 16, CACHE>(p, s);
    if (p.d <= 256) return launch_n<T, A, 32, CACHE>(p, s);
    return launch_n<T, A, 64, false>(p, s);      // rope only: caches hold heads of at most 256
}

// Launches of pieces of eight elements, in parts that a grid can hold.
template <typename F>
hipError_t in_parts(const Kv4Layout& L, int64_t tokens, F f) {
    const int64_t per = (int64_t)L.heads * 4 * L.groups, most = ((int64_t)1 << 30) / per;
    for (int64_t t = 0; t < tokens; t += most) {
        const int64_t n = tokens - t < most ? tokens - t : most;
        f(t, n * per, (unsigned)((n * per + 255) / 256));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_rope(int type, const HeadsParams& p, hipStream_t s) {
    if (type == kF32) return launch_t<float, float, false>(p, s);
    if (type == kBF16) return launch_t<__bf16, float, false>(p, s);
    return launch_t<_Float16, float, false>(p, s);
}

hipError_t launch_kv4_append(int type, const HeadsParams& p, hipStream_t s) {
    if (type == kF32) return launch_t<float, double, true>(p, s);
    if (type == kBF16) return launch_t<__bf16, double, true>(p, s);
    return launch_t<_Float16, double, true>(p, s);
}

hipError_t launch_kv4_pack(const Kv4Layout& L, int64_t tokens, const int64_t* slots, const uint8_t* k,
                           const void* ka, const uint8_t* v, const void* va, hipStream_t s) {
    return in_parts(L, tokens, [&](int64_t t, int64_t items, unsigned grid) {
        const int64_t c = t * L.heads * 32 * L.groups, a = t * L.heads * L.groups;
        k_pack<<<grid, 256, 0, s>>>(L, items, slots + t, k + c, (const uint16_t*)ka + a, v + c,
                                    (const uint16_t*)va + a);
    });
}

hipError_t launch_kv4_unpack(const Kv4Layout& L, int64_t tokens, const int64_t* slots, uint8_t* k, void* ka,
                             uint8_t* v, void* va, hipStream_t s) {
    return in_parts(L, tokens, [&](int64_t t, int64_t items, unsigned grid) {
        const int64_t c = t * L.heads * 32 * L.groups, a = t * L.heads * L.groups;
        k_unpack<<<grid, 256, 0, s>>>(L, items, slots + t, k ? k + c : nullptr, ka ? (uint16_t*)ka + a : nullptr,
                                      v ? v + c : nullptr, va ? (uint16_t*)va + a : nullptr);
    });
}

}  // namespace esb
