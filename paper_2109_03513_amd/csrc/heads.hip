// Heads of queries, keys and values on their way into attention, one pass over each:
//
//  * the norm over a head and the rotation of its first `rot` elements: y = x rstd w,
//    rstd = 1 / sqrt(mean x^2 + eps); pairs (a, b) become (a c - b s, b c + a s), c and s from the
//    table's row of the token's position;
//  * keys (normed and rotated so) and values into the 4-bit cache, with alpha = bf16(max|y| / 6) per
//    32 elements and the nearest of the eight magnitudes to |y| / alpha, ties to the larger.
//
// A head has 4 to 64 lanes of a wave, each with sixteen elements: eight pairs of the rotation, or sixteen that stay.  So
// no pair crosses lanes, and heads may be rotated in place; only the sum of squares does, and for
// the cache a key's elements go through LDS once, into lanes of half a group.  A wave goes over heads of one
// token, whose cosines and sines it keeps.
//
// Keys for the cache are computed in fp64 and rounded once to fp32 before they get their codes: the
// same call gives the same codes wherever the borders lie.  esb_rope computes in fp32 around an fp64
// sum of squares, which does not overflow.
#include "kv4.h"

namespace esb {

namespace {

constexpr float kTiny = 0x1p-126f;

__device__ __forceinline__ float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

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

// Eight nibbles of one token into its block.
template <bool KEY>
__device__ __forceinline__ void store_codes(const Kv4Layout& L, uint8_t* b, int t, int e, uint32_t w) {
    if (KEY) {
        *key_word(L, b, t, e) = w;
    } else {
        uint8_t* o = value_byte(L, b, t, e);
#pragma unroll
        for (int i = 0; i < 4; i++) o[i * 4 * L.groups] = (uint8_t)(w >> (8 * i));
    }
}

// Codes of eight elements y under the scale a.  The borders are exact in fp32: three bits times eight.
__device__ __forceinline__ uint32_t nibbles(f32x8 y, float a) {
    const float b1 = 0.25f * a, b2 = 0.75f * a, b3 = 1.25f * a, b4 = 1.75f * a, b5 = 2.5f * a, b6 = 3.5f * a, b7 = 5.0f * a;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float v = fabsf(y[i]);
        const bool c4 = v >= b4, c2 = v >= (c4 ? b6 : b2);
        const bool c1 = v >= (c4 ? (c2 ? b7 : b5) : (c2 ? b3 : b1));
        const uint32_t c = (c4 ? 4u : 0u) + (c2 ? 2u : 0u) + (c1 ? 1u : 0u);
        w |= (c ? c | (__float_as_uint(y[i]) >> 28 & 8u) : 0u) << (4 * i);
    }
    return w;
}
// max |y| on bit patterns: a NaN is above every number.
__device__ __forceinline__ uint32_t magnitude(f32x8 y) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(y[i]) & 0x7fffffffu);
    return m;
}
// Codes and scale of sixteen elements from e on, half a group, whose other half a neighbouring lane has.
template <bool KEY>
__device__ __forceinline__ void store_half_group(const Kv4Layout& L, bool there, int64_t slot, int h, int e, f32x8 lo, f32x8 hi) {
    uint32_t m = max(magnitude(lo), magnitude(hi));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true));      // lanes 1 0 3 2 of four
    const bool fine = m < 0x7f800000u;
    const __bf16 a16 = (__bf16)fmaxf(__uint_as_float(m) / 6.0f, kTiny);
    const float a = (float)a16;
    if (!there) return;
    uint8_t* b = L.block(slot >> L.shift, h);
    const int t = (int)slot & (L.page - 1);
    store_codes<KEY>(L, b, t, e, fine ? nibbles(lo, a) : 0u);
    store_codes<KEY>(L, b, t, e + 8, fine ? nibbles(hi, a) : 0u);
    if ((e & 31) == 0)
        *scale_at(L, b, KEY ? L.key_scales_at() : L.value_scales_at(), t, e >> 5) = fine ? __builtin_bit_cast(uint16_t, a16) : (uint16_t)0x7fc0;
}

template <typename T>
__device__ __forceinline__ const T* head_at(const HeadsView& v, int64_t t, int h) {
    return (const T*)v.p + t * v.token + h * v.head;
}

template <int CTRL> __device__ __forceinline__ double turned(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// The sum over LPR neighbouring lanes, in each of them.
template <int LPR> __device__ __forceinline__ double lanes_sum(double v) {
    v += turned<0xb1>(v);                       // lanes 1 0 3 2 of four
    v += turned<0x4e>(v);                       // lanes 2 3 0 1
    if (LPR >= 8) v += turned<0x141>(v);        // eight lanes mirrored
    if (LPR >= 16) v += turned<0x140>(v);       // sixteen
    if (LPR >= 32) v += __shfl_xor(v, 16);
    if (LPR >= 64) v += __shfl_xor(v, 32);
    return v;
}

// 1 / sqrt(x) for positive x, by the hardware's approximation and two Newton steps: within a few 2^-53.
__device__ __forceinline__ double reciprocal_root(double x) {
    const double y0 = __builtin_amdgcn_rsq(x);
    const double y1 = fma(0.5 * y0, fma(-x * y0, y0, 1.0), y0);
    const double y2 = fma(0.5 * y1, fma(-x * y1, y1, 1.0), y1);
    return x < __builtin_inf() ? y2 : y0;      // 0 for infinity
}

// v in the precision of the work.  For fp64 anew wherever it is used: kept over a wave's steps, the wider copies
// of weights and table would cost it half its registers.
template <typename A> __device__ __forceinline__ A wide(float v) {
    if (sizeof(A) == 8) asm volatile("" : "+v"(v));
    return (A)v;
}

// Bound by HBM (86 MB of 4096 tokens, 40 heads of 128, rotated: 18.7 us, 4.6 TB/s), into the cache by latency (19 MB read
// and 5 written in 17.2 us: 155 registers, three waves a SIMD) and for few tokens by launch and one round trip (4.0 us).
// Rows over lanes of eight elements with the rotation across lanes took 29; loads asked for at once, the root by Newton
// steps and codes by three comparisons 18.8 -> 17.1 for the cache.
// Iterations of a wave: 64 / LPR heads of one kind (queries, keys, values) at a time, q_steps + k_steps + v_steps for a
// token; a wave takes `per` of them in turn.
template <typename T, typename A, int LPR, bool CACHE>
__global__ __launch_bounds__(256) void k_heads(HeadsParams p, int64_t token0, uint32_t waves, int per) {
    typedef typename Vec8<T>::type V;
    constexpr int HW = 64 / LPR;
    const int lane = threadIdx.x & 63, sub = lane / LPR, l = lane % LPR;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    __shared__ float rows[CACHE ? 4 : 1][CACHE ? HW * LPR * 16 : 1];
    if (wave >= waves) return;
    const int qs = (p.q.heads + HW - 1) / HW, ks = (p.k.heads + HW - 1) / HW, vs = CACHE ? (p.v.heads + HW - 1) / HW : 0;
    const int all = qs + ks + vs;
    const uint32_t parts = (all + per - 1) / per;
    const int64_t t = token0 + wave / parts;
    const int from = (int)(wave % parts) * per, to = min(from + per, all);

    // The lane's two runs of eight elements, and how many of each there are: eight pairs (j, j + rot / 2) of the
    // rotation, or of elements after it; adjacent pairs, and values: sixteen in a row.
    const int d = p.d, rot = p.rot, half = rot >> 1, turning = (half + 7) >> 3;
    int ea, eb, na, nb, pair = 8 * l;
    if (p.adjacent || rot == 0) {
        ea = 16 * l, eb = ea + 8, na = d - ea, nb = d - eb;
    } else if (l < turning) {
        ea = 8 * l, eb = half + ea, na = nb = half - ea;
    } else {
        ea = rot + 16 * (l - turning), eb = ea + 8, na = d - ea, nb = d - eb, pair = half;
    }
    // the position, the slot and the first heads are asked for at once, then the table's row
    const bool turned_step = from < qs + ks;
    const int64_t pos = rot && turned_step ? p.positions[t] : 0;
    const int64_t slot = CACHE ? p.slots[t] : -1;
    struct In {
        V a, b;
    };
    auto step_of = [&](int i, int* kind) {      // the first head of the step's
        *kind = i < qs ? 0 : i < qs + ks ? 1 : 2;
        return HW * (i - (i < qs ? 0 : i < qs + ks ? qs : qs + ks)) + sub;
    };
    auto load = [&](int i) {
        int kind;
        const int h = step_of(i, &kind);
        const HeadsView& v = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
        In in = {V{}, V{}};
        if (i < to && h < v.heads) {
            const T* x = head_at<T>(v, t, h);
            if (CACHE && kind == 2) {
                if (16 * l < d) in.a = load8(x + 16 * l, 8), in.b = load8(x + 16 * l + 8, 8);
            } else {
                if (na > 0) in.a = load8(x + ea, na);
                if (nb > 0) in.b = load8(x + eb, nb);
            }
        }
        return in;
    };
    In next = load(from);
    const bool known = !rot || (pos >= 0 && pos < p.rows);
    const bool there = CACHE && slot >= 0 && (slot >> p.cache.shift) < p.cache.pages;
    const int turns = half - pair;      // the lane's pairs that are rotated, from the first on
    f32x8 c = {}, s = {};
    if (known && turns > 0 && turned_step) {
        const float* row = p.table + pos * rot;
        c = load8(row + pair, turns), s = load8(row + half + pair, turns);
    }
    int weights_of = -1;
    f32x8 wa, wb;
    for (int i = from; i < to; i++) {
        const In in = next;
        next = load(i + 1);
        int kind;
        const int h = step_of(i, &kind);
        if (CACHE && kind == 2) {
            store_half_group<false>(p.cache, there && h < p.v.heads && 16 * l < d, slot, h, 16 * l, __builtin_convertvector(in.a, f32x8),
                                    __builtin_convertvector(in.b, f32x8));
            continue;
        }
        A rstd = 1;
        if (p.eps > 0.0f) {
            if (kind != weights_of) {
                weights_of = kind;
                wa = wb = f32x8{1, 1, 1, 1, 1, 1, 1, 1};
                const float* w = kind == 0 ? p.qw : p.kw;
                if (w && na > 0) wa = load8(w + ea, na);
                if (w && nb > 0) wb = load8(w + eb, nb);
            }
            double ss = 0.0;
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const double a = (double)(float)in.a[k], b = (double)(float)in.b[k];
                ss = fma(a, a, fma(b, b, ss));
            }
            ss = lanes_sum<LPR>(ss);
            rstd = (A)reciprocal_root(fma(ss, p.inv_d, (double)p.eps));
        }
        if (!known) rstd = (A)__builtin_nan("");
        // element k of the lane's first run and of its second, normed
        auto first = [&](int k) { return p.eps > 0.0f ? (A)(float)in.a[k] * rstd * wide<A>(wa[k]) : known ? (A)(float)in.a[k] : rstd; };
        auto second = [&](int k) { return p.eps > 0.0f ? (A)(float)in.b[k] * rstd * wide<A>(wb[k]) : known ? (A)(float)in.b[k] : rstd; };
        f32x8 lo, hi;
        if (p.adjacent) {
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const A a = first(k), b = first(k + 1), c0 = wide<A>(c[k / 2]), s0 = wide<A>(s[k / 2]);
                const bool t0 = k / 2 < turns, t1 = 4 + k / 2 < turns;
                lo[k] = (float)(t0 ? fma(a, c0, -(b * s0)) : a), lo[k + 1] = (float)(t0 ? fma(b, c0, a * s0) : b);
                const A u = second(k), v = second(k + 1), c1 = wide<A>(c[4 + k / 2]), s1 = wide<A>(s[4 + k / 2]);
                hi[k] = (float)(t1 ? fma(u, c1, -(v * s1)) : u), hi[k + 1] = (float)(t1 ? fma(v, c1, u * s1) : v);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const A a = first(k), b = second(k), co = wide<A>(c[k]), si = wide<A>(s[k]);
                lo[k] = (float)(k < turns ? fma(a, co, -(b * si)) : a), hi[k] = (float)(k < turns ? fma(b, co, a * si) : b);
            }
        }
        if (!CACHE || kind == 0) {
            const HeadsView& v = kind == 0 ? p.qo : p.ko;
            if (h < v.heads) {
                T* o = (T*)head_at<T>(v, t, h);
                if (na > 0) store8(o + ea, __builtin_convertvector(lo, V), na);
                if (nb > 0) store8(o + eb, __builtin_convertvector(hi, V), nb);
            }
            continue;
        }
        if (!p.adjacent && rot) {      // into sixteen elements in a row
            float* row = rows[threadIdx.x >> 6] + sub * d;
            if (na > 0) store8(row + ea, lo, na);
            if (nb > 0) store8(row + eb, hi, nb);
            __builtin_amdgcn_wave_barrier();      // LDS serves a wave in order
            if (16 * l < d) lo = load8(row + 16 * l, 8), hi = load8(row + 16 * l + 8, 8);
            __builtin_amdgcn_wave_barrier();
        }
        store_half_group<true>(p.cache, there && h < p.k.heads && 16 * l < d, slot, h, 16 * l, lo, hi);
    }
}

// ESB(4,1) codes 0 .. 7 are 1, 1.5, 2, 3, 4, 6, 0, 0.5: E2M1's order turned by two.  A thread to eight elements, bytes in
// and out as wide as they come: 4096 tokens of 8 heads of 128 unpacked in 6.3 us (13 MB), latency.
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
    store_codes<true>(L, b, at, e, word(k));
    store_codes<false>(L, b, at, e, word(v));
    if (e & 31) return;
    auto kept = [](uint16_t a) { return (a & 0x7f80) == 0x7f80 ? (uint16_t)0x7fc0 : a; };      // infinities as NaN
    *scale_at(L, b, L.key_scales_at(), at, e >> 5) = kept(ka[s]);
    *scale_at(L, b, L.value_scales_at(), at, e >> 5) = kept(va[s]);
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
    constexpr int HW = 64 / LPR;
    auto steps = [](int heads) { return (heads + HW - 1) / HW; };
    const int64_t all = (int64_t)steps(p.q.heads) + steps(p.k.heads) + (CACHE ? steps(p.v.heads) : 0);
    // One step a wave while that makes up to four waves a SIMD, about what the registers allow.  4096 tokens of 40 heads
    // (us, with half and twice as many): rotated 18.7 (18.6, 19.3), into the cache 17.2 (17.2, 18.1).
    const int64_t most_waves = 16 * num_cus();
    int64_t per = (p.tokens * all + most_waves - 1) / most_waves;
    if (per > all) per = all;
    const int64_t parts = (all + per - 1) / per, most = ((int64_t)1 << 28) / parts;      // tokens of one launch
    for (int64_t t = 0; t < p.tokens; t += most) {
        const uint32_t waves = (uint32_t)((p.tokens - t < most ? p.tokens - t : most) * parts);
        k_heads<T, A, LPR, CACHE><<<(waves + 3) / 4, 256, 0, s>>>(p, t, waves, (int)per);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, typename A, bool CACHE>
hipError_t launch_t(const HeadsParams& p, hipStream_t s) {
    const int half = p.rot / 2;
    int lanes = (p.d + 15) / 16;
    if (!p.adjacent) {
        const int n = (half + 7) / 8 + (p.d - p.rot + 15) / 16;
        if (n > lanes) lanes = n;
    }
    if (lanes <= 4) return launch_n<T, A, 4, CACHE>(p, s);
    if (lanes <= 8) return launch_n<T, A, 8, CACHE>(p, s);
    if (lanes <= 16) return launch_n<T, A, 16, CACHE>(p, s);
    if (lanes <= 32) return launch_n<T, A, 32, CACHE>(p, s);
    return launch_n<T, A, 64, CACHE>(p, s);
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
