// Attention over the 4-bit paged cache:
//   o = softmax(scale q k^T) v over keys j <= length - n + i for the i-th of a sequence's n queries,
//   k = alpha_k q_k, v = alpha_v q_v, alpha per 32 elements of a key's or value's head.
//
// The scores are formed transposed, S^T = K Q^T, on 16x16x32 MFMAs: E2M1 codes are exact in bf16 and fp16,
// one MFMA covers one scale group, whose alpha multiplies its fp32 sum.  A lane then holds eight keys of one
// query, which is what the second product O^T = V^T P^T wants of its operand: the probabilities never
// leave the lane.  A value's alpha multiplies the probability (one operand per group), so its codes
// go into the MFMA unscaled.  The product of probability and alpha is rounded to bf16 (for fp16 outputs to
// the sum of two bf16, one more MFMA): 2^-9 of each of the terms that a softmax averages, which is
// below the rounding of a bf16 output.
//
// A workgroup takes 16 NT rows (queries x heads that share a key head) and some of their keys; its four
// waves take every fourth step of 32 keys, each with its own running maximum and sum, and join them in
// LDS.  The keys are split over workgroups too, in runs or in even shares of all work (split() below),
// and a k_join_... adds the parts.  The running maximum moves only when a score passes it by 2^8, so
// most steps cross no lanes.  Rows whose sums near the end of fp32 for that, or whose maximum is beyond 2^20, so that x
// scale - m in one rounding is off by too much, are gone over once more (wide_pass): looking for them costs 1 %, checks
// within the loop cost up to 5.
#include <algorithm>
#include <type_traits>

#include "attend.h"

namespace esb {

namespace {

constexpr int kMostEven = 1024;      // sequences among which work is shared evenly, at most
constexpr uint32_t kLarge = 0x71800000;      // 2^100: as many parts of it as there may be are within fp32
constexpr int kRuns = 16;      // parts of a row that one thread joins, at most

template <int N> struct Words {
    typedef uint32_t w __attribute__((ext_vector_type(N)));
};

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// Rows 32 c + 2 i and 32 c + 2 i + 1 of V^T, from the words of two runs: byte t of a word is key t of its run.
__device__ __forceinline__ void value_pairs(uint32_t a, uint32_t b, bf16x8* even, bf16x8* odd) {
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int hh = 0; hh < 2; hh++) {
        const uint32_t w = hh ? b : a;
        const uint32_t t0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
        const uint32_t t1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
        const uint32_t t2 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
        const uint32_t t3 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
        lo[2 * hh] = __builtin_amdgcn_perm(t1, t0, 0x05040100);
        lo[2 * hh + 1] = __builtin_amdgcn_perm(t3, t2, 0x05040100);
        hi[2 * hh] = __builtin_amdgcn_perm(t1, t0, 0x07060302);
        hi[2 * hh + 1] = __builtin_amdgcn_perm(t3, t2, 0x07060302);
    }
    *even = join4<bf16x8>(lo[0], lo[1], lo[2], lo[3]);
    *odd = join4<bf16x8>(hi[0], hi[1], hi[2], hi[3]);
}
// Over the four lanes that hold one column.
__device__ __forceinline__ float column_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float column_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// Whether sums of weights of up to 2^kLazy times values are not finite, or so large that those of further parts might leave
// fp32.  Such rows take wide_pass, if it is for their values.
__device__ __forceinline__ bool is_large(f32x8 o) {
    int above = 0;
    uint32_t below = 0;      // by sign
#pragma unroll
    for (int e = 0; e < 8; e++) above = max(above, __float_as_int(o[e])), below = max(below, __float_as_uint(o[e]));
    return above >= (int)kLarge || below >= (kLarge | 0x80000000u);
}
// Whether weights under this maximum may be off by more than exp2 may be given (kFar), even infinite: rows whose maximum was
// far in some wave, at some time, take it too.  A wave tells by the sign of its sum.
__device__ __forceinline__ bool is_far(float m) { return fabsf(m) > kFar && fabsf(m) < __builtin_inff(); }
__device__ __forceinline__ float marked(float sum, int mark) { return __builtin_copysignf(sum, mark ? -1.0f : 1.0f); }
__device__ __forceinline__ bool is_marked(float sum) { return __float_as_int(sum) < 0; }
// The rows of which some of a wave's lanes, N to a row, say so.
template <int N> __device__ __forceinline__ uint32_t rows_of(uint64_t lanes) {
    uint32_t rows = 0;
#pragma unroll
    for (int j = 0; j < 64 / N; j++)
        if (lanes >> N * j & ((1ull << N) - 1)) rows |= 1u << j;
    return rows;
}

// What a wave brings of 32 keys, in two halves of 16.  Keys: the lane's words of key lane % 16; values: its
// bytes of the run of four keys lane / 16; scales: of the same run.
template <int CP> struct Step {
    typename Words<CP>::w k[2], v[2];
    uint2 ka[2][CP], va[2][CP];
    int bad;             // halves whose page is none of the cache's
};

// Rows of heads in tiles of sixteen, one scale group to an MFMA.  Bound by VALU issue (decoding a group's codes, its
// scales and exp2, once for 16 NT rows): 64 sequences of 2048 keys, 8 queries of 4 heads of 128 to a key head, 71 us,
// 240 TFLOP/s; drafts of five tokens, fp16 heads of 64, 15.2 us and 4 of joins, latency.  Waves without LDS in the loop:
// each loads its own keys, two steps in flight.
// CP: the head's groups, padded (FULL: exactly).  What is padded meets zeros of the query, or makes outputs that
// are not stored; its scales repeat the last group's.
template <typename T, int CP, int NT, bool FULL, bool EVEN>
__global__ __launch_bounds__(256, CP * NT <= 2 ? 3 : CP * NT <= 4 ? 2 : 1)
void k_kv4(Kv4AttentionParams p, Kv4Split sp, float* part, float2* stats) {
    typedef typename Vec8<T>::type V;
    constexpr int R = 16 * NT;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int C = FULL ? CP : p.cache.groups;
    __shared__ int kept[EVEN ? 4 : 1][6][64];
    asm volatile("" ::"s"(part), "s"(stats));      // asked for with the first arguments, not when they are used
    Work<EVEN> work(p, sp, R, kept);
    while (work.next()) {
        const Rows& rw = work.rw;
        const int h = work.h;
        const int32_t* table = p.table + rw.seq * p.table_pitch;
        const int page = p.cache.page;
        struct Ids {
            int a, b;
        };
        auto ids = [&](int at) {      // pages of the halves of a step; behind the last key whatever the table holds
            return Ids{table[min(at >> p.cache.shift, p.columns - 1)],
                       table[min((at + 16) >> p.cache.shift, p.columns - 1)]};
        };
        const int at0 = work.from + 32 * wave;
        Ids next = p.columns > 0 ? ids(at0) : Ids{0, 0};
        V qf[NT][CP];
#pragma unroll
        for (int u = 0; u < NT; u++) {
            const int r = rw.row0 + 16 * u + i, t = r / p.group;
            const T* q = (const T*)p.q.p + (rw.begin + t) * p.q.token + (h * p.group + r % p.group) * p.q.head;
#pragma unroll
            for (int s = 0; s < CP; s++) {
                qf[u][s] = V{};
                if (r < rw.rows && s < C) qf[u][s] = load8(q + 32 * s + 8 * g, 8);
            }
        }

        const int first = rw.len - rw.n;                    // the last key of query t is first + t
        const int keys = max(first + (min(rw.row0 + R, rw.rows) - 1) / p.group + 1, 0);
        const int k1 = min(work.to, keys);
        const int open = first + rw.row0 / p.group;         // keys up to here are seen by every row

        int last[NT];
#pragma unroll
        for (int u = 0; u < NT; u++) last[u] = first + (rw.row0 + 16 * u + i) / p.group;

        auto load = [&](int at, Ids pg) {
            Step<CP> st;
            st.bad = 0;
#pragma unroll
            for (int hh = 0; hh < 2; hh++) {
                int pid = __builtin_amdgcn_readfirstlane(hh ? pg.b : pg.a);
                if (pid < 0 || pid >= p.cache.pages) pid = 0, st.bad |= 1 << hh;
                const uint8_t* b = p.cache.block(pid, h);
                const int t = (at + 16 * hh) & (page - 1);
                // words past the head's groups are of what follows in the block, and nothing uses them
                st.k[hh] = ((const Loose<typename Words<CP>::w, uint32_t>*)(b + (t + i) * 16 * C + g * 4 * C))->v;
                st.v[hh] = ((const Loose<typename Words<CP>::w, uint32_t>*)(b + p.cache.values_at() + ((t >> 2) + g) * 64 * C +
                                                                i * 4 * C))->v;
                const uint8_t* ks = b + p.cache.key_scales_at() + ((t >> 2) + g) * 8 * C;
                const uint8_t* vs = b + p.cache.value_scales_at() + ((t >> 2) + g) * 8 * C;
#pragma unroll
                for (int s = 0; s < CP; s++) {
                    const int g8 = FULL ? 8 * s : 8 * min(s, C - 1);
                    st.ka[hh][s] = *(const uint2*)(ks + g8);
                    st.va[hh][s] = *(const uint2*)(vs + g8);
                }
            }
            return st;
        };

        f32x4 acc[NT][CP][2] = {};
        float top[NT], sum[NT];      // the running maximum (times scale) and the lane's part of the sum
        int distant = 0;             // bit u: the maximum was far (is_far) at some time
#pragma unroll
        for (int u = 0; u < NT; u++) top[u] = kNegInf, sum[u] = 0.0f;

        auto compute = [&](const Step<CP>& st, int at, auto masks) {
            constexpr bool MASK = decltype(masks)::value;
            f32x4 x[NT][2];
#pragma unroll
            for (int hh = 0; hh < 2; hh++)
#pragma unroll
                for (int s = 0; s < CP; s++) {
                    const V kf = decode(st.k[hh][s], T{});
                    const f32x4 a = four(st.ka[hh][s]);
#pragma unroll
                    for (int u = 0; u < NT; u++) {
                        const f32x4 z = mma(kf, qf[u][s], f32x4{0, 0, 0, 0});
#pragma unroll
                        for (int r = 0; r < 4; r++) x[u][hh][r] = s ? fmaf(a[r], z[r], x[u][hh][r]) : a[r] * z[r];
                    }
                }
            float most[NT];
            bool moves = false;
#pragma unroll
            for (int u = 0; u < NT; u++) {
                most[u] = kNegInf;
#pragma unroll
                for (int hh = 0; hh < 2; hh++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        if (MASK) {
                            if (st.bad >> hh & 1) x[u][hh][r] = __builtin_nanf("");
                            if (at + 16 * hh + 4 * g + r > last[u]) x[u][hh][r] = kNegInf;
                        }
                        most[u] = fmaxf(most[u], x[u][hh][r]);
                    }
                most[u] *= p.scale;
                moves |= passes(most[u], top[u]);
            }
            if (__ballot(moves)) {
#pragma unroll
                for (int u = 0; u < NT; u++) {
                    // row by row: what a row gives does not depend on its neighbours
                    const float all = column_max(most[u]), now = passes(all, top[u]) ? all : top[u];
                    const float f = now == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(top[u] - now);
                    top[u] = now;
                    if (is_far(now)) distant |= 1 << u;
                    sum[u] *= f;
#pragma unroll
                    for (int c = 0; c < CP; c++) acc[u][c][0] *= f, acc[u][c][1] *= f;
                }
            }
#pragma unroll
            for (int u = 0; u < NT; u++) {
                const float m = top[u] == kNegInf ? 0.0f : top[u];
#pragma unroll
                for (int hh = 0; hh < 2; hh++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        x[u][hh][r] = __builtin_amdgcn_exp2f(fmaf(x[u][hh][r], p.scale, -m));
                        sum[u] += x[u][hh][r];
                    }
            }
#pragma unroll
            for (int c = 0; c < CP; c++) {
                bf16x8 v0, v1;
                value_pairs(st.v[0][c], st.v[1][c], &v0, &v1);
                const f32x4 a0 = four(st.va[0][c]), a1 = four(st.va[1][c]);
#pragma unroll
                for (int u = 0; u < NT; u++) {
                    f32x8 w;
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        w[r] = x[u][0][r] * a0[r];
                        w[4 + r] = x[u][1][r] * a1[r];
                        if (MASK) {      // scales behind the last key may be anything
                            if (at + 4 * g + r > last[u]) w[r] = 0.0f;
                            if (at + 16 + 4 * g + r > last[u]) w[4 + r] = 0.0f;
                        }
                    }
                    const bf16x8 hi = __builtin_convertvector(w, bf16x8);
                    acc[u][c][0] = mma(v0, hi, acc[u][c][0]);
                    acc[u][c][1] = mma(v1, hi, acc[u][c][1]);
                    if (std::is_same<T, _Float16>::value) {
                        const bf16x8 lo = __builtin_convertvector(w - __builtin_convertvector(hi, f32x8), bf16x8);
                        acc[u][c][0] = mma(v0, lo, acc[u][c][0]);
                        acc[u][c][1] = mma(v1, lo, acc[u][c][1]);
                    }
                }
            }
        };

        int at = at0;
        if (at < k1) {
            Step<CP> cur = load(at, next);
            next = ids(at + 128);
            for (; at < k1; at += 128) {
                Step<CP> st = cur;
                if (at + 128 < k1) cur = load(at + 128, next);
                next = ids(at + 256);
                if (at + 31 > open || st.bad) compute(st, at, std::true_type{});
                else compute(st, at, std::false_type{});
            }
        }

        const bool whole = work.whole;
        // join the waves
        __shared__ float2 waves[4][NT][16];
        __shared__ float sums[4][16][132];
        float factor[NT], total[NT];
        int apart = 0;      // bit u: the column's row of tile u had a far maximum
#pragma unroll
        for (int u = 0; u < NT; u++) {
            sum[u] = column_sum(sum[u]);
            if (g == 0) waves[wave][u][i] = make_float2(top[u], marked(sum[u], distant >> u & 1));
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < NT; u++) {
            float m = kNegInf;
#pragma unroll
            for (int w = 0; w < 4; w++) m = fmaxf(m, waves[w][u][i].x);
            float l = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float2 o = waves[w][u][i];
                if (is_marked(o.y)) apart |= 1 << u;
                l += o.x == kNegInf ? fabsf(o.y) : fabsf(o.y) * __builtin_amdgcn_exp2f(o.x - m);
            }
            factor[u] = top[u] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(top[u] - m);
            total[u] = l;
            top[u] = m;
        }
        const int col = threadIdx.x >> 4, dd = 8 * (threadIdx.x & 15);
        uint32_t large = 0, far = 0;      // bit 16 u: of tile u
#pragma unroll
        for (int u = 0; u < NT; u++) {
#pragma unroll
            for (int c0 = 0; c0 < CP; c0 += 4) {
                if (c0 >= C) continue;
                __syncthreads();
#pragma unroll
                for (int c = c0; c < c0 + 4 && c < CP; c++)
#pragma unroll
                    for (int r = 0; r < 4; r++)
#pragma unroll
                        for (int e = 0; e < 2; e++)
                            sums[wave][i][32 * (c - c0) + 8 * g + 2 * r + e] = acc[u][c][e][r] * factor[u];
                __syncthreads();
                const float m = __shfl(top[u], col), l = __shfl(total[u], col);
                const bool distant = __shfl(apart, col) >> u & 1;
                const int r = rw.row0 + 16 * u + col, e0 = 32 * c0 + dd;
                f32x8 o = {};
                if (r < rw.rows && e0 < 32 * C) {
#pragma unroll
                    for (int w = 0; w < 4; w++)
#pragma unroll
                        for (int e = 0; e < 8; e++) o[e] += sums[w][col][dd + e];
                    large |= is_large(o) ? 1u << (16 * u) : 0;
                    far |= distant ? 1u << (16 * u) : 0;
                    const int t = r / p.group, head = h * p.group + r % p.group;
                    if (!whole) {
                        const int64_t at = EVEN ? (int64_t)work.place * R + 16 * u + col
                                                : ((rw.begin + t) * p.q.heads + head) * sp.chunks + work.place;
                        *(f32x8*)(part + at * 32 * C + e0) = o;
                        if (e0 == 0) stats[at] = make_float2(m, l);
                    } else {
                        if (rw.bad) o = f32x8{} + __builtin_nanf("");
                        else if (first + t >= 0) o *= 1.0f / l;
                        store8((T*)p.o.p + (rw.begin + t) * p.o.token + head * p.o.head + e0,
                               __builtin_convertvector(o, V), 8);
                    }
                }
            }
        }
        if (__builtin_expect(__any(large | far), 0)) {
            if (!large_values(p, rw, h, work.from, work.to)) large = 0;
            __threadfence();      // what follows comes after the stores above
            uint32_t mask = 0;
#pragma unroll
            for (int u = 0; u < NT; u++) mask |= rows_of<16>(__ballot((large | far) >> (16 * u) & 1)) << (16 * u + 4 * wave);
            if (mask)
                wide_pass<T, EVEN>(p, rw, h, work.from, work.to, rw.row0, mask, whole ? -1 : EVEN ? (int64_t)work.place * R : work.place,
                                   sp.chunks, part, stats);
        }
        if (EVEN) __syncthreads();      // the next item uses the same LDS
    }
}

// Few rows, one per (query, head): 16 / CP of them to a tile, whose columns are (row, scale group).  A column's query
// has only its own group's elements, so that one MFMA after the other leaves each group's sum in a column
// of its own, and a lane needs the scales of one group: four of a key's, four of a value's.  The sum over the
// groups crosses CP neighbouring lanes; of O^T a column keeps the rows of its group.  Against a tile of 16 rows, most of
// them empty: fewer scales, and registers for three workgroups a CU instead of two (64 ragged sequences up to 8192 keys,
// 4 heads of 128 to a key head: 127 -> 91 us).  Bound by HBM: those 386 MB in 77 us, 5.0 TB/s (a copy moves 5.2); one
// sequence of 32768 keys 12.1 us, 3.1 TB/s, launch and ramp.
template <int CP> __device__ __forceinline__ float over_groups(float v) {
    auto turned = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v += turned(v, std::integral_constant<int, 0xb1>{});                  // lanes 1 0 3 2 of four
    if (CP >= 4) v += turned(v, std::integral_constant<int, 0x4e>{});     // lanes 2 3 0 1
    if (CP >= 8) v += turned(v, std::integral_constant<int, 0x141>{});    // eight lanes mirrored
    return v;
}

template <typename T, int CP, int NT, bool FULL, bool EVEN>
__global__ __launch_bounds__(256, CP * NT <= 2 ? 4 : CP * NT <= 4 ? 3 : CP * NT <= 8 ? 2 : 1)
void k_kv4_few(Kv4AttentionParams p, Kv4Split sp, float* part, float2* stats) {
    typedef typename Vec8<T>::type V;
    typedef typename Words<CP>::w W;
    constexpr int HR = 16 / CP, R = HR * NT;
    const int C = FULL ? CP : p.cache.groups;
    __shared__ int kept[EVEN ? 4 : 1][6][64];
    asm volatile("" ::"s"(part), "s"(stats));      // asked for with the first arguments, not when they are used
    Work<EVEN> work(p, sp, R, kept);
    while (work.next()) {
        const Rows& rw = work.rw;
        const int h = work.h;
        int thread = threadIdx.x;
        if (EVEN) asm volatile("" : "+v"(thread));      // nothing of the lane is kept from item to item: registers are short
        const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
        const int i = lane & 15, g = lane >> 4, own = i % CP;

        const int32_t* table = p.table + rw.seq * p.table_pitch;
        const int page = p.cache.page;
        struct Ids {
            int a, b;
        };
        auto ids = [&](int at) {      // pages of the halves of a step; behind the last key whatever the table holds
            return Ids{table[min(at >> p.cache.shift, p.columns - 1)],
                       table[min((at + 16) >> p.cache.shift, p.columns - 1)]};
        };
        const int at0 = work.from + 32 * wave;
        Ids next = p.columns > 0 ? ids(at0) : Ids{0, 0};
        V qf[NT][CP];
#pragma unroll
        for (int u = 0; u < NT; u++) {
            const int r = rw.row0 + HR * u + i / CP, t = r / p.group;
            const T* q = (const T*)p.q.p + (rw.begin + t) * p.q.token + (h * p.group + r % p.group) * p.q.head;
            V mine = {};
            if (r < rw.rows && own < C) mine = load8(q + 32 * own + 8 * g, 8);
#pragma unroll
            for (int s = 0; s < CP; s++) qf[u][s] = s == own ? mine : V{};
        }

        const int first = rw.len - rw.n;                    // the last key of query t is first + t
        const int keys = max(first + (min(rw.row0 + R, rw.rows) - 1) / p.group + 1, 0);
        const int k1 = min(work.to, keys);
        const int open = first + rw.row0 / p.group;         // keys up to here are seen by every row

        int last[NT];
#pragma unroll
        for (int u = 0; u < NT; u++) last[u] = first + (rw.row0 + HR * u + i / CP) / p.group;

        struct Piece {
            W k[2], v[2];
            uint2 ka[2], va[2];
            int bad;
        };
        // what a lane adds to a half's place in its block
        const uint32_t k_at = i * 16 * C + g * 4 * C, v_at = g * 64 * C + i * 4 * C;
        const uint32_t s_at = g * 8 * C + 8 * (FULL ? own : min(own, C - 1));
        auto load = [&](int at, Ids pg) {
            Piece st;
            st.bad = 0;
#pragma unroll
            for (int hh = 0; hh < 2; hh++) {
                int pid = __builtin_amdgcn_readfirstlane(hh ? pg.b : pg.a);
                if (pid < 0 || pid >= p.cache.pages) pid = 0, st.bad |= 1 << hh;
                const int t = (at + 16 * hh) & (page - 1);
                // words past the head's groups are of what follows in the block, and nothing uses them
                const uint8_t* b = p.cache.block(pid, h);
                const uint8_t *kb = b + t * 16 * C, *vb = b + p.cache.values_at() + t * 16 * C;
                const uint8_t* ks = b + p.cache.key_scales_at() + t * 2 * C;
                const uint8_t* vs = b + p.cache.value_scales_at() + t * 2 * C;
                st.k[hh] = ((const Loose<W, uint32_t>*)(kb + k_at))->v;
                st.v[hh] = ((const Loose<W, uint32_t>*)(vb + v_at))->v;
                st.ka[hh] = *(const uint2*)(ks + s_at);
                st.va[hh] = *(const uint2*)(vs + s_at);
            }
            return st;
        };

        f32x4 acc[NT][CP][2] = {};
        float top[NT], sum[NT];
        int distant = 0;
#pragma unroll
        for (int u = 0; u < NT; u++) top[u] = kNegInf, sum[u] = 0.0f;

        auto compute = [&](const Piece& st, int at) {
            const bool masks = at + 31 > open || st.bad;
            f32x4 x[NT][2];
#pragma unroll
            for (int hh = 0; hh < 2; hh++) {
                f32x4 z[NT] = {};
#pragma unroll
                for (int s = 0; s < CP; s++) {
                    const V kf = decode(st.k[hh][s], T{});
#pragma unroll
                    for (int u = 0; u < NT; u++) z[u] = mma(kf, qf[u][s], z[u]);
                }
                const f32x4 a = four(st.ka[hh]);
#pragma unroll
                for (int u = 0; u < NT; u++)
#pragma unroll
                    for (int r = 0; r < 4; r++) x[u][hh][r] = over_groups<CP>(a[r] * z[u][r]);
            }
            if (masks) {
#pragma unroll
                for (int u = 0; u < NT; u++)
#pragma unroll
                    for (int hh = 0; hh < 2; hh++)
#pragma unroll
                        for (int r = 0; r < 4; r++) {
                            if (st.bad >> hh & 1) x[u][hh][r] = __builtin_nanf("");
                            if (at + 16 * hh + 4 * g + r > last[u]) x[u][hh][r] = kNegInf;
                        }
            }
            float most[NT];
            bool moves = false;
#pragma unroll
            for (int u = 0; u < NT; u++) {
                most[u] = kNegInf;
#pragma unroll
                for (int hh = 0; hh < 2; hh++)
#pragma unroll
                    for (int r = 0; r < 4; r++) most[u] = fmaxf(most[u], x[u][hh][r]);
                most[u] *= p.scale;
                moves |= passes(most[u], top[u]);
            }
            if (__ballot(moves)) {
#pragma unroll
                for (int u = 0; u < NT; u++) {
                    // row by row: what a row gives does not depend on its neighbours
                    const float all = column_max(most[u]), now = passes(all, top[u]) ? all : top[u];
                    const float f = now == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(top[u] - now);
                    top[u] = now;
                    if (is_far(now)) distant |= 1 << u;
                    sum[u] *= f;
#pragma unroll
                    for (int c = 0; c < CP; c++) acc[u][c][0] *= f, acc[u][c][1] *= f;
                }
            }
            const f32x4 b[2] = {four(st.va[0]), four(st.va[1])};
            bf16x8 hi[NT], lo[NT];
#pragma unroll
            for (int u = 0; u < NT; u++) {
                const float m = top[u] == kNegInf ? 0.0f : top[u];
                f32x8 w;
#pragma unroll
                for (int hh = 0; hh < 2; hh++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(x[u][hh][r], p.scale, -m));
                        sum[u] += e;
                        w[4 * hh + r] = e * b[hh][r];
                    }
                if (masks)      // scales behind the last key may be anything
#pragma unroll
                    for (int r = 0; r < 8; r++)
                        if (at + 4 * (r & 4) + 4 * g + (r & 3) > last[u]) w[r] = 0.0f;
                hi[u] = __builtin_convertvector(w, bf16x8);
                if (std::is_same<T, _Float16>::value)
                    lo[u] = __builtin_convertvector(w - __builtin_convertvector(hi[u], f32x8), bf16x8);
            }
#pragma unroll
            for (int c = 0; c < CP; c++) {
                bf16x8 v0, v1;
                value_pairs(st.v[0][c], st.v[1][c], &v0, &v1);
#pragma unroll
                for (int u = 0; u < NT; u++) {
                    acc[u][c][0] = mma(v0, hi[u], acc[u][c][0]);
                    acc[u][c][1] = mma(v1, hi[u], acc[u][c][1]);
                    if (std::is_same<T, _Float16>::value) {
                        acc[u][c][0] = mma(v0, lo[u], acc[u][c][0]);
                        acc[u][c][1] = mma(v1, lo[u], acc[u][c][1]);
                    }
                }
            }
        };

        int at = at0;
        if (at < k1) {
            Piece cur = load(at, next);
            next = ids(at + 128);
            for (; at < k1; at += 128) {
                const Piece st = cur;
                if (at + 128 < k1) cur = load(at + 128, next);
                next = ids(at + 256);
                compute(st, at);
            }
        }

        const bool whole = work.whole;
        // join the waves: each leaves its sums under the common maximum
        __shared__ float2 waves[4][NT][16];
        __shared__ __align__(16) float sums[4][R][32 * CP];
#pragma unroll
        for (int u = 0; u < NT; u++) {
            sum[u] = column_sum(sum[u]);
            if (g == 0) waves[wave][u][i] = make_float2(top[u], marked(sum[u], distant >> u & 1));
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < NT; u++) {
            float m = kNegInf;
#pragma unroll
            for (int w = 0; w < 4; w++) m = fmaxf(m, waves[w][u][i].x);
            const float f = top[u] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(top[u] - m);
            f32x8 o;
#pragma unroll
            for (int c = 0; c < CP; c++)
                if (c == own)
#pragma unroll
                    for (int r = 0; r < 8; r++) o[r] = acc[u][c][r & 1][r >> 1] * f;
            *(f32x8*)&sums[wave][HR * u + i / CP][32 * own + 8 * g] = o;
        }
        __syncthreads();
        const int row = thread / (4 * CP), e = 8 * (thread % (4 * CP)), r = rw.row0 + row;
        bool large = false, far = false;
        if (row < R && r < rw.rows && e < 32 * C) {
            float m = kNegInf, l = 0.0f;
            const int u = row / HR, column = row % HR * CP;
#pragma unroll
            for (int w = 0; w < 4; w++) m = fmaxf(m, waves[w][u][column].x);
            f32x8 o = {};
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float2 x = waves[w][u][column];
                far |= is_marked(x.y);
                l += x.x == kNegInf ? fabsf(x.y) : fabsf(x.y) * __builtin_amdgcn_exp2f(x.x - m);
                o += *(const f32x8*)&sums[w][row][e];
            }
            large = is_large(o);
            const int t = r / p.group, head = h * p.group + r % p.group;
            if (!whole) {
                const int64_t to = EVEN ? (int64_t)work.place * R + row
                                        : ((rw.begin + t) * p.q.heads + head) * sp.chunks + work.place;
                *(f32x8*)(part + to * 32 * C + e) = o;
                if (e == 0) stats[to] = make_float2(m, l);
            } else {
                if (rw.bad) o = f32x8{} + __builtin_nanf("");
                else if (first + t >= 0) o *= 1.0f / l;
                store8((T*)p.o.p + (rw.begin + t) * p.o.token + head * p.o.head + e, __builtin_convertvector(o, V), 8);
            }
        }
        if (__builtin_expect(__any(large || far), 0)) {
            if (!large_values(p, rw, h, work.from, work.to)) large = false;
            __threadfence();      // what follows comes after the stores above
            const uint32_t mask = rows_of<4 * CP>(__ballot(large || far)) << (16 / CP * wave);
            if (mask)
                wide_pass<T, EVEN>(p, rw, h, work.from, work.to, rw.row0, mask, whole ? -1 : EVEN ? (int64_t)work.place * R : work.place,
                                   sp.chunks, part, stats);
        }
        if (EVEN) __syncthreads();      // the next item uses the same LDS
    }
}

// What a join has to know of a row: the query's token and head, and its keys' runs.
struct JoinRow {
    bool live, bad;
    int keys;
};
__device__ __forceinline__ JoinRow join_row(const Kv4AttentionParams& p, int seq, int64_t begin, int64_t end, int64_t token) {
    const int64_t len = p.lengths[seq];
    JoinRow r;
    r.live = token >= begin && token < end;
    r.bad = len > (int64_t)p.columns * p.cache.page;
    r.keys = r.bad || len < 0 ? 0 : max((int)len - (int)(end - begin) + (int)(token - begin) + 1, 0);
    return r;
}

// The parts of one row (query and head) joined, a workgroup to a row: threads take four elements each, groups of
// threads the parts in turn, eight in flight.
template <typename T>
__global__ __launch_bounds__(256) void k_join_row(Kv4AttentionParams p, int run, int chunks, const float* part,
                                              const float2* stats) {
    __shared__ float sums[256][4];
    __shared__ float tops[256], totals[256];
    const int64_t row = blockIdx.x, token = row / p.q.heads;
    const int head = (int)(row % p.q.heads);
    JoinRow jr;
    if (p.starts) {
        const Tile t = find_sequence(p.starts, p.seqs, p.tokens, token);
        if (t.seq < 0) return;
        jr = join_row(p, t.seq, t.begin, t.end, token);
    } else {
        jr = join_row(p, (int)token, token, token + 1, token);
    }
    if (!jr.live) return;
    const int used = (jr.keys + run - 1) / run;
    const int d = 32 * p.cache.groups, per = d / 4, groups = 256 / per;
    const int e = 4 * (threadIdx.x % per), grp = threadIdx.x / per;
    const float2* st = stats + row * chunks;
    const float* pt = part + row * chunks * d + e;
    float m = kNegInf, l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    if (grp < groups)
        for (int c0 = grp; c0 < used; c0 += 8 * groups) {
            float2 s[8];
            f32x4 v[8];
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const int c = c0 + k * groups;
                s[k] = make_float2(kNegInf, 0.0f), v[k] = f32x4{0, 0, 0, 0};
                if (c < used) s[k] = st[c], v[k] = *(const f32x4*)(pt + (int64_t)c * d);
            }
            float now = m;
#pragma unroll
            for (int k = 0; k < 8; k++) now = fmaxf(now, s[k].x);
            const float f = m == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m - now);
            l *= f, o *= f, m = now;
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const float g = s[k].x == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(s[k].x - m);
                l = fmaf(g, s[k].y, l);
                o += v[k] * g;
            }
        }
    tops[threadIdx.x] = m;
    totals[threadIdx.x] = l;
    *(f32x4*)sums[threadIdx.x] = o;
    __syncthreads();
    if (grp) return;
    for (int w = 1; w < groups; w++) m = fmaxf(m, tops[threadIdx.x + w * per]);
    l = 0.0f, o = f32x4{0, 0, 0, 0};
    for (int w = 0; w < groups; w++) {
        const int at = threadIdx.x + w * per;
        const float f = tops[at] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(tops[at] - m);
        l += f * totals[at];
        o += *(const f32x4*)sums[at] * f;
    }
    if (jr.bad) o = f32x4{0, 0, 0, 0} + __builtin_nanf("");
    else if (jr.keys) o *= 1.0f / l;
    typedef T t4 __attribute__((ext_vector_type(4)));
    ((Loose<t4, T>*)((T*)p.o.p + token * p.o.token + head * p.o.head + e))->v = __builtin_convertvector(o, t4);
}

// The parts of an item joined, `rows` of its R rows: threads to four elements each, sets of threads the parts in turn,
// eight in flight.  ITEMS: a workgroup has the item of its number, else the last one that workgroup blockIdx.x began.
template <typename T, bool ITEMS>
__global__ __launch_bounds__(256) void k_join_items(Kv4AttentionParams p, int R, int rows, int count, const float* part,
                                              const float2* stats) {
    __shared__ float sums[256][4];
    __shared__ float tops[256], totals[256];
    __shared__ int kept[4][6][64];
    Kv4Walk walk(p, kept, R, count);
    if (walk.total == 0) return;
    Kv4Item it;
    int w = blockIdx.x;
    if (ITEMS) {
        it = walk.item(w);
        w = it.begin / walk.per;
    } else {
        const int u1 = min((w + 1) * walk.per, walk.total);
        if (w * walk.per >= u1) return;
        it = walk.item(u1 - 1, u1);
        if (it.begin < w * walk.per) return;
    }
    const int u0 = w * walk.per, parts = (it.end - 1) / walk.per - w + 1;
    if (it.end <= it.begin || parts == 1) return;
    const int d = 32 * p.cache.groups, per = d / 4, sets = 256 / per / rows;
    const int e = 4 * (threadIdx.x % per), set = threadIdx.x / per / rows;
    const int row = blockIdx.y * rows + threadIdx.x / per % rows;
    const int r = it.rw.row0 + row, t = r / p.group, head = it.h * p.group + r % p.group;
    const bool live = set < sets && r < it.rw.rows;
    auto place = [&](int k) { return (int64_t)(2 * (w + k) + (k == 0 && it.begin > u0 ? 1 : 0)) * R + row; };
    float m = kNegInf, l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    if (live)
        for (int k0 = set; k0 < parts; k0 += 8 * sets) {
            float2 s[8];
            f32x4 v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int k = k0 + i * sets;
                s[i] = make_float2(kNegInf, 0.0f), v[i] = f32x4{0, 0, 0, 0};
                if (k < parts) s[i] = stats[place(k)], v[i] = *(const f32x4*)(part + place(k) * d + e);
            }
            float now = m;
#pragma unroll
            for (int i = 0; i < 8; i++) now = fmaxf(now, s[i].x);
            const float f = m == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m - now);
            l *= f, o *= f, m = now;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float g = s[i].x == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(s[i].x - m);
                l = fmaf(g, s[i].y, l);
                o += v[i] * g;
            }
        }
    tops[threadIdx.x] = m;
    totals[threadIdx.x] = l;
    *(f32x4*)sums[threadIdx.x] = o;
    __syncthreads();
    if (set || !live) return;
    const int step = per * rows;
    for (int k = 1; k < sets; k++) m = fmaxf(m, tops[threadIdx.x + k * step]);
    l = 0.0f, o = f32x4{0, 0, 0, 0};
    for (int k = 0; k < sets; k++) {
        const int at = threadIdx.x + k * step;
        const float f = tops[at] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(tops[at] - m);
        l += f * totals[at];
        o += *(const f32x4*)sums[at] * f;
    }
    if (it.rw.bad) o = f32x4{} + __builtin_nanf("");
    else if (it.rw.len - it.rw.n + t >= 0) o *= 1.0f / l;      // no key: zeros
    typedef T t4 __attribute__((ext_vector_type(4)));
    ((Loose<t4, T>*)((T*)p.o.p + (it.rw.begin + t) * p.o.token + head * p.o.head + e))->v = __builtin_convertvector(o, t4);
}

// At most kRuns parts: a thread to four elements of a row.
template <typename T>
__global__ __launch_bounds__(256) void k_join_runs(Kv4AttentionParams p, int run, int chunks, const float* part,
                                                  const float2* stats) {
    const int d = 32 * p.cache.groups, per = d / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / per, token = row / p.q.heads;
    const int head = (int)(row % p.q.heads), e = 4 * (int)(id % per);
    if (token >= p.tokens) return;
    // every part that there may be is on its way before the row's keys are known
    const float2* st = stats + row * chunks;
    const float* pt = part + row * chunks * d + e;
    float2 s[kRuns];
    f32x4 v[kRuns];
#pragma unroll
    for (int c = 0; c < kRuns; c++)
        if (c < chunks) s[c] = st[c], v[c] = *(const f32x4*)(pt + (int64_t)c * d);
    JoinRow jr;
    if (p.starts) {
        // the sequence of the workgroup's first token, then on from there
        const Tile t = find_sequence(p.starts, p.seqs, p.tokens, (int64_t)blockIdx.x * 256 / per / p.q.heads);
        int seq = t.seq;
        while (seq + 1 < p.seqs && p.starts[seq + 1] <= token) seq++;
        if (seq < 0) return;
        const int64_t a = min(max((int64_t)p.starts[seq], (int64_t)0), p.tokens);
        const int64_t b = min(max((int64_t)p.starts[seq + 1], a), p.tokens);
        jr = join_row(p, seq, a, b, token);
    } else {
        jr = join_row(p, (int)token, token, token + 1, token);
    }
    if (!jr.live) return;
    const int used = min((jr.keys + run - 1) / run, chunks);
    float m = kNegInf, l = 0.0f;
#pragma unroll
    for (int c = 0; c < kRuns; c++) {
        if (c >= used) s[c] = make_float2(kNegInf, 0.0f), v[c] = f32x4{0, 0, 0, 0};
        m = fmaxf(m, s[c].x);
    }
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < kRuns; c++) {
        const float f = s[c].x == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(s[c].x - m);
        l = fmaf(f, s[c].y, l);
        o += v[c] * f;
    }
    if (jr.bad) o = f32x4{0, 0, 0, 0} + __builtin_nanf("");
    else if (jr.keys) o *= 1.0f / l;
    typedef T t4 __attribute__((ext_vector_type(4)));
    ((Loose<t4, T>*)((T*)p.o.p + token * p.o.token + head * p.o.head + e))->v = __builtin_convertvector(o, t4);
}

Kv4Split split(int64_t tokens, int q_heads, int d, int kv_heads, int seqs, bool starts, int64_t longest) {
    Kv4Split s = {};
    const int group = q_heads / kv_heads, cus = num_cus();
    const int64_t rows = starts ? (tokens + seqs - 1) / seqs * group : group;      // of a sequence, on average
    const int cp = d <= 64 ? 2 : d <= 128 ? 4 : 8, narrow = 16 / cp;      // rows of a tile whose columns are (row, group)
    // Few rows: to one tile of short heads, to two of others.  64 sequences, us in tiles of (row, group) and in tiles of 16
    // rows: heads of 64, 16 rows of 8192 keys 101 and 87; of 128, 8 rows of 4096 70 and 70; of 256, 4 rows of 4096 152 and
    // 249.  Many: past 64 rows.  64 sequences of 2048 keys in tiles of 16 and of 128 rows: 64 rows 138 and 145, 96 rows 196
    // and 150 (eight sequences: 28 and 39, 41 and 50).
    s.kind = rows <= (cp == 2 ? 1 : 2) * narrow ? kKv4Few : rows <= 64 ? kKv4Some : kKv4Many;
    s.NT = rows <= (s.kind == kKv4Few ? narrow : s.kind == kKv4Some ? 16 : 192) || (s.kind != kKv4Few && d > 128) ? 1 : 2;
    s.R = (s.kind == kKv4Few ? narrow : s.kind == kKv4Some ? 16 : 128) * s.NT;
    s.chunks = 1;
    s.tiles = (group + s.R - 1) / s.R;
    s.slots = starts ? tokens * group / s.R + seqs : (int64_t)seqs * s.tiles;
    const int64_t tiles = starts ? std::max(tokens * group / s.R, std::min((int64_t)seqs, tokens)) : s.slots;      // about
    if (s.kind != kKv4Many) {
        // workgroups that run at once, by the registers that their kernels take
        const int few = cp * s.NT == 2 ? 4 : cp * s.NT == 4 ? 3 : cp * s.NT == 8 ? 2 : 1;
        const int some = cp * s.NT == 2 ? 3 : cp * s.NT == 4 ? 2 : 1;
        const int64_t at_once = cus * (s.kind == kKv4Few ? few : some), base = s.slots * kv_heads;
        // Even shares of the work, where there is much: heavy workgroups from four units each on (64 sequences of 2048
        // keys, heads of 128: 8 queries of 4 heads 71 us, 134 in runs; 2 queries 41 and 63; 16 sequences of 1024, 8
        // queries 21 and 30).  They cost two to seven us more where there is little (one sequence of 32768, one query
        // of 4 heads 18 and 15 in runs; 64 of 512, 24 and 12).  Workgroups of one tile are light enough that whole
        // contexts fill the card (64 of 8192 keys: 121 and 108; as many ragged ones 82 and 81), but a sequence of 32768
        // by itself takes 207 whole: shares for contexts from 4096 on, which may be as different as that.  Tiles of long
        // heads have no registers for it (256: 8 queries 277, 240 in runs).  Of thousands of sequences there are enough
        // workgroups without, and each would go over all their lengths.
        const bool light = s.kind == kKv4Few && s.NT == 1;
        if (base * ((longest + 127) / 128) >= (light ? 16 : 4) * at_once && longest >= (light ? 4096 : 256) &&
            (s.kind == kKv4Few || d <= 128) && seqs <= kMostEven) {
            s.count = (int)at_once;
            return s;
        }
        // Whole to 4096 keys, or runs of a power of two up to 2048, so that one long sequence is not left alone (runs of 3,
        // 5 or 6 times 128 measured up to a fifth slower than those of 4 and 8), whichever takes the least time, counted in
        // about 2.1 ns: a key of a head of 128 takes three alone on a CU, five beside another workgroup, eight beside two;
        // a workgroup 1430 before and after its keys, the join 1900 and ten a part.  One query of 4 heads, us in runs of
        // 512, 1024, 2048: a sequence of 32768 keys 16.4, 16.8, 23.2; of 131072 39, 35, 31; 64 of 2048 35, 35 and, whole,
        // 27; 256 of 1024 68 and, whole, 54.
        const double key = cp / 4.0 * s.NT * (s.kind == kKv4Few ? 1 : 2);
        auto time = [&](int64_t run, int64_t parts) {
            const int64_t workgroups = tiles * kv_heads * parts;
            auto round = [&](int64_t some) {      // of so many workgroups at once
                const int64_t beside = (some + cus - 1) / cus;
                return some ? run * key * (beside == 1 ? 3 : beside == 2 ? 5 : 3 * beside - 1) + 1430.0 : 0.0;
            };
            return workgroups / at_once * round(at_once) + round(workgroups % at_once) +
                   (parts > 1 ? 1900.0 + 10.0 * parts : 0.0);
        };
        int64_t best = longest <= 4096 ? std::max((longest + 127) / 128 * 128, (int64_t)128) : 2048;
        double least = time(best, (longest + best - 1) / best);
        for (int64_t run = 128; run < longest && run <= 2048; run *= 2) {
            const double t = time(run, (longest + run - 1) / run);
            if (t < least) least = t, best = run;
        }
        s.run = (int)best;
        s.chunks = std::max((int)((longest + best - 1) / best), 1);
        return s;
    }
    // What takes the least time: rounds of as many workgroups as run at once (256 rows a CU, 128 of long heads), each
    // as long as its part of the keys; and the join, which moves a part's sums in about the time of 1700 keys.  Heads of
    // 128, 32 over 8, us: two sequences of 8192 keys and 512 queries 290 whole, 192 in two parts; 16 of 2048 and 64 queries
    // 87 and 122.  Or even shares, of which each workgroup and each tile leaves a part: for sequences of different
    // lengths, which runs of one length do not fit, where they are not a fifth behind (two ragged ones of up to 512 over
    // 8192 172 -> 146, two equal ones 217 and 222, one of 16384 179 and 191); where the first queries of a tile see few
    // of its keys the shares would not be even.
    const int64_t base = tiles * kv_heads, at_once = (d > 128 ? 1 : 2 / s.NT) * cus;
    int64_t n = 1;
    double least = 0.0;
    for (int64_t m = 1; m <= kRuns && 576 * (m - 1) < longest; m++) {
        const double rounds = (double)((base * m + at_once - 1) / at_once) / m;
        const double time = rounds + (m > 1 ? 1700.0 * m / longest * base / at_once : 0.0);
        if (m == 1 || time < least) least = time, n = m;
    }
    const double even = (double)base / at_once + 1700.0 / longest * (base + at_once) / at_once;
    if (even < (seqs > 1 ? 1.2 : 1.0) * least && d <= 128 && 4 * (rows / group) <= longest &&
        seqs <= kMostEven) {
        s.count = (int)at_once;
        return s;
    }
    const int64_t run = std::max(((longest + n - 1) / n + 127) / 128 * 128, (int64_t)128);
    s.run = (int)run;
    s.chunks = std::max((int)((longest + run - 1) / run), 1);
    return s;
}

// Rows of partial sums that a call keeps.
int64_t places(const Kv4Split& s, int64_t rows) {
    return s.count ? (int64_t)2 * s.count * s.R : s.chunks > 1 ? rows * s.chunks : 0;
}
size_t stats_bytes(int64_t places) { return ((size_t)places * sizeof(float2) + 255) & ~(size_t)255; }

template <typename T, int CP, bool FULL, bool EVEN>
hipError_t launch_cp(const Kv4AttentionParams& p, const Kv4Split& sp, float* part, float2* stats, hipStream_t s) {
    const unsigned grid = (unsigned)(EVEN ? sp.count : sp.slots * p.cache.heads * sp.chunks);
    if (sp.kind == kKv4Few) {
        if (sp.NT == 1) k_kv4_few<T, CP, 1, FULL, EVEN><<<grid, 256, 0, s>>>(p, sp, part, stats);
        else if constexpr (CP > 2) k_kv4_few<T, CP, 2, FULL, EVEN><<<grid, 256, 0, s>>>(p, sp, part, stats);
    } else if constexpr (!EVEN || CP < 8) {
        // long heads: one tile, two would not fit the registers, nor one with what an even share takes
        if (sp.NT == 1) k_kv4<T, CP, 1, FULL, EVEN><<<grid, 256, 0, s>>>(p, sp, part, stats);
        else k_kv4<T, CP, CP == 8 ? 1 : 2, FULL, EVEN><<<grid, 256, 0, s>>>(p, sp, part, stats);
    }
    return hipGetLastError();
}

template <typename T, bool EVEN>
hipError_t launch_d(const Kv4AttentionParams& p, const Kv4Split& sp, float* part, float2* stats, hipStream_t s) {
    if (p.d == 64) return launch_cp<T, 2, true, EVEN>(p, sp, part, stats, s);
    if (p.d == 128) return launch_cp<T, 4, true, EVEN>(p, sp, part, stats, s);
    if (p.d == 256) return launch_cp<T, 8, true, EVEN>(p, sp, part, stats, s);
    if (p.d < 64) return launch_cp<T, 2, false, EVEN>(p, sp, part, stats, s);
    if (p.d < 128) return launch_cp<T, 4, false, EVEN>(p, sp, part, stats, s);
    return launch_cp<T, 8, false, EVEN>(p, sp, part, stats, s);
}

template <typename T>
hipError_t launch_t(int type, const Kv4AttentionParams& p, hipStream_t s) {
    const Kv4Split sp = split(p.tokens, p.q.heads, p.d, p.cache.heads, p.seqs, p.starts != nullptr,
                              (int64_t)p.columns * p.cache.page);
    const int64_t rows = p.tokens * p.q.heads;
    float2* stats = (float2*)p.ws;
    float* part = (float*)(p.ws + stats_bytes(places(sp, rows)));
    if (sp.count) {
        const hipError_t e = sp.kind == kKv4Many ? launch_kv4_many(type, p, sp, part, stats, s)
                                                 : launch_d<T, true>(p, sp, part, stats, s);
        if (e != hipSuccess) return e;
        // As many rows as fit, or four workgroups to an item of many parts.
        const bool items = sp.slots * p.cache.heads < sp.count;
        int at_a_time = 8 * sp.slots * p.cache.heads < sp.count ? std::max(sp.R / 4, 1) : sp.R;
        while (at_a_time * (p.d / 4) > 256) at_a_time /= 2;
        const dim3 grid((unsigned)(items ? sp.slots * p.cache.heads : sp.count), sp.R / at_a_time);
        auto join = items ? k_join_items<T, true> : k_join_items<T, false>;
        join<<<grid, 256, 0, s>>>(p, sp.R, at_a_time, sp.count, part, stats);
        return hipGetLastError();
    }
    const hipError_t e = sp.kind == kKv4Many ? launch_kv4_many(type, p, sp, part, stats, s)
                                             : launch_d<T, false>(p, sp, part, stats, s);
    if (e != hipSuccess || sp.chunks == 1) return e;
    const int64_t threads = rows * (p.d / 4);
    const unsigned blocks = (unsigned)((threads + 255) / 256);
    if (sp.chunks <= kRuns) k_join_runs<T><<<blocks, 256, 0, s>>>(p, sp.run, sp.chunks, part, stats);
    else k_join_row<T><<<(unsigned)rows, 256, 0, s>>>(p, sp.run, sp.chunks, part, stats);
    return hipGetLastError();
}

}  // namespace

size_t kv4_attention_workspace(int64_t tokens, int q_heads, int d, int kv_heads, int seqs, bool starts,
                               int64_t longest) {
    const Kv4Split s = split(tokens, q_heads, d, kv_heads, seqs, starts, longest);
    const int64_t n = places(s, tokens * q_heads);
    return n ? stats_bytes(n) + (size_t)n * d * sizeof(float) : 0;
}

bool kv4_attention_counts(int64_t tokens, int q_heads, int d, int kv_heads, int seqs, bool starts, int64_t longest) {
    const Kv4Split s = split(tokens, q_heads, d, kv_heads, seqs, starts, longest);
    const int64_t group = q_heads / kv_heads;
    if (tokens * group > INT32_MAX - 256) return false;
    if (!s.count) return s.slots * kv_heads <= INT32_MAX / s.chunks;
    return s.slots * kv_heads <= (1 << 30) / ((longest + 127) / 128 + 1);
}

hipError_t launch_kv4_attention(int type, const Kv4AttentionParams& p, hipStream_t s) {
    return type == kBF16 ? launch_t<__bf16>(type, p, s) : launch_t<_Float16>(type, p, s);
}

}  // namespace esb
