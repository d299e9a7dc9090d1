// Attention over the 4-bit paged cache for many rows (a prompt or a part of one): kv4_attention.hip's definition, in
// the form of attention.hip.  A workgroup of 128 or 256 rows, 32 to a wave, decodes a tile of 64 keys and values once,
// with their scales, into LDS as fp16, where its waves read it.
//
// E2M1 times a bf16 scale has ten bits: exact in fp16, where its range allows.  So a tile's key scales are
// brought below 2^(kUp + 1) by a power of two (which the scores get back with the scale of the softmax), a row of bf16
// queries to the end of fp16 likewise, and the value scales by the largest exponent met so far (when it grows, the
// sums follow).  Then scales down to 2^-kSpread of the largest keep all their bits, elements of a query down to 2^-32.  The
// products are fp16 MFMAs for both types of queries; probabilities are rounded to fp16.
//
// Larger keys and values that a row does not see, or gives no weight, must not cost it the bits of those that it
// sees.  So where scales or a query's elements lie further apart, the item is gone over once more in the form of
// kv4_attention.hip (wide_pass), whose scales stay fp32: codes and queries as they are into the MFMAs, a key's scale on
// the sum of its group, a value's on the probability, which enters as two bf16.  Looking for that costs -3 to 3 % (heads of
// 64 to 128, us, without and with: the two ragged sequences below 141 and 141, 2048 queries over 8192 keys 300 and 305, 64
// over 2048 33.9 and 34.6), and heads of 256 nothing (268).  Scales below 2^-125 are those of zeros: they are not
// looked for, so that zeros among other tokens stay as fast.
//
// Values whose scale is not finite count as zero in the products, and their elements become NaN at the end for
// the rows that see them.
#include <type_traits>

#include "attend.h"

namespace esb {

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t bits(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ f16x2 halves(uint32_t v) { return __builtin_bit_cast(f16x2, v); }

// The two nibbles of each byte of w, as fp16.
__device__ __forceinline__ void pairs(uint32_t w, f16x2 (&o)[4]) {
    o[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0));
    o[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1));
    o[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2));
    o[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3));
}
__device__ __forceinline__ float bf16_value(uint32_t b) { return __uint_as_float(b << 16); }
// Exponent field of a bf16 scale, 0 where it is not finite.
__device__ __forceinline__ int exponent(uint32_t b) {
    const int e = (b >> 7) & 0xff;
    return e == 0xff ? 0 : e;
}
constexpr int kUp = 12;          // a tile's largest scale is brought to this exponent: times 6 it is within fp16
constexpr int kSpread = 28;      // 2^(kUp - kSpread) in eight bits times 0.5 is a multiple of 2^-24, fp16's smallest step
constexpr int kBias = 127 + kUp;
constexpr int kMost = 80 - kUp;      // values below 2^84 under weights of up to 2^8 have sums within fp32
// Whether a scale of at least 2^-125 lies too far below 2^(e + kUp): is_below(scale, limit(e)).
__device__ __forceinline__ uint32_t limit(int e) { return (uint32_t)max(e + kBias - kSpread - 2, 0); }
__device__ __forceinline__ bool is_below(uint32_t b, uint32_t limit) { return (b >> 7 & 0xff) - 2u < limit; }
template <int CTRL> __device__ __forceinline__ int turned(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
// The value of lane k of four.
__device__ __forceinline__ uint32_t of_four(uint32_t v, int k) {
    return (uint32_t)(k == 0 ? turned<0x00>((int)v) : k == 1 ? turned<0x55>((int)v) : k == 2 ? turned<0xaa>((int)v) : turned<0xff>((int)v));
}
// The largest of a wave's values, in every lane.
__device__ __forceinline__ int wave_max(int v) {
    v = max(v, turned<0xb1>(v));       // lanes 1 0 3 2 of four
    v = max(v, turned<0x4e>(v));       // lanes 2 3 0 1
    v = max(v, turned<0x141>(v));      // eight lanes mirrored
    v = max(v, turned<0x140>(v));      // sixteen
    return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
               max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

// Bound by the matrix cores and VALU in turn, and by what the fewest tiles leave idle: 2048 queries of 32 heads of 128
// over 16384 keys 583 to 635 us by card, 870 to 940 TFLOP/s; two ragged sequences of up to 512 over 8192 keys 141, 596.
// Decoded in registers by each wave it was 378, into LDS by four waves 236, scales shared by the
// lanes of a group 191, by eight waves for twice the rows 172, in even shares 146, each with the join.
template <typename T, int DP, int WAVES, bool EVEN>
__global__ __launch_bounds__(64 * WAVES, DP == 256 ? 1 : 2)
void k_kv4_many(Kv4AttentionParams p, Kv4Split sp, float* part, float2* stats) {
    typedef typename Vec8<T>::type V;
    constexpr int KT = 64, R = 32 * WAVES, P = DP / 8, CP = DP / 32, DB = DP / 32;
    __shared__ f16x8 kt[2][KT * P];              // rows of keys, pieces turned
    __shared__ f16x8 vt[2][KT / 8 * DP];         // [16 keys][half][element]: keys 4 half .. + 3 and 8 + 4 half .. + 3
    __shared__ _Float16 vscales[WAVES][16 / WAVES][4 * CP];      // a wave's: [run][group][key of the run]
    __shared__ int2 peaks[2][WAVES];             // by wave: largest exponents of the key and the value scales
    __shared__ int odd;                          // some value's scale is not finite
    __shared__ int wide;                         // scales, or a query's elements, lie too far apart
    __shared__ int kept[EVEN ? WAVES : 1][6][64];
    Work<EVEN> work(p, sp, R, kept);
    while (work.next()) {
        int tid = threadIdx.x;
        if (EVEN) asm volatile("" : "+v"(tid));      // nothing of the lane is kept from item to item: registers are short
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int col = lane & 31, half = lane >> 5, C = p.cache.groups;
        const Rows& rw = work.rw;
        const int h = work.h;
        const int first = rw.len - rw.n;                    // the last key of query t is first + t
        auto last_of = [&](int r) { return first + r / p.group; };
        const int keys = max(last_of(min(rw.row0 + R, rw.rows) - 1) + 1, 0);
        const int k0 = work.from, k1 = min(work.to, keys);
        if (!EVEN && !work.whole && k0 >= k1) return;       // the join does not look at it

        const int row = rw.row0 + 32 * wave + col;
        const bool live = row < rw.rows, alive = rw.row0 + 32 * wave < rw.rows;      // the lane's row, any of the wave's
        const int last = last_of(row), wave_open = last_of(rw.row0 + 32 * wave);
        const int head = h * p.group + row % p.group;
        const int64_t token = rw.begin + row / p.group;

        Attend<_Float16, DP, KT> fl;
        fl.start();
        int q_exponent = 0;
        bool q_wide = false;
        {
            V raw[DP / 16];
            uint32_t most = 0, least = ~0u;
            const T* q = (const T*)p.q.p + token * p.q.token + head * p.q.head;
#pragma unroll
            for (int s = 0; s < DP / 16; s++) {
                const int e = 16 * s + 8 * half;
                raw[s] = V{};
                if (live && e < p.d) raw[s] = load8(q + e, 8);
                const f32x8 v = __builtin_convertvector(raw[s], f32x8);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
                    if (b <= 0x7f800000u) most = max(most, b);
                    least = min(least, b - 1);      // but for zero
                }
            }
            most = max(most, (uint32_t)__shfl_xor((int)most, 32));
            if (std::is_same<T, __bf16>::value && most && most < 0x7f800000u) {
                q_exponent = (int)(most >> 23) - 127 - 15;
                q_wide = (least >> 23) + 32 < (most >> 23);
            }
#pragma unroll
            for (int s = 0; s < DP / 16; s++) {
                f32x8 v = __builtin_convertvector(raw[s], f32x8);
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] = __builtin_amdgcn_ldexpf(v[i], -q_exponent);
                fl.qf[s] = __builtin_convertvector(v, f16x8);
            }
        }

        // A thread's part of a tile: the words of CT groups (all, or with eight waves half of them) of one key,
        // elements 8 a4 of a group on; and of a run of four values (of the same page), elements 2 a16 of a group on.
        // Of the scales it brings one of its key's (two for CT = 8), those of its groups by a4, and those of its run
        // that lie a16 (and 16 further) on; the others' come from its neighbours.
        constexpr int H = WAVES / 4, CT = CP / H, NK = CT == 8 ? 2 : 1, NV = CP == 8 ? 2 : 1;
        typedef uint32_t WT __attribute__((ext_vector_type(CT)));
        const int key = tid / (4 * H), a4 = tid & 3, run4 = tid / (16 * H), a16 = tid & 15;
        const int gk = H == 2 ? CT * (tid >> 2 & 1) : 0, gv = H == 2 ? CT * (tid >> 4 & 1) : 0;      // first groups
        const int32_t* table = p.table + rw.seq * p.table_pitch;
        const int page = p.cache.page;
        WT kw, vw;
        uint32_t ka[NK], va[NV];
        // a wave's keys lie in sixteen in a row, so in one page
        const int wave_key = __builtin_amdgcn_readfirstlane(key & ~15), in16 = key & 15;
        const uint32_t k_at = in16 * 16 * C + a4 * 4 * C + 4 * gk, v_at = (in16 >> 2) * 64 * C + a16 * 4 * C + 4 * gv;
        auto page_of = [&](int j0) { return table[min(j0 + wave_key, keys - 1) >> p.cache.shift]; };
        auto load = [&](int j0, int pid) {
            pid = __builtin_amdgcn_readfirstlane(pid);
            const bool bad = pid < 0 || pid >= p.cache.pages;
            const int t = (j0 + wave_key) & (page - 1);
            // words past the head's groups are of what follows in the block, and meet zeros of the query or make
            // outputs that are not stored; their scales repeat others
            const uint8_t* b = p.cache.block(bad ? 0 : pid, h);
            kw = ((const Loose<WT, uint32_t>*)(b + t * 16 * C + k_at))->v;
            vw = ((const Loose<WT, uint32_t>*)(b + p.cache.values_at() + t * 16 * C + v_at))->v;
            const uint8_t* ks = b + p.cache.key_scales_at() + p.cache.scale_run(t);
            const uint8_t* vs = b + p.cache.value_scales_at() + p.cache.scale_run(t);
            const uint32_t run = (in16 >> 2) * 8 * C;
#pragma unroll
            for (int u = 0; u < NK; u++) {
                ka[u] = *(const uint16_t*)(ks + (run + 8 * min(gk + a4 % CT + 4 * u, C - 1) + 2 * (in16 & 3)));
                if (bad) ka[u] = 0x7fc0u;
                if (j0 + key >= keys) ka[u] = 0;      // scales behind the last key may be anything
            }
#pragma unroll
            for (int u = 0; u < NV; u++) {
                const int n = min(a16 + 16 * u, 4 * C - 1);
                va[u] = *(const uint16_t*)(vs + (run + 2 * n));
                if (j0 + 4 * run4 + (n & 3) >= keys) va[u] = 0;
            }
        };
        auto put_peaks = [&](int stage) {
            int k = exponent(ka[0]), v = exponent(va[0]);
            if (NK == 2) k = max(k, exponent(ka[NK - 1]));
            if (NV == 2) v = max(v, exponent(va[NV - 1]));
            k = wave_max(k), v = wave_max(v);
            if (lane == 0) peaks[stage][wave] = make_int2(k, v);
        };
        auto peak = [&](int stage) {
            int2 m = peaks[stage][0];
#pragma unroll
            for (int w = 1; w < WAVES; w++) m.x = max(m.x, peaks[stage][w].x), m.y = max(m.y, peaks[stage][w].y);
            return make_int2(m.x - kBias, m.y - kBias);
        };
        // The tile that was brought, as fp16 under the two exponents: share() first, then decoded() in registers, then
        // put() into LDS, so that the arithmetic may run beside products of the other stage.
        uint32_t ks[NK];      // key scales, twice in one word
        uint2 vs4[CT];        // value scales of the run
        u32x4 kd[CT], vd[CT];
        auto share = [&](int ke, int ve) {
            _Float16* own = vscales[wave][run4 & (4 / H - 1)];
            const uint32_t lk = limit(ke), lv = limit(ve);
            bool below = false;
#pragma unroll
            for (int u = 0; u < NV; u++) {
                const float v = bf16_value(va[u]);
                const bool fine = fabsf(v) < __builtin_inff();
                if (!fine) odd = 1;
                below |= is_below(va[u], lv);
                if (CP >= 4 || a16 < 8) own[a16 + 16 * u] = fine ? (_Float16)__builtin_amdgcn_ldexpf(v, -ve) : (_Float16)0.0f;
            }
#pragma unroll
            for (int u = 0; u < NK; u++) {
                below |= is_below(ka[u], lk);
                const _Float16 k = (_Float16)__builtin_amdgcn_ldexpf(bf16_value(ka[u]), -ke);
                ks[u] = bits(f16x2{k, k});
            }
            if (__builtin_expect(__ballot(below) != 0, 0)) wide = 1;
            __builtin_amdgcn_wave_barrier();      // LDS serves a wave in order
#pragma unroll
            for (int g = 0; g < CT; g++) vs4[g] = ((const uint2*)own)[gv + g];
            __builtin_amdgcn_wave_barrier();
        };
        auto decoded = [&]() {
#pragma unroll
            for (int g = 0; g < CT; g++) {
                f16x2 o[4];
                pairs(kw[g], o);
                const f16x2 s = halves(of_four(ks[g / 4], g % 4));
                kd[g] = u32x4{bits(o[0] * s), bits(o[1] * s), bits(o[2] * s), bits(o[3] * s)};
                const f16x2 s01 = halves(vs4[g].x), s23 = halves(vs4[g].y);
                pairs(vw[g], o);      // o[t]: the two elements of key t
                const uint32_t e01 = __builtin_amdgcn_perm(bits(o[1]), bits(o[0]), 0x05040100);
                const uint32_t e23 = __builtin_amdgcn_perm(bits(o[3]), bits(o[2]), 0x05040100);
                const uint32_t o01 = __builtin_amdgcn_perm(bits(o[1]), bits(o[0]), 0x07060302);
                const uint32_t o23 = __builtin_amdgcn_perm(bits(o[3]), bits(o[2]), 0x07060302);
                vd[g] = u32x4{bits(halves(e01) * s01), bits(halves(e23) * s23), bits(halves(o01) * s01), bits(halves(o23) * s23)};
            }
        };
        auto put = [&](int stage) {
            uint2* vo = (uint2*)&vt[stage][((run4 >> 2) * 2 + (run4 & 1)) * DP + 32 * gv + 2 * a16] + (run4 >> 1 & 1);
#pragma unroll
            for (int g = 0; g < CT; g++) {
                kt[stage][key * P + ((4 * (gk + g) + a4) ^ key_turn<DP>(key))] = __builtin_bit_cast(f16x8, kd[g]);
                vo[64 * g] = uint2{vd[g][0], vd[g][1]};
                vo[64 * g + 2] = uint2{vd[g][2], vd[g][3]};
            }
        };

        if (tid == 0) odd = wide = 0;
        int ke = 0, ve = -kBias, ve_first = -kBias;
        if (k0 < k1) {
            load(k0, page_of(k0));
            int next = page_of(k0 + KT);
            put_peaks(0);
            __syncthreads();
            ke = peak(0).x, ve = ve_first = peak(0).y;
            if (q_wide || ve > kMost) wide = 1;
            share(ke, ve);
            decoded();
            put(0);
            load(k0 + KT, next), next = page_of(k0 + 2 * KT);
            // Past the last tile the same goes on with its last key's page, under scales of zero.
            for (int j0 = k0, stage = 0; j0 < k1; j0 += KT, stage ^= 1) {
                put_peaks(stage ^ 1);
                __syncthreads();      // this tile is there; the next one's peaks are; no one reads the other stage any more
                const int ke_next = peak(stage ^ 1).x, ve_next = max(ve, peak(stage ^ 1).y);
                share(ke_next, ve_next);
                if (alive) {
                    fl.scores(kt[stage]);
                    decoded();
#pragma unroll
                    for (int i = 0; i < DP / 8; i++) {      // between the MFMAs
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                     // LDS read
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                     // MFMA
                        __builtin_amdgcn_sched_group_barrier(0x002, H == 2 ? 4 : 7, 0);        // VALU
                    }
                } else {
                    decoded();
                }
                put(stage ^ 1);
                load(j0 + 2 * KT, next), next = page_of(j0 + 3 * KT);
                if (alive) {
                    const f16x8* vs = vt[stage];
                    // at least the smallest normal number, under which all scores are as good as zero: a zero would make
                    // masked ones, -infinity, NaN; and no infinity, which would make NaN of scores of zero
                    const float scale = __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(p.scale, q_exponent + ke), 0x1p-126f,
                                                                0x1.fffffep127f);
                    fl.weights(scale, j0 + KT - 1 > wave_open, last - j0 - 4 * half);
                    fl.products([&](int r, int d) { return vs[((r >> 4) * 2 + half) * DP + 32 * d + col]; });
                    if (ve_next > ve) {
                        const float f = __builtin_amdgcn_ldexpf(1.0f, max(ve - ve_next, -126));
#pragma unroll
                        for (int d = 0; d < DB; d++) fl.acc[d] *= f;
                        // sums keep their bits while they come down by less than 2^60; before ve_first there were zeros
                        if (ve < 2 - kBias) ve_first = ve_next;
                        if (ve_next - ve_first > 60 || ve_next > kMost) wide = 1;
                    }
                }
                ke = ke_next, ve = ve_next;
            }
            __syncthreads();
            if (__builtin_expect(wide, 0)) {
                if (alive)
                    wide_pass<T, EVEN>(p, rw, h, k0, k1, rw.row0 + 32 * wave, ~0u,
                                       work.whole ? -1 : EVEN ? (int64_t)work.place * R + 32 * wave : work.place, sp.chunks, part, stats);
                if (!EVEN) return;
                __syncthreads();
                continue;
            }
            if (__builtin_expect(odd, 0)) {
                for (int j = k0; j < k1; j++) {
                    const int pid = table[j >> p.cache.shift];
                    if (pid < 0 || pid >= p.cache.pages) continue;
                    const int t = j & (page - 1);
                    const uint8_t* vs = p.cache.block(pid, h) + p.cache.value_scales_at() + p.cache.scale_run(t) + (t & 3) * 2;
#pragma unroll
                    for (int d = 0; d < DB; d++) {
                        const uint32_t b = *(const uint16_t*)(vs + 8 * min(d, C - 1));
                        if ((b & 0x7f80) == 0x7f80 && j <= last) fl.acc[d] = f32x16{} + __builtin_nanf("");
                    }
                }
            }
        }

        const float sum = fl.sum + other_half(fl.sum);
        if (live) {
            const bool whole = work.whole;
            const int64_t to = EVEN ? (int64_t)work.place * R + 32 * wave + col
                                    : (token * p.q.heads + head) * sp.chunks + work.place;
            const float f = !whole ? 1.0f : last >= 0 ? 1.0f / sum : 0.0f;       // no key: zeros
            if (!whole && half == 0) stats[to] = make_float2(fl.top, sum);
            T* o = (T*)p.o.p + token * p.o.token + head * p.o.head;
#pragma unroll
            for (int d = 0; d < DB; d++)
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const int e = 32 * d + 8 * k + 4 * half;
                    if (e >= p.d) continue;
                    f32x4 w;
#pragma unroll
                    for (int i = 0; i < 4; i++) w[i] = __builtin_amdgcn_ldexpf(fl.acc[d][4 * k + i] * f, ve);
                    if (!whole) {
                        *(f32x4*)(part + to * p.d + e) = w;
                    } else {
                        if (rw.bad) w = f32x4{0, 0, 0, 0} + __builtin_nanf("");
                        typedef T t4 __attribute__((ext_vector_type(4)));
                        ((Loose<t4, T>*)(o + e))->v = __builtin_convertvector(w, t4);
                    }
                }
        }
        if (EVEN) __syncthreads();      // the next item uses the same LDS
    }
}

template <typename T, int DP>
hipError_t launch_d(const Kv4AttentionParams& p, const Kv4Split& sp, float* part, float2* stats, hipStream_t s) {
    // long heads: eight waves a CU would not fit the registers
    constexpr int most = DP == 256 ? 4 : 8;
    if (sp.count) {
        if constexpr (DP < 256) {
            if (sp.NT == 1) k_kv4_many<T, DP, 4, true><<<sp.count, 256, 0, s>>>(p, sp, part, stats);
            else k_kv4_many<T, DP, most, true><<<sp.count, 64 * most, 0, s>>>(p, sp, part, stats);
        }
        return hipGetLastError();
    }
    const unsigned grid = (unsigned)(sp.slots * p.cache.heads * sp.chunks);
    if (sp.NT == 1) k_kv4_many<T, DP, 4, false><<<grid, 256, 0, s>>>(p, sp, part, stats);
    else k_kv4_many<T, DP, most, false><<<grid, 64 * most, 0, s>>>(p, sp, part, stats);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const Kv4AttentionParams& p, const Kv4Split& sp, float* part, float2* stats, hipStream_t s) {
    if (p.d <= 64) return launch_d<T, 64>(p, sp, part, stats, s);
    if (p.d <= 128) return launch_d<T, 128>(p, sp, part, stats, s);
    return launch_d<T, 256>(p, sp, part, stats, s);
}

}  // namespace

hipError_t launch_kv4_many(int type, const Kv4AttentionParams& p, const Kv4Split& sp, float* part, float2* stats,
                           hipStream_t s) {
    return type == kBF16 ? launch_t<__bf16>(p, sp, part, stats, s) : launch_t<_Float16>(p, sp, part, stats, s);
}

}  // namespace esb
