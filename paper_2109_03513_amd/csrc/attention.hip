// Attention over packed prompts: o = softmax(scale q k^T) v, per sequence, causal or not, query heads in groups
// that share a key head.
//
// A workgroup takes 128 rows (queries x heads of one group), 32 to a wave, and goes over the sequence's
// keys in tiles that its waves share in LDS.  The scores are formed transposed, S^T = K Q^T, on 32x32x16 MFMAs:
// a lane then holds, of one query, the keys that the second product O^T = V^T P^T wants of its operand, so
// that the probabilities never leave their lane; V^T is read from the row-major tile by the
// transposing LDS read.  One pass with a running maximum and sum; the maximum moves only when a score
// passes it by 2^8, so most tiles scale nothing.  Probabilities are rounded to the type of v for the MFMA
// (their sum is not): an error of the terms that is below the rounding of the output.
#include <type_traits>

#include "attend.h"

namespace esb {

namespace {

constexpr float kLarge = 0x1p15f;    // in bf16 and fp16

typedef short i16x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) const void lds_void;

// 16 bytes a lane, from base + at of each, to LDS from the wave's place on.  Written out, so that reads of the other
// stage do not wait for it: the compiler takes every LDS read behind a DMA for one of its data.  The
// caller waits for vmcnt(0) before the barrier that hands the tile over.  (m0 is reserved: nothing else here uses it.)
__device__ __forceinline__ void dma16(const void* base, uint32_t at, const void* wave_place) {
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)wave_place);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(lds), "v"(at), "s"(base) : "memory");
}
// Values of a tile are rows of DP / 8 16-byte pieces too, piece c at c ^ value_turn(row), so that the 64 bytes that
// a transposing read takes of eight rows lie in distinct banks.
template <int DP> __device__ __forceinline__ int value_turn(int row) { return DP == 64 ? (row >> 1 & 1) * 4 : (row & 3) * 4; }

template <typename T> __device__ __forceinline__ bool finite(T v) {
    constexpr uint16_t e = std::is_same<T, __bf16>::value ? 0x7f80 : 0x7c00;
    return (__builtin_bit_cast(uint16_t, v) & e) != e;
}

// Bound by MFMA and VALU issue (50 and 47 % of all SIMD cycles; they add up) at a power-limited clock: causal prompts,
// heads of 128, 527 to 559 us by card for 550 GFLOP, 1.0 PFLOP/s, where a library product reaches 1.22.  Tiles by loads to
// registers 1110 us, by DMA in two stages 582, that written out 529.  32 rows to a wave and 64 keys to a tile: what
// the registers of two workgroups a CU hold.
// KS: sets of four waves that take every KS-th tile, each in stages of its own, and join their sums at the end.  FULL: heads
// of DP elements; else their rows end before the tiles'.
template <typename T, int DP, int KT, int KS, bool DMA, bool FULL>
__global__ __launch_bounds__(256 * KS, DP == 256 ? 1 : 2) void k_attention(AttentionParams p) {
    typedef typename Vec8<T>::type V;
    constexpr int R = 128, P = DP / 8, NP = KT * P / 256, DB = DP / 32;
    __shared__ V all_tiles[KS][2][2][KT * P];      // two stages of keys and values
    __shared__ float2 other_stats[KS == 2 ? 256 : 1];
    __shared__ int odd;                    // some tile with masks holds values that are not finite
    const int set = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & 255;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    V (&tiles)[2][2][KT * P] = all_tiles[set];
    const int h = blockIdx.x % p.k.heads;
    const int64_t slot = gridDim.x / p.k.heads - 1 - blockIdx.x / p.k.heads;      // the longest rows first
    const int k_start = p.seqs < 64 ? p.k_starts[min(lane, p.seqs)] : 0;
    const Tile t = find_tile(p.q_starts, p.seqs, p.q_tokens, p.group, R, slot, nullptr, nullptr);
    const int n = (int)(t.end - t.begin), rows = n * p.group;
    if (t.index < 0 || (int64_t)t.index * R >= rows) return;
    const int row0 = t.index * R;
    const int k_from = p.seqs < 64 ? __builtin_amdgcn_readlane(k_start, t.seq) : p.k_starts[t.seq];
    const int k_to = p.seqs < 64 ? __builtin_amdgcn_readlane(k_start, t.seq + 1) : p.k_starts[t.seq + 1];
    const int64_t ka = min(max((int64_t)k_from, (int64_t)0), p.k_tokens);
    const int nk = (int)(min(max((int64_t)k_to, ka), p.k_tokens) - ka);
    const int ahead = p.causal ? nk - n : nk;        // query i sees keys up to i + ahead
    auto last_of = [&](int r) { return min(r / p.group + ahead, nk - 1); };
    const int keys = last_of(min(row0 + R, rows) - 1) + 1;

    const int row = row0 + 32 * wave + col;
    const bool live = row < rows;
    const int last = last_of(row);
    const int open = last_of(row0), wave_open = last_of(row0 + 32 * wave);      // every row sees keys up to here
    const int wave_keys = row0 + 32 * wave < rows ? last_of(min(row0 + 32 * wave + 32, rows) - 1) + 1 : 0;

    Attend<T, DP, KT> fl;
    fl.start();
    {
        const T* q = (const T*)p.q.p + (t.begin + row / p.group) * p.q.token + (h * p.group + row % p.group) * p.q.head;
#pragma unroll
        for (int s = 0; s < DP / 16; s++) {
            const int e = 16 * s + 8 * half;
            fl.qf[s] = V{};
            if (live && e < p.d) fl.qf[s] = load8(q + e, 8);
        }
    }
    const T* kp = (const T*)p.k.p + ka * p.k.token + h * p.k.head;
    const T* vp = (const T*)p.v.p + ka * p.v.token + h * p.v.head;

    // A tile into LDS.  Rows past the last key repeat the last one, and are masked.  Pieces past the head are zeros from the
    // start on for keys, as an infinity would make NaN of the query's zeros, and repeat the last one for values, whose outputs
    // there are not stored.
    const int most = p.d / 8 - 1, piece = tid % P, r0 = tid / P;
    constexpr int RU = 256 / P;                 // rows that the workgroup brings at a time
    // pieces by the row's turn, which repeats after two of them
    const int ck[2] = {8 * min(piece ^ key_turn<DP>(r0), most), 8 * min(piece ^ key_turn<DP>(r0 + RU), most)};
    const int cv[2] = {8 * min(piece ^ value_turn<DP>(r0), most), 8 * min(piece ^ value_turn<DP>(r0 + RU), most)};
    auto held = [&](int u) { return FULL || (piece ^ key_turn<DP>(r0 + (u & 1) * RU)) <= most; };
    if (!FULL)
#pragma unroll
        for (int u = 0; u < NP; u++)
            if (!held(u)) tiles[0][0][tid + 256 * u] = tiles[1][0][tid + 256 * u] = V{};
    const int k_pitch = (int)p.k.token, v_pitch = (int)p.v.token;      // DMA: tiles' offsets fit 32 bits
    auto fetch = [&](int j0, int stage) {
        const T* kb = kp + (int64_t)j0 * p.k.token;
        const T* vb = vp + (int64_t)j0 * p.v.token;
        const int end = nk - 1 - j0;
        if (DMA) {
            const int place = 64 * wave;
            const bool all = end >= KT - 1;
            auto key = [&](int u) {
                const int r = all ? r0 : min(r0 + u * RU, end);
                dma16(all ? kb + (int64_t)(u * RU) * p.k.token : kb, 2 * (uint32_t)(r * k_pitch + ck[u & 1]), &tiles[stage][0][place + 256 * u]);
            };
            auto value = [&](int u) {
                const int r = all ? r0 : min(r0 + u * RU, end);
                dma16(all ? vb + (int64_t)(u * RU) * p.v.token : vb, 2 * (uint32_t)(r * v_pitch + cv[u & 1]), &tiles[stage][1][place + 256 * u]);
            };
            if (!FULL)      // lanes apart, whose pieces are the same ones in every row, or every other one
#pragma unroll
                for (int turn = 0; turn < (DP == 256 ? 2 : 1); turn++)
                    if (held(turn)) {
                        if (all) {
#pragma unroll
                            for (int u = turn; u < NP; u += DP == 256 ? 2 : 1) key(u);
                        } else {
#pragma unroll 1
                            for (int u = turn; u < NP; u += DP == 256 ? 2 : 1) key(u);
                        }
                    }
            if (all) {
#pragma unroll
                for (int u = 0; u < NP; u++) {
                    if (FULL) key(u);
                    value(u);
                }
            } else {
#pragma unroll 1
                for (int u = 0; u < NP; u++) {
                    if (FULL) key(u);
                    value(u);
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < NP; u++) {
                const int64_t r = min(r0 + u * RU, end);
                if (held(u)) tiles[stage][0][tid + 256 * u] = load8(kb + r * p.k.token + ck[u & 1], 8);
                tiles[stage][1][tid + 256 * u] = load8(vb + r * p.v.token + cv[u & 1], 8);
            }
        }
    };

    // Keys r .. r + 3 and r + 8 .. r + 11 of element 32 d + lane % 32, by the 16 lanes that hold them row by row.
    auto values = [&](const V* vt, int r, int d) {
        typedef short i16x8 __attribute__((ext_vector_type(8)));
        typedef __attribute__((address_space(3))) i16x4* lds;
        const int e = 32 * d + 16 * (lane >> 4 & 1) + 4 * (lane & 3);
        auto four = [&](int row) {
            return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds)((T*)vt + (row * P + ((e >> 3) ^ value_turn<DP>(row))) * 8 + (e & 7)));
        };
        const i16x4 lo = four(r + ((lane & 15) >> 2)), hi = four(r + 8 + ((lane & 15) >> 2));
        const i16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(V, v);
    };
    if (tid == 0) odd = 0;
    if (KT * set < keys) fetch(KT * set, 0);
    for (int first = 0, stage = 0; first < keys; first += KT * KS, stage ^= 1) {
        const int j0 = first + KT * set;
        if (DMA) __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0): this wave's part of the tile
        __syncthreads();                                  // everyone's; and no one reads the other stage any more
        if (j0 + KT * KS < keys) fetch(j0 + KT * KS, stage ^ 1);
        const V* kt = tiles[stage][0];
        V* vt = tiles[stage][1];
        if (first + KT * KS - 1 > open) {
            // values that are not finite would reach every row: zeros here, the rows that see them below
            bool mine = false;
            if (j0 < keys)
#pragma unroll 1
                for (int u = 0; u < NP; u++) {
                    V v = vt[tid + 256 * u];
                    bool any = false;
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        if (!finite(v[i])) v[i] = (T)0.0f, any = true;
                    if (any) vt[tid + 256 * u] = v;
                    mine |= any;
                }
            if (mine) odd = 1;
            __syncthreads();
        }
        if (j0 >= wave_keys) continue;
        fl.scores(kt);
        fl.weights(p.scale, j0 + KT - 1 > wave_open, last - j0 - 4 * half);
        fl.products([&](int r, int d) { return values(vt, r, d); });
    }
    if constexpr (KS == 2) {
        __syncthreads();
        float* other = (float*)all_tiles + tid;
        if (set == 1) {
            other_stats[tid] = make_float2(fl.top, fl.sum);
#pragma unroll
            for (int d = 0; d < DB; d++)
#pragma unroll
                for (int i = 0; i < 16; i++) other[256 * (16 * d + i)] = fl.acc[d][i];
        }
        __syncthreads();
        if (set == 1) return;
        const float2 o = other_stats[tid];
        const float now = fmaxf(fl.top, o.x);
        const float f = fl.top == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(fl.top - now);
        const float g = o.x == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(o.x - now);
        fl.sum = fl.sum * f + o.y * g;
#pragma unroll
        for (int d = 0; d < DB; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) fl.acc[d][i] = fl.acc[d][i] * f + other[256 * (16 * d + i)] * g;
    } else if (keys > 0) {
        __syncthreads();
    }
    if (keys > 0 && odd) {
        // a multiple of a number that overflows for every such value that a row sees, by products with ones
        const int from = max(open + 1, 0) / (KT * KS) * (KT * KS);
#pragma unroll
        for (int d = 0; d < DB; d++) {
            f32x16 up = {}, down = {};
            const int e = 32 * d + col;
#pragma unroll 1
            for (int j0 = from; j0 < keys; j0 += 16) {
                V plus, minus, sees;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int j = j0 + 8 * half + i;
                    const T v = j < nk && e < p.d ? vp[(int64_t)j * p.v.token + e] : (T)0.0f;
                    plus[i] = finite(v) || v < (T)0.0f ? (T)0.0f : (T)kLarge;
                    minus[i] = finite(v) || v > (T)0.0f ? (T)0.0f : (T)-kLarge;
                    sees[i] = j <= last ? (T)1.0f : (T)0.0f;
                }
                up = mma(plus, sees, up);
                down = mma(minus, sees, down);
            }
#pragma unroll
            for (int i = 0; i < 16; i++) {      // the products overflow, and inf - inf is NaN
                fl.acc[d][i] += up[i] * 0x1p126f;
                fl.acc[d][i] += down[i] * 0x1p126f;
            }
        }
    }

    const float sum = fl.sum + other_half(fl.sum);
    if (!live) return;
    const float f = last >= 0 ? 1.0f / sum : 0.0f;       // no key: zeros
    T* o = (T*)p.o.p + (t.begin + row / p.group) * p.o.token + (h * p.group + row % p.group) * p.o.head;
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int e = 32 * d + 8 * k + 4 * half;
            if (e >= p.d) continue;
            typedef T t4 __attribute__((ext_vector_type(4)));
            f32x4 w;
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = fl.acc[d][4 * k + i] * f;
            ((Loose<t4, T>*)(o + e))->v = __builtin_convertvector(w, t4);
        }
}

// Whether DMA takes the rows: 16-byte pieces, and a tile's rows within 32-bit offsets.
template <typename T> bool dma_takes(const HeadsView& v) {
    return (uintptr_t)v.p % 16 == 0 && v.token % 8 == 0 && (v.heads == 1 || v.head % 8 == 0) && v.token < (1 << 24);
}

template <typename T, int DP, int KT, bool FULL>
hipError_t launch_d(const AttentionParams& p, hipStream_t s) {
    const int64_t slots = p.q_tokens * p.group / 128 + p.seqs;
    const unsigned grid = (unsigned)(slots * p.k.heads);
    const bool dma = dma_takes<T>(p.k) && dma_takes<T>(p.v);
    // Few workgroups: their keys in two sets of waves (causal, heads of 128, one set and two: 1024 tokens of 32 heads 29.0
    // and 25.6 us, 4096 of 4 heads 85 and 64), unless there are many or the keys are short (4096 tokens of 32 heads 158
    // and 174, eight sequences of 512 43 and 56).  Long heads have no registers for a second set.
    if constexpr (DP < 256)
        if (grid <= 2u * num_cus() && p.k_tokens >= (int64_t)256 * p.seqs) {
            if (dma) k_attention<T, DP, KT, 2, true, FULL><<<grid, 512, 0, s>>>(p);
            else k_attention<T, DP, KT, 2, false, FULL><<<grid, 512, 0, s>>>(p);
            return hipGetLastError();
        }
    if (dma) k_attention<T, DP, KT, 1, true, FULL><<<grid, 256, 0, s>>>(p);
    else k_attention<T, DP, KT, 1, false, FULL><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const AttentionParams& p, hipStream_t s) {
    if (p.d == 64) return launch_d<T, 64, 64, true>(p, s);
    if (p.d == 128) return launch_d<T, 128, 64, true>(p, s);
    if (p.d == 256) return launch_d<T, 256, 32, true>(p, s);
    if (p.d < 64) return launch_d<T, 64, 64, false>(p, s);
    if (p.d < 128) return launch_d<T, 128, 64, false>(p, s);
    return launch_d<T, 256, 32, false>(p, s);
}

}  // namespace

hipError_t launch_attention(int type, const AttentionParams& p, hipStream_t s) {
    return type == kBF16 ? launch_t<__bf16>(p, s) : launch_t<_Float16>(p, s);
}

}  // namespace esb
