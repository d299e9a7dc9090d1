// Heads of a decoder's attention, and the 4-bit paged cache of its keys and values: what heads.hip,
// kv4_attention.hip, attention.hip and the C ABI share.
#pragma once

#include "float_rows.h"

namespace esb {

// Element i of head h of token t at p[t * token + h * head + i].
struct HeadsView {
    void* p;
    int64_t token, head;
    int heads;
};

// A page holds `page` tokens (a power of two, at least 16) of every head, one block per head after
// the other.  With G = d / 32 scale groups a block has 36 G bytes a token:
//   keys    [token][4][G] words: the eight nibbles of elements 32 g + 8 a .. + 7 in word (a, g),
//   values  [token / 4][16][G][token % 4] bytes: elements 32 g + 2 a, + 1 in byte (a, g),
//   scales  of keys, then of values: [token / 4][G][token % 4] bf16.
// So one 16-byte piece is what a lane of a 16x16x32 MFMA wants of a key (every G, its eight
// elements of the contraction) and of four values (every G, its two rows of the output).
struct Kv4Layout {
    uint8_t* data;
    int64_t pages;
    int page, shift, heads, groups;
    __host__ __device__ int64_t block_bytes() const { return (int64_t)36 * groups * page; }
    __device__ __forceinline__ uint8_t* block(int64_t pg, int head) const {
        return data + (pg * heads + head) * block_bytes();
    }
    __device__ __forceinline__ int values_at() const { return 16 * groups * page; }
    __device__ __forceinline__ int key_scales_at() const { return 32 * groups * page; }
    __device__ __forceinline__ int value_scales_at() const { return 34 * groups * page; }
    // Scales start of the four-token run that holds token t of the block.
    __device__ __forceinline__ int scale_run(int t) const { return (t >> 2) * 8 * groups; }
};

// Norm and rotation of heads, and their way into the cache (heads.hip).
struct HeadsParams {
    HeadsView q, k, v, qo, ko;      // v only with a cache; ko only without
    int64_t tokens;
    int d;
    const float* qw;                // norm weights, or NULL (ones)
    const float* kw;
    float eps;                      // 0: no norm
    double inv_d;                   // 1 / d
    const float* table;             // rows x rot: cosines, then sines
    int64_t rows;
    int rot, adjacent;              // rot 0: no rotation
    const int32_t* positions;
    const int64_t* slots;           // with a cache
    Kv4Layout cache;
};
hipError_t launch_rope(int type, const HeadsParams& p, hipStream_t s);
hipError_t launch_kv4_append(int type, const HeadsParams& p, hipStream_t s);
// Codes (ESB(4,1), one a byte) and scales [tokens][heads][d], [tokens][heads][d / 32], contiguous, in and
// out (values as E4M3 bytes); any of the four may be NULL on the way out.
hipError_t launch_kv4_pack(const Kv4Layout& L, int64_t tokens, const int64_t* slots, const uint8_t* k,
                           const void* ka, const uint8_t* v, const void* va, hipStream_t s);
hipError_t launch_kv4_unpack(const Kv4Layout& L, int64_t tokens, const int64_t* slots, uint8_t* k, void* ka,
                             uint8_t* v, void* va, hipStream_t s);

// Attention over the cache (kv4_attention.hip).
struct Kv4AttentionParams {
    HeadsView q, o;
    int64_t tokens;
    Kv4Layout cache;
    int d, group;                   // query heads per key head
    int seqs;
    const int32_t* starts;          // seqs + 1, or NULL: one token each
    const int32_t* lengths;
    const int32_t* table;           // pages of a sequence, pitch in elements
    int64_t table_pitch;
    int columns;
    float scale;                    // of the products, times log2(e)
    uint8_t* ws;
};
// How a call is split, from what the host knows (kv4_attention.hip).
struct Kv4Split {
    int kind;            // kKv4Few, kKv4Some, kKv4Many: which kernel
    int NT, R;           // row tiles of a wave; rows of a workgroup
    int count;           // workgroups that share the work evenly; 0: each has a run of a tile's keys
    int tiles;           // tiles of a sequence of one query
    int64_t slots;       // tiles of all sequences
    int run, chunks;     // keys of a workgroup, and how many there are of such runs
};
constexpr int kKv4Few = 0, kKv4Some = 1, kKv4Many = 2;
// The kernel of many rows (kv4_prompt.hip): R of them to a workgroup.
hipError_t launch_kv4_many(int type, const Kv4AttentionParams& p, const Kv4Split& sp, float* part, float2* stats,
                           hipStream_t s);
size_t kv4_attention_workspace(int64_t tokens, int q_heads, int d, int kv_heads, int seqs, bool starts,
                               int64_t longest);
// Whether the call's workgroups and units of work are within 32 bits.
bool kv4_attention_counts(int64_t tokens, int q_heads, int d, int kv_heads, int seqs, bool starts, int64_t longest);
hipError_t launch_kv4_attention(int type, const Kv4AttentionParams& p, hipStream_t s);

// Attention over packed prompts (attention.hip).
struct AttentionParams {
    HeadsView q, k, v, o;
    int64_t q_tokens, k_tokens;
    int d, group, seqs, causal;
    const int32_t* q_starts;        // seqs + 1 each
    const int32_t* k_starts;
    float scale;                    // of the products, times log2(e)
};
hipError_t launch_attention(int type, const AttentionParams& p, hipStream_t s);

// The sequence that tile `slot` belongs to, where the sequences' tiles of R rows are numbered from
// first(s) = starts[s] * per / R + s (per rows a token): no sequence has more tiles than lie between
// its own number and the next one's, so that tiles need no list.  Every lane of the wave gets the
// answer; the starts may hold anything.
struct Tile {
    int seq, index;        // index: of the sequence's tiles
    int64_t begin, end;    // its tokens
};
// The sequence of a token: the last one that starts at it or before (seq < 0: none).
__device__ __forceinline__ Tile find_sequence(const int32_t* starts, int seqs, int64_t tokens, int64_t token) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int s0 = 0; s0 < seqs; s0 += 64)
        n += __builtin_popcountll(__ballot(s0 + lane < seqs && starts[min(s0 + lane, seqs - 1)] <= token));
    Tile t;
    t.seq = __builtin_amdgcn_readfirstlane(n - 1), t.index = 0;
    t.begin = t.end = 0;
    if (t.seq < 0) return t;
    t.begin = min(max((int64_t)starts[t.seq], (int64_t)0), tokens);
    t.end = min(max((int64_t)starts[t.seq + 1], t.begin), tokens);
    return t;
}
__device__ __forceinline__ Tile find_tile(const int32_t* starts, int seqs, int64_t tokens, int per, int R, int64_t slot,
                                          const int32_t* lengths, int* length) {
    const int lane = threadIdx.x & 63;
    Tile t;
    int64_t a, b;
    if (seqs < 64) {      // starts and lengths in one trip to memory
        const int start = starts[min(lane, seqs)], kept = lengths ? lengths[min(lane, seqs - 1)] : 0;
        const bool before = lane < seqs && (int64_t)max(start, 0) * per / R + lane <= slot;
        t.seq = max(__builtin_popcountll(__ballot(before)) - 1, 0);
        a = __builtin_amdgcn_readlane(start, t.seq), b = __builtin_amdgcn_readlane(start, t.seq + 1);
        if (lengths) *length = __builtin_amdgcn_readlane(kept, t.seq);
    } else {
        int n = 0;
        for (int s0 = 0; s0 < seqs; s0 += 64) {
            const int s = min(s0 + lane, seqs - 1);
            n += __builtin_popcountll(__ballot(s0 + lane < seqs && (int64_t)max(starts[s], 0) * per / R + s <= slot));
        }
        t.seq = __builtin_amdgcn_readfirstlane(max(n - 1, 0));
        a = starts[t.seq], b = starts[t.seq + 1];
        if (lengths) *length = lengths[t.seq];
    }
    t.begin = min(max(a, (int64_t)0), tokens);
    t.end = min(max(b, t.begin), tokens);
    t.index = (int)(slot - (t.begin * per / R + t.seq));
    return t;
}

// A sequence as one workgroup sees it.
struct Rows {
    int seq, n, len;     // its queries, its cached keys
    int64_t begin;       // its first query
    int row0, rows;      // rows of the tile start here, of all
    bool bad;            // its length passes its pages
};

__device__ __forceinline__ Rows find_rows(const Kv4AttentionParams& p, int64_t slot, int tiles, int R) {
    Rows r;
    int index, kept;
    if (p.starts) {
        const Tile t = find_tile(p.starts, p.seqs, p.tokens, p.group, R, slot, p.lengths, &kept);
        r.seq = t.seq, r.begin = t.begin, r.n = (int)(t.end - t.begin), index = t.index;
    } else {
        r.seq = (int)(slot / tiles), index = (int)(slot % tiles), r.begin = r.seq, r.n = 1;
        kept = p.lengths[r.seq];
    }
    r.rows = r.n * p.group;
    r.row0 = index < 0 || (int64_t)index * R >= r.rows ? r.rows : index * R;
    const int64_t len = kept;
    r.bad = len > (int64_t)p.columns * p.cache.page;
    r.len = r.bad || len < 0 ? 0 : (int)len;
    return r;
}

// Work shared evenly: a unit is 128 keys of one item (tile of R rows, key head, sequence), units are numbered through
// the items, sequences first, then heads, then tiles, and workgroup w of `count` has the units from w * per on,
// whatever items they belong to.  Every wave works this out by itself from the starts and lengths, a sequence to a
// lane, and keeps it in LDS, as registers are short in the loops between.
struct Kv4Item {
    Rows rw;
    int h, begin, end;     // the key head; the item's units
    int from, to;          // its units that were asked for
};
// The sum of v over the lanes up to each: within rows of sixteen, then from row to row.
__device__ __forceinline__ int scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // from the lane 1, 2, 4, 8 below
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // rows 1 and 3: the last of the row before
    return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // rows 2 and 3: lane 31
}

struct Kv4Walk {
    const Kv4AttentionParams& p;
    int (*const kept)[64];            // the wave's, of 64 sequences: units to its end, tiles, steps, queries, keys, begin
    const int R;
    int total, per;                   // units, and of a workgroup
    int s0, before, units;            // the first of those sequences, units before it and of the 64

    __device__ __forceinline__ Kv4Walk(const Kv4AttentionParams& q, int (*lds)[6][64], int rows_of_tile, int count)
        : p(q), kept(lds[threadIdx.x >> 6]), R(rows_of_tile) {
        asm volatile("" ::"s"(count));      // asked for with the first arguments, not when it is used
        total = 0;
        bool falls = false;
        for (int s = 0; s < p.seqs; s += 64) {
            falls |= look(s);
            total += units;
        }
        if (falls) total = 0;      // starts that do not ascend: nothing, as their sum may pass the tokens
        per = (unsigned)(total + count - 1) / (unsigned)count;
        before = 0;
        if (p.seqs > 64) s0 = -64, units = 0;
    }
    __device__ __forceinline__ bool look(int first) {
        const int lane = threadIdx.x & 63, s = first + lane, at = min(s, p.seqs - 1);
        int64_t a = at, b = at + 1;
        bool falls = false;
        if (p.starts) {
            a = p.starts[at], b = p.starts[at + 1], falls = __any(b < a);
            a = min(max(a, (int64_t)0), p.tokens), b = min(max(b, a), p.tokens);
        }
        const int64_t keys = p.lengths[at];
        const bool fits = keys <= (int64_t)p.columns * p.cache.page;
        const int len = fits ? (int)max(keys, (int64_t)0) : -1;      // -1: passes its pages
        const int n = (int)(b - a), tiles = s < p.seqs ? (int)((unsigned)(n * p.group + R - 1) / (unsigned)R) : 0;
        const int steps = max((len + 127) >> 7, 1);
        const int u = scan(tiles * p.cache.heads * steps);
        kept[0][lane] = u, kept[1][lane] = tiles, kept[2][lane] = steps;
        kept[3][lane] = n, kept[4][lane] = len, kept[5][lane] = (int)a;
        __builtin_amdgcn_wave_barrier();
        s0 = first, units = __builtin_amdgcn_readlane(u, 63);
        return falls;
    }
    // The item of unit u, not below those asked for before; of its units those up to `end`.
    __device__ __forceinline__ Kv4Item item(int u, int end) {
        while (u >= before + units) {
            before += units;
            look(s0 + 64);
        }
        const int l = __builtin_ctzll(__ballot(u < before + kept[0][threadIdx.x & 63]));
        const int t = of(1, l), k = of(2, l);
        Kv4Item it = numbered(l, (unsigned)(u - before - of(0, l) + t * p.cache.heads * k) / (unsigned)k);
        it.from = u, it.to = min(it.end, end);
        return it;
    }
    // Item `number` of all, or one of no units.
    __device__ __forceinline__ Kv4Item item(int number) {
        if (s0 < 0) look(0);
        for (;;) {
            const int items = scan(kept[1][threadIdx.x & 63] * p.cache.heads);
            const uint64_t has = __ballot(number < items);
            if (has) {
                const int l = __builtin_ctzll(has);
                return numbered(l, number - __builtin_amdgcn_readlane(items, l) + of(1, l) * p.cache.heads);
            }
            if (s0 + 64 >= p.seqs) return Kv4Item{};
            number -= __builtin_amdgcn_readlane(items, 63), before += units;
            look(s0 + 64);
        }
    }

  private:
    __device__ __forceinline__ int of(int what, int l) { return __builtin_amdgcn_readfirstlane(kept[what][l]); }
    // Item `number` of lane l's sequence.
    __device__ __forceinline__ Kv4Item numbered(int l, int number) {
        Kv4Item it;
        const int t = of(1, l), k = of(2, l), len = of(4, l);
        it.h = (unsigned)number / (unsigned)t;
        it.begin = it.from = before + of(0, l) - (t * p.cache.heads - number) * k, it.end = it.to = it.begin + k;
        it.rw.seq = s0 + l, it.rw.n = of(3, l), it.rw.begin = of(5, l);
        it.rw.bad = len < 0, it.rw.len = max(len, 0);
        it.rw.rows = it.rw.n * p.group, it.rw.row0 = (number - it.h * t) * R;
        return it;
    }
};

// What a workgroup has: keys from .. to - 1 of a tile of rows and a head, item by item.  EVEN: its share of all
// units; else one run of keys, chosen by the host.
template <bool EVEN> struct Work {
    Kv4Walk walk;
    int unit, first, last;
    Rows rw;
    int h, from, to, place;
    bool whole;                       // no other workgroup has keys of it
    __device__ __forceinline__ Work(const Kv4AttentionParams& p, const Kv4Split& sp, int R, int (*kept)[6][64])
        : walk(p, kept, R, sp.count) {
        first = unit = (int)blockIdx.x * walk.per, last = min(unit + walk.per, walk.total);
    }
    __device__ __forceinline__ bool next() {
        if (unit >= last) return false;
        const Kv4Item it = walk.item(unit, last);
        unit = it.to;
        rw = it.rw, h = it.h, from = 128 * (it.from - it.begin), to = 128 * (it.to - it.begin);
        whole = it.from == it.begin && it.to == it.end;
        place = 2 * blockIdx.x + (it.begin > first ? 1 : 0);      // what began before or with its units: 0
        return true;
    }
};
template <> struct Work<false> {
    Rows rw;
    int h, from, to, place;
    bool whole, more;
    __device__ __forceinline__ Work(const Kv4AttentionParams& p, const Kv4Split& sp, int R, int (*)[6][64]) {
        int64_t id = blockIdx.x;
        place = (int)(id % sp.chunks);
        id /= sp.chunks;
        h = (int)(id % p.cache.heads);
        rw = find_rows(p, id / p.cache.heads, sp.tiles, R);
        from = place * sp.run, to = from + sp.run, whole = sp.chunks == 1, more = rw.row0 < rw.rows;
    }
    __device__ __forceinline__ bool next() {
        const bool had = more;
        more = false;
        return had;
    }
};

}  // namespace esb
