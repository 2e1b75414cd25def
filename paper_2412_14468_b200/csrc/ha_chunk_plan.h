// How the attention of new tokens is dealt out over the CTAs (plain arithmetic, included by ha_chunk.cu; compiles for the host).
//
// A unit is one KV head of one sequence and up to 256 query rows: 256 / G consecutive new tokens times the G query heads of the
// group.  Its work is a number of key tiles of 128 tokens.  All tiles of all units, in the order (sequence, KV head, unit, tile),
// lie on one line, each as long as its cost, and CTA c of C takes the stretch [W c / C, W (c + 1) / C) of it: every CTA has the same
// work whatever the lengths are, a long cache with one new token is split over many CTAs, and consecutive units of a CTA read the
// same keys.  A unit that a boundary cuts is finished by the last of its parts to arrive (see ha_chunk.cu).
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define HA_HD __host__ __device__ __forceinline__
#else
#define HA_HD inline
#endif
// Numbers that a kernel in front may have written after this one began: past L1, which may hold what was there before.
#ifdef __CUDA_ARCH__
#define HA_FROM_L2(p) __ldcg(p)
#else
#define HA_FROM_L2(p) (*(p))
#endif

namespace ha {

constexpr int kChunkRows = 256;                    // query rows of a unit: two tiles of 128
constexpr int kChunkTile = 128;                    // tokens of a key tile
// Cost of a key tile: two units for two row tiles; one where 128 rows or fewer let the two halves of a CTA take tiles in turn.
constexpr int kChunkCostPair = 2, kChunkCostSplit = 1, kChunkCostMost = 2;
// What a unit costs besides its tiles (its rows to fetch, results to write, the pipeline to fill: about 5 us, of pairs of tiles that take 1.9).
constexpr int kChunkFixedPair = 8, kChunkFixedSplit = 2;

struct ChunkSeq {   // one sequence
    int n, cnt, row0;                              // cached tokens, new ones among them, first row of q
    int units;                                     // per KV head
};
struct ChunkUnit {
    int tok0, toks, tiles, cost, fixed;            // first new token, new tokens, key tiles, cost of one, of the unit besides
    int first_pos;                                 // cache position of tok0 (< 0 where a sequence has more new tokens than cached ones)
    bool split;
    HA_HD long long total() const { return (long long)tiles * cost + fixed; }
};

HA_HD int chunk_tokens_per_unit(int log2g) { return kChunkRows >> log2g; }

// Offsets that do not describe rows of q (bad) count as no new tokens.
HA_HD ChunkSeq chunk_seq(int seq_len, int off0, int off1, int n_rows, int log2g, bool &bad) {
    ChunkSeq s;
    s.n = seq_len > 0 ? seq_len : 0;
    s.row0 = off0;
    bad = off0 < 0 || off1 < off0 || off1 > n_rows;
    s.cnt = bad ? 0 : off1 - off0;
    const int t = chunk_tokens_per_unit(log2g);
    s.units = (int)(((long long)s.cnt + t - 1) >> (8 - log2g));
    return s;
}

static_assert(kChunkRows == 256 && kChunkTile == 128, "shifts by 8 and 7 below");
HA_HD int chunk_tiles(long long hi) { return hi <= kChunkTile ? 1 : (int)((hi + kChunkTile - 1) >> 7); }

HA_HD ChunkUnit chunk_unit(const ChunkSeq &s, int u, int log2g, bool causal) {
    ChunkUnit r;
    const int t = chunk_tokens_per_unit(log2g);
    r.tok0 = u * t;
    r.toks = s.cnt - r.tok0 < t ? s.cnt - r.tok0 : t;
    r.split = (r.toks << log2g) <= kChunkRows / 2;
    r.cost = r.split ? kChunkCostSplit : kChunkCostPair;
    r.fixed = r.split ? kChunkFixedSplit : kChunkFixedPair;
    r.first_pos = s.n - s.cnt + r.tok0;
    r.tiles = chunk_tiles(causal ? (long long)r.first_pos + r.toks : (long long)s.n);
    return r;
}

// a / b for a >= 0, b > 0; most fit 32 bits, whose division takes a tenth of the time
HA_HD long long chunk_div(long long a, long long b) {
    return ((unsigned long long)(a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

// sum over y = 1 .. x of floor(y / 2^lk)
HA_HD long long chunk_floor_sum(long long x, int lk) {
    const long long t = x >> lk, r = x & ((1 << lk) - 1);
    return ((t * (t - 1) / 2) << lk) + t * (r + 1);
}

// Cost of units 0 .. u - 1 of one KV head, all of them with all their tokens (u <= units, the last unit apart).
HA_HD long long chunk_cost_full_units(const ChunkSeq &s, int u, int log2g, bool causal) {
    if (u <= 0) return 0;
    const long long fixed = (long long)u * kChunkFixedPair;
    if (!causal) return fixed + (long long)u * chunk_tiles(s.n) * kChunkCostPair;
    const int t = chunk_tokens_per_unit(log2g);
    const long long a = (long long)s.n - s.cnt;     // tokens in front of the new ones; negative: units that see nothing cost one tile
    long long m = u, skipped = 0;
    if (a < 0) {                                    // units whose last position lies below 1 have one tile
        skipped = (-a) >> (8 - log2g);
        if (skipped > m) skipped = m;
    }
    // unit i (counted from 1) sees a + i t tokens: ceil((a + i t) / 128) tiles
    const long long base = a + skipped * t + kChunkTile - 1;
    m -= skipped;
    long long tiles = skipped;
    if (m == 0) return fixed + tiles * kChunkCostPair;
    if (t == 2 * kChunkTile) {
        // floor((base + 256 i) / 128) = floor(base / 128) + 2 i, base >= -255 + 127
        const long long q = base >> 7;              // rounds down
        tiles += m * q + m * (m + 1);
    } else {
        // k = 128 / t: floor((base + i t) / 128) = floor((floor(base / t) + i) / k)
        const int lk = log2g - 1;
        const long long q = base >> (8 - log2g);    // base > 127 - t >= -1
        tiles += chunk_floor_sum(q + m, lk) - chunk_floor_sum(q, lk);
    }
    return fixed + tiles * kChunkCostPair;
}

HA_HD long long chunk_cost_head(const ChunkSeq &s, int log2g, bool causal) {
    if (s.units == 0) return 0;
    const ChunkUnit last = chunk_unit(s, s.units - 1, log2g, causal);
    return chunk_cost_full_units(s, s.units - 1, log2g, causal) + last.total();
}

// CTAs that share W: every stretch is at least as long as the dearest tile, so that no part in the middle of a unit is empty.
HA_HD int chunk_ctas(long long W, int most) {
    const long long c = W / kChunkCostMost;
    return c < 1 ? 1 : c < most ? (int)c : most;
}
HA_HD long long chunk_bound(long long W, int C, int c) { return chunk_div(W * c, C); }
HA_HD int chunk_cta_of(long long W, int C, long long x) { return (int)chunk_div((x + 1) * C - 1, W); }
// first tile of a unit beginning at u0 that a stretch beginning at f takes; the unit's fixed cost lies in front of its tiles
HA_HD int chunk_first_tile(long long f, long long u0, const ChunkUnit &u) {
    const long long g = f - u0 - u.fixed;
    if (g <= 0) return 0;
    const long long t = chunk_div(g + u.cost - 1, u.cost);
    return t < u.tiles ? (int)t : u.tiles;
}

// The parts of a CTA's stretch in order.
struct ChunkWalk {
    long long W, f0, f1, u0;
    int C, log2g, B, Hkv, n_rows;
    bool causal;
    const int32_t *seq_lens, *offsets;
    int b, h, u;
    ChunkSeq s;
    ChunkUnit unit;
    int t0, t1;                                    // tiles of the current part
    bool cut;                                      // the unit has other parts
    int first_cta, n_parts;

    HA_HD void load() {
        bool bad;
        s = chunk_seq(HA_FROM_L2(seq_lens + b), HA_FROM_L2(offsets + b), HA_FROM_L2(offsets + b + 1), n_rows, log2g, bad);
    }
    // the unit that holds position f0, which lies `rest` behind the beginning of sequence b_
    HA_HD void begin(int cta, int b_, long long rest) {
        f0 = chunk_bound(W, C, cta);
        f1 = chunk_bound(W, C, cta + 1);
        b = b_;
        load();
        const long long per_head = chunk_cost_head(s, log2g, causal);
        h = (int)chunk_div(rest, per_head);
        rest -= h * per_head;
        int lo = 0, hi = s.units - 1;              // the last unit that begins at or before `rest`
        while (lo < hi) {
            const int mid = lo + (hi - lo + 1) / 2;
            if (chunk_cost_full_units(s, mid, log2g, causal) <= rest) lo = mid;
            else hi = mid - 1;
        }
        u = lo;
        u0 = f0 - (rest - chunk_cost_full_units(s, u, log2g, causal));
        --u;
        unit.tiles = unit.cost = unit.fixed = 0;
        first_cta = n_parts = 0;
    }
    // false: no part is left
    HA_HD bool next() {
        for (;;) {
            u0 += unit.total();
            if (++u >= s.units) {
                u = 0;
                if (++h >= Hkv) {
                    h = 0;
                    do {
                        if (++b >= B) return false;
                        load();
                    } while (s.cnt == 0);
                }
            }
            if (u0 >= f1) return false;
            unit = chunk_unit(s, u, log2g, causal);
            t0 = chunk_first_tile(f0, u0, unit);
            t1 = chunk_first_tile(f1, u0, unit);
            if (t0 < t1) break;
        }
        cut = t0 > 0 || t1 < unit.tiles;
        if (cut) {
            first_cta = chunk_cta_of(W, C, u0 + unit.fixed);
            int last = chunk_cta_of(W, C, u0 + unit.total() - 1);
            if (chunk_first_tile(chunk_bound(W, C, last), u0, unit) >= unit.tiles) --last;
            n_parts = last - first_cta + 1;
        }
        return true;
    }
};

} // namespace ha
