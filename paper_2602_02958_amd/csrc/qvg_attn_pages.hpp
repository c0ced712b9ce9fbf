// Where the tokens of an attention over 16-bit pages lie, and how a call is divided: plain arithmetic, the same on the host (where tests
// walk through it) and on the device.
#pragma once
#include "qvg_rows.hpp"

namespace qvg {

struct PgLens { int kv, live; };                    // a sequence's tokens and new tokens, as given

// What a sequence's rows see, together: tokens 0 .. sink - 1 and lo .. kv - 1 (sink < lo, or both 0); and in tiles.
struct PgSpan { int kv, live, sink, lo, sink_tiles, main_tile, total; };
template <bool PAGED>
__host__ __device__ __forceinline__ int pg_tile_of(const PageAttnArgs &a, int n) {
    if (!PAGED) return n / kPgTile;
    const int pi = (int)quotient((uint32_t)n, a.by_page);
    return pi * (int)a.by_tiles.d + (n - pi * (int)a.by_page.d) / kPgTile;
}
template <bool PAGED>
__host__ __device__ __forceinline__ PgSpan pg_span_of(const PageAttnArgs &a, PgLens n) {
    auto clamp = [](int v, int hi) { return v < 0 ? 0 : (v > hi ? hi : v); };
    PgSpan s;
    s.live = clamp(n.live, a.t.n_new);
    s.kv = s.live ? clamp(n.kv, (int)(a.c.table_pages * a.c.page_len)) : 0;      // no row: nothing to read
    s.sink = s.lo = 0;
    const int place = s.kv - s.live;                                     // of the first row
    if (a.t.window > 0 && place >= a.t.window) {
        s.lo = place - a.t.window + 1;
        s.sink = a.t.sink < s.lo ? a.t.sink : s.lo;
        if (s.sink == s.lo) s.sink = s.lo = 0;                           // no gap
    }
    s.sink_tiles = s.sink ? pg_tile_of<PAGED>(a, s.sink - 1) + 1 : 0;
    const int from = s.lo ? pg_tile_of<PAGED>(a, s.lo) : 0, end = s.kv ? pg_tile_of<PAGED>(a, s.kv - 1) + 1 : 0;
    s.main_tile = from > s.sink_tiles ? from : s.sink_tiles;
    s.total = s.sink_tiles + (end > s.main_tile ? end - s.main_tile : 0);
    return s;
}

// A tile: tokens first .. last - 1 of the sequence, some of which may lie in the gap that no row sees; paged: all in one page.
struct PgTile { int first, last, page_index; int64_t page; };
// The span's v-th tile, of a part that ends before tile `end` (at least one lies before it).  Behind that comes the last token of the part's
// last tile: loads without a use, which cost no traffic and no branch.
template <bool PAGED>
__host__ __device__ __forceinline__ PgTile pg_tile_at(const PageAttnArgs &a, const PgSpan &s, int v, int end) {
    const int at = v < end ? v : end - 1, ti = at < s.sink_tiles ? at : at - s.sink_tiles + s.main_tile;
    PgTile x;
    x.page_index = 0; x.page = 0;
    auto least = [](int p, int q) { return p < q ? p : q; };
    if (PAGED) {
        const int L = (int)a.by_page.d;
        x.page_index = (int)quotient((uint32_t)ti, a.by_tiles);
        x.first = x.page_index * L + (ti - x.page_index * (int)a.by_tiles.d) * kPgTile;
        x.last = least(least(x.first + kPgTile, (x.page_index + 1) * L), s.kv);
    } else {
        x.first = ti * kPgTile;
        x.last = least(x.first + kPgTile, s.kv);
    }
    if (v >= end) x.first = x.last - 1;
    return x;
}
// A part's tiles: as many as the others' or one more.
__host__ __device__ __forceinline__ void pg_part(int total, int part, int parts, int &lo, int &hi) {
    const int each = (int)((uint32_t)total / (uint32_t)parts), more = total - each * parts;
    lo = part * each + (part < more ? part : more);
    hi = lo + each + (part < more ? 1 : 0);
}
// How the slots of a divided call (a.slots of them, the same for every head and row block) are dealt to the sequences: a slot for every q
// tiles or part of them, and one at least.  With n sequences and a.extra = slots - n the sum of ceil(T / q) is at most total / q + n, so that
// q = total / extra suffices.  Where there are few sequences it is the smallest that does, or nearly: it lies between total / slots and
// that, and is found in five halvings.  Where there are many it stays: the usual ones are taken whole, and those of more than q
// tiles, fewer than `extra`, have 2 extra parts at most, which are all that leave partial results.
__host__ __device__ __forceinline__ int pg_parts(int tiles, int q) {
    const int p = (int)(((uint32_t)tiles + (uint32_t)q - 1u) / (uint32_t)q);
    return p < 1 ? 1 : p;
}
constexpr int kPgLeast = 4;                       // tiles of a slot: one to a wavefront
constexpr int kPgHalvings = 5;
// The q that suffices, and one below which none does; total, and the reciprocals of extra and slots, to 2^-17 or better
struct PgShare { int lo, q; };
__host__ __device__ __forceinline__ PgShare pg_share(float total, float by_extra, float by_slots, int n, int extra) {
    auto most = [](int p, int q) { return p > q ? p : q; };
    // (rounded up, and down, by more than the sum is off; 2^26: more tiles than a sequence has)
    const float q = total * (1.0001f * by_extra);
    PgShare s;
    s.q = most((int)(q < 67108863.0f ? q : 67108863.0f) + 1, kPgLeast);
    s.lo = n <= extra ? most((int)(total * (0.9999f * by_slots)), kPgLeast) : s.q;
    return s;
}
// Token `off` of a tile, or one of the tile that some row sees instead of it: what is loaded is finite and in the pool.
__host__ __device__ __forceinline__ int pg_seen_token(const PgSpan &s, const PgTile &x, int off) {
    const int n = x.first + off < x.last ? x.first + off : x.last - 1;
    // (a tile that ends in the gap began below the sink's end)
    return n >= s.sink && n < s.lo ? (s.lo < x.last ? s.lo : s.sink - 1) : n;
}

// A part's partial result: [rows][D] sums, then the rows' references, then their sums of weights.
__host__ __device__ inline int64_t part_floats(int rows, int d) { return (int64_t)rows * (d + 2); }
// How a call is divided, a function of its sizes.
inline PagePlan page_plan(const qvg_page_cache &c, const qvg_page_step &t) {
    PagePlan p{16, 1, 0, 0, 0, 0, 0};
    // Tiles end where pages do, so that a tile's page is uniform, unless that would leave many of them short.
    p.paged = c.page_len % kPgTile == 0 || c.page_len >= 8 * kPgTile;
    // tiles that a sequence's rows see, at most
    int64_t tiles = p.paged ? (int64_t)c.table_pages * page_tiles((int)c.page_len) : page_tiles((int)(c.table_pages * c.page_len));
    if (t.window > 0) {
        const int64_t seen = (int64_t)t.window + t.n_new + t.sink, most = seen / kPgTile + 4 + (p.paged ? seen / c.page_len : 0);
        if (most < tiles) tiles = most;
    }
    const int64_t rows = (int64_t)t.group * t.n_new;
    p.rows = rows <= 16 ? 16 : 32;
    p.row_blocks = (int)((rows + p.rows - 1) / p.rows);
    const int64_t units = (int64_t)c.n_heads * p.row_blocks;             // of a sequence
    if (c.n_seqs < 1 || c.n_seqs > 256 || rows < 1) return p;
    // Two workgroups to a CU, which lengths that differ are dealt to best, or one where no two fit a CU, and for a sequence alone, whose
    // parts are all alike (4 heads x 64 rows over 32768 tokens 27 -> 23 us, 256 channels 176 -> 168; a ragged batch of 16: 182 -> 176 us
    // with two; three take up to 20 % longer, four up to 41 %); a tile to a wavefront at least.  With more sequences than that a call
    // is divided only for those that are much longer than the others (extra).
    // Not divided below 28 tiles, which cost less than the second launch (16 sequences of 500 tokens, 8 heads: 9.6 us, 13.4
    // divided; 8 of 700: 10.8 and 13.0; but one of 1000: 12.6 and 8.2).
    const int chip = c.n_seqs == 1 || c.head_dim > 192 || c.head_dim * p.rows > 16 * 256 ? 256 : 512;
    if (tiles < 28 || (c.n_seqs == 1 && units > 128)) return p;          // (1024 rows of 8 heads over 8192: 79 us, 94 divided)
    // (The cut at 128 units is coarse: divided, 144 and 160 units over 8192 tokens take 63 and 70 us instead of 78, over 65536 443 and 468
    // instead of 628 and 650; 240 units 89 instead of 78 to 80, and 606 and 670 instead of 609 and 639.)
    const int64_t full = (chip + units - 1) / units;
    int64_t slots = chip / units;
    if (slots >= 2 * (int64_t)c.n_seqs) {
        const int64_t most = c.n_seqs * (tiles / kPgLeast);
        if (slots > most) slots = most;
        p.extra = (int)(slots - c.n_seqs);
        p.kept = (int)slots;
    } else {
        if (tiles < 256 || units >= chip || c.n_seqs * c.n_heads * rows > (1 << 22)) return p;       // (128 of 2000 tokens: 178 us, 215 so)
        slots = c.n_seqs + full;
        p.extra = (int)full;
        p.kept = (int)(2 * full < slots ? 2 * full : slots);
    }
    p.slots = (int)slots;
    p.state_bytes = (size_t)(units * p.kept * part_floats(p.rows, c.head_dim)) * sizeof(float) + (size_t)c.n_seqs * sizeof(int2);
    return p;
}

}  // namespace qvg
