// Where the tokens of an attention over 16-bit pages lie: plain arithmetic, the same on the host (where tests walk through it) and on
// the device.
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
// Token `off` of a tile, or one of the tile that some row sees instead of it: what is loaded is finite and in the pool.
__host__ __device__ __forceinline__ int pg_seen_token(const PgSpan &s, const PgTile &x, int off) {
    const int n = x.first + off < x.last ? x.first + off : x.last - 1;
    // (a tile that ends in the gap began below the sink's end)
    return n >= s.sink && n < s.lo ? (s.lo < x.last ? s.lo : s.sink - 1) : n;
}

}  // namespace qvg
