// Where the tokens of an attention over 16-bit pages lie, walked through on the CPU (test_host_pages.py compiles this file for the host only).
// Prints one line per rule: its name, then "ok" or what is wrong.
#include <cstdio>
#include <vector>

#include "qvg_attn_pages.hpp"

using namespace qvg;

static PageAttnArgs args(int64_t table_pages, int64_t L, bool paged, int n_new, int window, int sink) {
    PageAttnArgs a{};
    a.c.table_pages = (int32_t)table_pages; a.c.page_len = L; a.t.n_new = n_new; a.t.window = window; a.t.sink = sink;
    a.paged = paged;
    a.by_page = fast_div((uint32_t)L); a.by_tiles = fast_div((uint32_t)page_tiles((int)L));
    return a;
}

static PgSpan span_of(const PageAttnArgs &a, PgLens n) { return a.paged ? pg_span_of<true>(a, n) : pg_span_of<false>(a, n); }
static PgTile tile_at(const PageAttnArgs &a, const PgSpan &s, int v, int end) { return a.paged ? pg_tile_at<true>(a, s, v, end) : pg_tile_at<false>(a, s, v, end); }

// Every token that some row sees lies in one tile of one part; every address that a wavefront forms, behind its last tile too, is one
// of such a token, in the tile's page.
static const char *walk(const PageAttnArgs &a, PgLens lens, int parts) {
    const PgSpan s = span_of(a, lens);
    const int L = (int)a.c.page_len;
    if (s.kv > a.c.table_pages * L || s.kv < 0 || (s.sink >= s.lo && s.lo)) return "span";
    auto seen = [&](int n) { return n >= 0 && n < s.kv && (n < s.sink || n >= s.lo); };
    std::vector<char> met(s.kv, 0);
    for (int part = 0; part < parts; ++part) {
        int lo, hi;
        pg_part(s.total, part, parts, lo, hi);
        if (lo >= hi) continue;
        for (int v = lo; v < hi + 24; ++v) {
            const PgTile x = tile_at(a, s, v, hi);
            for (int off = 0; off < kPgTile; ++off) {
                const int n = pg_seen_token(s, x, off);
                if (!seen(n)) return "token";
                if (a.paged && n / L != x.page_index) return "page";
                if (v < hi && x.first + off < x.last && seen(x.first + off)) {
                    if (n != x.first + off) return "place";
                    if (met[n]++) return "twice";
                }
            }
            if (x.last - x.first > kPgTile || x.last <= x.first) return "size";
        }
    }
    for (int n = 0; n < s.kv; ++n)
        if (met[n] != (seen(n) ? 1 : 0)) return "left out";
    return "ok";
}

static const char *small(bool paged) {
    const int Ls[] = {1, 3, 16, 31, 32, 33, 50, 64, 100, 256, 300}, windows[] = {0, 1, 2, 5, 31, 32, 33, 64, 90, 400, 0x7fffffff},
              sinks[] = {0, 1, 7, 31, 32, 33, 40, 100, 500, 0x7fffffff};
    for (int L : Ls)
        for (int w : windows)
            for (int sink : sinks)
                for (int n_new : {1, 4, 70})
                    for (int kv : {0, 1, 2, 5, 31, 32, 33, 34, 63, 64, 65, 100, 129, 255, 256, 300, 301, 350, 600, -3})
                        for (int live : {0, 1, 3, n_new, n_new + 5, -1}) {
                            const PageAttnArgs a = args((420 + L - 1) / L, L, paged, n_new, w, sink);
                            for (int parts : {1, 2, 7}) {
                                const char *r = walk(a, PgLens{kv, live}, parts);
                                if (r[0] != 'o') {
                                    static char text[200];
                                    snprintf(text, sizeof text, "%s: L %d window %d sink %d n_new %d kv %d live %d parts %d", r, L, w, sink, n_new, kv, live, parts);
                                    return text;
                                }
                            }
                        }
    return "ok";
}

// the ends of the largest sequences
static const char *large(bool paged) {
    for (int64_t L : {1ll, 16ll, 32ll, 48ll, 256ll, 4680ll, 1ll << 20, 1ll << 30})
        for (int w : {0, 1, 100, 1 << 29, 0x7fffffff})
            for (int sink : {0, 33, 1 << 28, 0x7fffffff})
                for (int n_new : {1, 1000}) {
                    const int64_t pages = (1ll << 30) / L;
                    const PageAttnArgs a = args(pages, L, paged, n_new, w, sink);
                    const PgSpan s = span_of(a, PgLens{0x7fffffff, 0x7fffffff});
                    if (s.kv != pages * L || s.live != n_new || s.total < 1) return "span";
                    for (int parts : {1, 7, 512})
                        for (int part : {0, parts / 2, parts - 1}) {
                            int lo, hi;
                            pg_part(s.total, part, parts, lo, hi);
                            if (part == parts - 1 && hi != s.total) return "end";
                            for (int v : {lo, lo + 1, lo + 3, (lo + hi) / 2, hi - 2, hi - 1, hi, hi + 15}) {
                                if (v < lo || lo >= hi) continue;
                                const PgTile x = tile_at(a, s, v, hi);
                                if (x.first < 0 || x.last <= x.first || x.last > s.kv || x.last - x.first > kPgTile) return "tile";
                                for (int off = 0; off < kPgTile; ++off) {
                                    const int n = pg_seen_token(s, x, off);
                                    if (n < 0 || n >= s.kv || (n >= s.sink && n < s.lo)) return "token";
                                    if (a.paged && n / L != x.page_index) return "page";
                                }
                            }
                        }
                }
    return "ok";
}

static const char *quotients() {
    for (uint64_t d = 1; d < (1ull << 31); d = d + 1 + d / 50) {
        for (uint64_t e : {d, d - 1, d + 1}) {
            if (e < 1 || e >= (1ull << 31)) continue;
            const FastDiv f = fast_div((uint32_t)e);
            for (uint64_t k = 0; k < 40; ++k) {
                const uint64_t m = k < 20 ? k * e : (0x7fffffffull / e - (k - 20)) * e;
                for (uint64_t n : {m, m + 1, m - 1, m + e - 1})
                    if (n < (1ull << 31) && quotient((uint32_t)n, f) != n / e) return "quotient";
            }
            if (quotient(0x7fffffffu, f) != 0x7fffffffu / e) return "largest";
        }
    }
    return "ok";
}

int main() {
    printf("quotients %s\n", quotients());
    printf("small_paged %s\n", small(true));
    printf("small_rows %s\n", small(false));
    printf("large_paged %s\n", large(true));
    printf("large_rows %s\n", large(false));
    return 0;
}
