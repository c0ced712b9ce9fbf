// How the sequences of a divided attention over 16-bit pages are dealt to workgroups, and where their partial results lie, on the CPU
// (test_host_page_division.py compiles this file for the host only).  Prints one line per rule: its name, then "ok" or what is wrong.
#include <cmath>
#include <cstdio>
#include <random>
#include <vector>

#include "qvg_attn_pages.hpp"

using namespace qvg;

static std::mt19937 rng(1);
static int any(int lo, int hi) { return lo + (int)(rng() % (uint32_t)(hi - lo + 1)); }

static PageAttnArgs args_of(const qvg_page_cache &c, const qvg_page_step &t, const PagePlan &p) {
    PageAttnArgs a{};
    a.c = c; a.t = t; a.paged = p.paged; a.rows = p.rows; a.row_blocks = p.row_blocks; a.slots = p.slots; a.extra = p.extra; a.kept = p.kept;
    a.by_page = fast_div((uint32_t)c.page_len); a.by_tiles = fast_div((uint32_t)page_tiles((int)c.page_len));
    return a;
}
struct Seen { int divided = 0, halved = 0, whole = 0, most_kept = 0; };

// The steps that a wavefront takes, its 64 lanes' sums as one; `off`: how far its reciprocals, and its sum of tiles, are off.
static const char *deal_all(const PageAttnArgs &a, const PagePlan &plan, const std::vector<PgLens> &lens, float off, Seen &seen) {
    const int n = a.c.n_seqs;
    std::vector<int> tiles(n);
    double sum = 0;
    for (int b = 0; b < n; ++b) sum += tiles[b] = (a.paged ? pg_span_of<true>(a, lens[b]) : pg_span_of<false>(a, lens[b])).total;
    int q;
    if (n == 1) {
        q = pg_parts(tiles[0], a.slots);
        if (q < kPgLeast) q = kPgLeast;
    } else {
        const PgShare s = pg_share((float)sum * (1.0f + off), 1.0f / a.extra * (1.0f + off), 1.0f / a.slots * (1.0f + off), n, a.extra);
        int lo = s.lo;
        q = s.q;
        if (lo > q) return "a share below its least";
        auto need = [&](int share) {
            int64_t m = 0;
            for (int b = 0; b < n; ++b) m += pg_parts(tiles[b], share);
            return m;
        };
        if (need(q) > a.slots) return "the share does not suffice";
        for (int h = 0; h < kPgHalvings && lo < q; ++h) {
            const int mid = lo + (q - lo) / 2;
            if (need(mid) <= a.slots) q = mid; else lo = mid + 1;
            ++seen.halved;
        }
    }
    int64_t slots = 0, kept = 0;
    for (int b = 0; b < n; ++b) {
        const int parts = pg_parts(tiles[b], q);
        int at = 0;
        for (int part = 0; part < parts; ++part) {
            int lo, hi;
            pg_part(tiles[b], part, parts, lo, hi);
            if (lo != at || hi < lo || (parts > 1 && hi - lo > q)) return "a part's tiles";
            at = hi;
        }
        if (at != tiles[b]) return "tiles left out";
        slots += parts;
        kept += parts > 1 ? parts : 0;
    }
    if (slots > a.slots) return "more parts than slots";
    if (kept > a.kept) return "more partial results than there is room for";
    if (kept > seen.most_kept) seen.most_kept = (int)kept;
    kept ? ++seen.divided : ++seen.whole;
    // the largest index of a partial result, and the places behind them
    const int64_t units = (int64_t)a.c.n_heads * a.row_blocks, floats = units * a.kept * part_floats(a.rows, a.c.head_dim);
    if (plan.state_bytes != (size_t)floats * sizeof(float) + (size_t)n * sizeof(int2)) return "bytes of scratch";
    if (floats % 4) return "alignment of the places";
    if (units * a.slots > (1 << 23)) return "workgroups";
    return "ok";
}

static std::vector<PgLens> lengths(int n, int most, int n_new, int kind) {
    std::vector<PgLens> v(n);
    for (int b = 0; b < n; ++b) {
        int kv = 0;
        if (kind == 0) kv = most;
        else if (kind == 1) kv = any(0, most);
        else if (kind == 2) kv = b == n / 2 ? most : any(0, 40);
        else if (kind == 3) kv = b % 64 == 63 ? most : any(0, most / 50 + 1);
        else if (kind == 4) kv = 0;
        else if (kind == 5) kv = (int)std::exp(std::log(most + 1.0) * any(0, 1000) / 1000.0);
        else kv = any(-5, 1) < 0 ? any(most / 2, most) : most;
        v[b] = PgLens{kv, any(0, 9) ? n_new : any(-1, n_new + 1)};
    }
    return v;
}

// few: two workgroups and more to a sequence; many: one to each, and extra ones
static const char *walk(bool few) {
    Seen seen;
    int plans = 0;
    const int heads[] = {1, 2, 3, 5, 8, 12, 40, 100, 255, 256, 511}, dims[] = {64, 96, 128, 192, 256}, Ls[] = {1, 16, 31, 32, 48, 64, 100, 256, 257, 4680, 1 << 20};
    for (int trial = 0; trial < 60000; ++trial) {
        qvg_page_cache c{};
        qvg_page_step t{};
        c.n_seqs = few ? any(1, 130) : any(1, 256); c.n_heads = heads[any(0, 10)]; c.head_dim = dims[any(0, 4)];
        c.page_len = Ls[any(0, 10)]; c.pool_pages = 1;
        const int64_t tokens = (int64_t)std::exp(std::log(1e9) * any(300, 1000) / 1000.0);
        c.table_pages = (int32_t)(tokens / c.page_len);
        t.group = any(0, 1) ? 1 : any(1, 20); t.n_new = any(0, 2) ? 1 : any(1, 40); t.causal = any(0, 1);
        t.window = any(0, 2) ? 0 : any(1, 40000); t.sink = t.window ? any(0, 100) : 0;
        const PagePlan p = page_plan(c, t);
        if (!p.slots) {
            if (p.state_bytes) return "bytes of a call that is not divided";
            continue;
        }
        const bool whole_batch = p.slots == c.n_seqs + p.extra && p.extra == (512 + c.n_heads * p.row_blocks - 1) / (c.n_heads * p.row_blocks);
        const bool half_batch = p.slots == c.n_seqs + p.extra && p.extra == (256 + c.n_heads * p.row_blocks - 1) / (c.n_heads * p.row_blocks);
        const bool extra_ones = whole_batch || half_batch;               // (a slot to a sequence and `extra`, wherever a sequence gets no two)
        if (!extra_ones && p.slots < 2 * c.n_seqs) return "the extra slots";
        if (few == extra_ones) continue;
        if (p.slots != c.n_seqs + p.extra || p.kept > p.slots) return "slots";
        ++plans;
        const PageAttnArgs a = args_of(c, t, p);
        const int most = (int)(c.table_pages * c.page_len);
        for (int kind = 0; kind < 7; ++kind) {
            const std::vector<PgLens> lens = lengths(c.n_seqs, most, t.n_new, kind);
            for (float off : {0.0f, 7e-6f, -7e-6f}) {
                const char *r = deal_all(a, p, lens, off, seen);
                if (r[0] != 'o') {
                    static char text[240];
                    snprintf(text, sizeof text, "%s: seqs %d heads %d dim %d page_len %lld pages %d group %d new %d window %d sink %d kind %d off %g", r, c.n_seqs, c.n_heads,
                             c.head_dim, (long long)c.page_len, c.table_pages, t.group, t.n_new, t.window, t.sink, kind, off);
                    return text;
                }
            }
        }
    }
    if (plans < 500 || seen.divided < 1000 || seen.whole < 100 || seen.halved < 1000) return "too few of a kind";
    return "ok";
}

int main() {
    printf("few %s\n", walk(true));
    printf("many %s\n", walk(false));
    return 0;
}
