// Attention of a step's tokens over a cache of 16-bit pages:
//     o = sum_n w_n v_n / sum_n w_n,   w_n = exp(scale q.k_n),
// in one pass over the tokens with the running maximum and sum of the soft-max.
//
// A workgroup takes a block of 16 or 32 query rows of one KV head (rows = group x new tokens) and a part of the sequence's tiles of
// 32 tokens; each of its wavefronts walks tiles of its own, so a tile costs no barrier.  Both contractions run on
// v_mfma_f32_16x16x32 with the operands where the loads put them, so keys and values pass through registers only:
//   S^T = K Q^T:   lane (c, kb) reads channels 32 i + 8 kb .. + 7 of tokens c and 16 + c;
//   O^T += V^T P:  lane (c, kb) reads an octet of channels (c, and 16 + c beyond 128) of tokens 4 kb + r and 16 + 4 kb + r, which
//                  are the tokens whose scores S^T leaves in the lane: P needs no movement, and pairs of tokens are packed
//                  channel by channel (v_perm_b32), which is the transposition.  MFMA j makes channels 8 c + j; the lane ends
//                  up with octets 4 kb + r of query row c.
// The weights enter as two numbers of the cache's type, w = hi + lo: the matrix cores have nothing else to do, and one number's
// rounding (2^-8 of a bf16 weight) would be as large as the output's own.
// A tile's keys are asked for when one before has been contracted, and so are its values: a wavefront has 16 KB (of 128 channels)
// on their way all the time; twice as much changes nothing (12 heads over 37440 tokens 41 us so and so).  Memory bounds it: 12 heads
// over 748800 tokens of 128 bf16, 4.6 GB, 675 us (6.8 TB/s; a large copy moves 4.9); a ragged batch of 16, 8 heads x 4, 1.08 GB,
// 175 us (6.1).  A call over few tokens is its launches, the walk to the first tile and 1 us a tile: 4.7 us for 100 tokens, 8 us for
// 1000 (one head, replayed in a graph).  Of many rows of a KV head each block of 32 reads its tokens again, and walks the tiles that any row
// of its sequence sees, not its own rows' alone: a causal prompt meets twice the pairs that are seen (1024 tokens, 8 heads x 4: 52 us, 167
// TFLOP/s of seen pairs), a chunk of 4680 with a window of 64 all of the chunk's; 12 heads x 4680 over 37440 tokens 2.3 ms (445 TFLOP/s).
#include "qvg_attn_pages.hpp"

#include <type_traits>

namespace qvg {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4_t;

constexpr int kPgThreads = 256, kPgWaves = kPgThreads / 64;
static_assert(kPgLeast == kPgWaves, "a slot has a tile for each wavefront");
constexpr float kPgNoScore = -3.402823466e38f;      // the running reference before any product
// References are products q.k, before the scale: a weight is exp2((product - reference) x scale + kPgUp), whose difference is exact where it
// matters, however large the products are.  A reference moves when a weight would pass 2^(kPgUp + kPgLag): they stay below 2^14,
// and the small ones of a row keep their bits in binary16 for longer.
constexpr float kPgUp = 7.0f, kPgLag = 7.0f;
// Binary16 ends at 2^-24, 2^-31 of a row's reference: many tokens that far below it are a part of the sum all the same (65536 tokens of
// 2^-33 and values 2^16 times as large as the heavy token's).  So a tile whose weights are all below 2^-kPgThin of the reference enters
// lifted by a power of two, with the row's sums lifted for as long (2^kPgMost of 2^60 at most): a weight is off by 2^-24 of the largest of
// its tile at most, as an fp32 sum would be.  (Nothing to be measured: 12 heads over 748800 tokens 679 us, 680 with most tiles lifted, 677 in
// bf16.)
constexpr float kPgThin = 8.0f, kPgMost = 40.0f;

struct PgBf16 {
    static constexpr bool kThin = false;
    static __device__ __forceinline__ floatx4_t mfma(const uint4 &a, const uint4 &b, const floatx4_t &c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) { return pack_bf16x2(x, y); }
    static __device__ __forceinline__ float lo(uint32_t w) { return bf16_lo(w); }
    static __device__ __forceinline__ float hi(uint32_t w) { return bf16_hi(w); }
};
struct PgF16 {
    static constexpr bool kThin = true;
    static __device__ __forceinline__ floatx4_t mfma(const uint4 &a, const uint4 &b, const floatx4_t &c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8_t, a), __builtin_bit_cast(halfx8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) { return pack_f16x2_rne(x, y); }
    static __device__ __forceinline__ float lo(uint32_t w) { return f16_bits_to_f32(w & 0xffffu); }
    static __device__ __forceinline__ float hi(uint32_t w) { return f16_bits_to_f32(w >> 16); }
};
// How a head of D channels lies in the operands: CH channels to a lane and set, NS sets of 16 lanes
template <int D> struct PgDim {
    static constexpr int CH = D > 64 ? 8 : 4, NS = (D + 16 * CH - 1) / (16 * CH), KK = D / 32, W = CH / 2;
    static constexpr int pitch = 16 * CH + 4;       // floats per row of a set where the wavefronts' results meet
};

__device__ __forceinline__ PgLens lens_of(const PageAttnArgs &a, int b) {
    return {a.c.table_pages ? a.c.kv_len[b] : 0, a.t.n_live ? a.t.n_live[b] : a.t.n_new};
}

// The slots of a divided call, dealt to the sequences as pg_share says.  Every wavefront works that out for itself from the lengths, which
// only the device knows (n <= 256: a call of more sequences is not divided).  Slots that are left over have nothing to do.
struct Slot { int b, part, parts, first; PgLens n; };                    // first: of the sequence's partial results; part >= parts: none
// Sums of lanes 0 .. i, and of all, between lanes of a row and then rows (no LDS, which five halvings of six exchanges would wait for)
template <typename N>
__device__ __forceinline__ N lanes_upto(N x) {
    auto from = [&](auto ctrl, auto rows) {
        return __builtin_bit_cast(N, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
    };
    typedef std::integral_constant<int, 0xf> all;
    x += from(std::integral_constant<int, 0x111>{}, all{});              // row_shr 1, 2, 4, 8
    x += from(std::integral_constant<int, 0x112>{}, all{});
    x += from(std::integral_constant<int, 0x114>{}, all{});
    x += from(std::integral_constant<int, 0x118>{}, all{});
    x += from(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});      // row_bcast 15, 31
    x += from(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return x;
}
template <typename N>
__device__ __forceinline__ N lanes_sum(N x) {
    return __builtin_bit_cast(N, __builtin_amdgcn_readlane(__builtin_bit_cast(int, lanes_upto(x)), 63));
}
// What a wavefront keeps of the sequences while it deals.  (Its loops are not unrolled: instructions that run once are waited for as they
// are fetched, and 2600 before the first tile cost every call 0.6 us more than these 1100.)
struct DealPlace { int2 lens[256]; int tiles[256]; };
template <bool PAGED>
__device__ __forceinline__ Slot deal(const PageAttnArgs &a, int slot, DealPlace &keep) {
    const int lane = threadIdx.x & 63, n = a.c.n_seqs;
    Slot p{0, 0, 0, 0, {0, 0}};
    if (n == 1) {
        p.n = lens_of(a, 0);
        const int total = pg_span_of<PAGED>(a, p.n).total, q = max(pg_parts(total, a.slots), kPgLeast);
        p.parts = pg_parts(total, q);
        p.part = slot;
        return p;
    }
    float total = 0.0f;
#pragma unroll 1
    for (int k = 0; k < n; k += 64) {
        const int i = k + lane;
        const PgLens l = lens_of(a, min(i, n - 1));
        const int t = i < n ? pg_span_of<PAGED>(a, l).total : 0;
        keep.lens[i] = make_int2(l.kv, l.live); keep.tiles[i] = t;
        total += (float)t;
    }
    total = lanes_sum(total);
    const PgShare share = pg_share(total, __builtin_amdgcn_rcpf((float)a.extra), __builtin_amdgcn_rcpf((float)a.slots), n, a.extra);
    int lo = share.lo, q = share.q;
#pragma unroll 1
    for (int h = 0; h < kPgHalvings && lo < q; ++h) {                    // uniform
        const int mid = lo + (q - lo) / 2;
        int need = 0;
#pragma unroll 1
        for (int k = 0; k < n; k += 64) need += k + lane < n ? pg_parts(keep.tiles[k + lane], mid) : 0;
        if (lanes_sum(need) <= a.slots) q = mid; else lo = mid + 1;
    }
    int before = 0, divided = 0;                                         // slots, and partial results, of the sequences before
#pragma unroll 1
    for (int k = 0; k < n; k += 64) {
        const int i = k + lane, mine = i < n ? pg_parts(keep.tiles[i], q) : 0, kept = mine > 1 ? mine : 0;
        const int upto = before + lanes_upto(mine), kept_upto = divided + lanes_upto(kept);
        const unsigned long long hit = __ballot(slot >= upto - mine && slot < upto);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            p.b = k + at; p.parts = __builtin_amdgcn_readlane(mine, at);
            p.part = slot - (__builtin_amdgcn_readlane(upto, at) - p.parts);
            p.first = __builtin_amdgcn_readlane(kept_upto - kept, at);
            asm volatile("" ::: "memory");                               // the wavefront's LDS operations stay in this order
            const int2 l = keep.lens[p.b];
            p.n = PgLens{__builtin_amdgcn_readfirstlane(l.x), __builtin_amdgcn_readfirstlane(l.y)};
            break;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
        divided = __builtin_amdgcn_readlane(kept_upto, 63);
    }
    return p;
}
// Where a query row lies: head h * group + r / n_new, row r % n_new of the sequence.
struct RowAt { int64_t head; int i; };
__device__ __forceinline__ RowAt row_at(const PageAttnArgs &a, int h, int64_t r) {
    RowAt p;
    const int u = (int)quotient((uint32_t)r, a.by_new);
    p.head = (int64_t)h * a.t.group + u; p.i = (int)r - u * a.t.n_new;
    return p;
}
// Store CH channels of a row from `ch` on: unnormalised sums o, the row's reference m and sum l of weights.  Where a score was no number l is
// none, and so is the lse (a row that sees nothing has -infinity); the row itself says so where none of its scores was a number (its query
// is none) or one was infinite, and is zero where some keys were none.
template <class T, int CH>
__device__ __forceinline__ void store_part(const PageAttnArgs &a, int b, int h, int64_t r, int live, int ch, const float *o, float m, float l) {
    const RowAt p = row_at(a, h, r);
    const bool seen = p.i < live && l > 0.0f, none = p.i < live && l != l;
    const float inv = seen ? 1.0f / l : 0.0f, lost = none && !(m > kPgNoScore && m < INFINITY) ? l : 0.0f;
    uint32_t w[CH / 2];
#pragma unroll
    for (int e = 0; e < CH / 2; ++e) w[e] = seen ? T::pack(o[2 * e] * inv, o[2 * e + 1] * inv) : T::pack(lost, lost);
    uint16_t *out = static_cast<uint16_t *>(a.t.out) + b * a.t.out_stride_seq + p.head * a.t.out_stride_head + p.i * a.t.out_stride_token + ch;
    if constexpr (CH == 8) *reinterpret_cast<uint4 *>(out) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2 *>(out) = make_uint2(w[0], w[1]);
    if (a.t.lse && ch == 0)
        a.t.lse[((int64_t)b * a.c.n_heads * a.t.group + p.head) * a.t.n_new + p.i] =
            seen ? (m * a.scale + (__builtin_log2f(l) - kPgUp)) * 0.6931471805599453f : (none ? l : -INFINITY);
}

// A lane's tokens of a tile are places in its page (paged), or rows anywhere in the pool, which lanes 0 .. 31 look up and leave in LDS.
// ONCE: no other workgroup reads the values again: they are loaded past the caches' usual order of eviction, which takes 4.6 GB at 6.75 TB/s
// instead of 6.06 (keys too: divided calls no faster than so, undivided ones slower, a ragged batch of 16 211 -> 246 us: a token's keys
// come by halves of a line).
template <class T, int D, int RB, bool PAGED, bool ONCE>
__global__ __launch_bounds__(kPgThreads, D > 192 || D * RB > 256 ? 1 : 2)
void attn_pages_kernel(PageAttnArgs a, int blocks, int per_xcd) {
    typedef PgDim<D> G;
    constexpr int kRows = 16 * RB, KK = G::KK, NS = G::NS, CH = G::CH, W = G::W;
    __shared__ __attribute__((aligned(16))) float meet[kPgWaves][16][G::pitch];
    __shared__ float ms[kPgWaves][kRows], ls[kPgWaves][kRows];
    __shared__ __attribute__((aligned(16))) int64_t rows_of[PAGED ? 1 : kPgWaves][kPgTile];
    // workgroups are dealt to the 8 XCDs round-robin: a head's row blocks, which read the same tokens, run on one
    const int w = (int)(blockIdx.x % 8u) * per_xcd + (int)(blockIdx.x / 8u);
    if (w >= blocks) return;                                             // uniform, before any barrier
    const int slot = (int)quotient((uint32_t)w, a.by_units), unit = w - slot * (int)a.by_units.d;
    const int h = (int)quotient((uint32_t)unit, a.by_blocks), rblk = unit - h * a.row_blocks;
    int b = slot, part = 0, parts = 1, first = 0;
    PgLens lens;
    if (a.slots) {
        __shared__ DealPlace keep[kPgWaves];
        const Slot s = deal<PAGED>(a, slot, keep[threadIdx.x >> 6]);
        if (s.part >= s.parts) return;                                   // uniform, before any barrier
        b = s.b; part = s.part; parts = s.parts; first = s.first; lens = s.n;
        if (unit == 0 && part == 0 && threadIdx.x == 0) a.places[b] = make_int2(first, parts);
    } else lens = lens_of(a, b);
    const PgSpan sq = pg_span_of<PAGED>(a, lens);
    int lo_tile, hi_tile;
    pg_part(sq.total, part, parts, lo_tile, hi_tile);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, kb = lane >> 4;
    const int64_t rows = (int64_t)a.t.group * a.t.n_new;
    const uint16_t *kp = static_cast<const uint16_t *>(a.c.k_pages) + h * a.c.stride_head;
    const uint16_t *vp = static_cast<const uint16_t *>(a.c.v_pages) + h * a.c.stride_head;
    const uint32_t row_bytes = (uint32_t)a.c.stride_token * 2u;

    // Q, and what each row sees: tokens below up[rb] that are at least low[rb], or below the sink.  Rows that are not there are
    // zeros, whose results nobody stores.
    uint4 q[RB][KK];
    int up[RB], low[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int64_t r = (int64_t)rblk * kRows + rb * 16 + c;
        up[rb] = low[rb] = 0;
        const uint16_t *qp = nullptr;
        if (r < rows) {
            const RowAt p = row_at(a, h, r);
            if (p.i < sq.live) {
                const int place = sq.kv - sq.live + p.i;
                up[rb] = a.t.causal ? place + 1 : sq.kv;
                low[rb] = a.t.window > 0 && place >= a.t.window ? place - a.t.window + 1 : 0;
                qp = static_cast<const uint16_t *>(a.t.q) + b * a.t.q_stride_seq + p.head * a.t.q_stride_head + p.i * a.t.q_stride_token;
            }
        }
#pragma unroll
        for (int i = 0; i < KK; ++i) q[rb][i] = qp ? *reinterpret_cast<const uint4 *>(qp + 32 * i + 8 * kb) : make_uint4(0u, 0u, 0u, 0u);
    }
    // tokens that every row of the sequence sees: all_low .. all_up - 1
    const int all_up = a.t.causal ? sq.kv - sq.live + 1 : sq.kv;
    const int all_low = a.t.window > 0 && sq.kv - 1 >= a.t.window ? sq.kv - a.t.window : 0;

    // ---- where a tile's tokens lie ------------------------------------------------------------
    auto in_pool = [&](int pg) -> int64_t { return pg < 0 ? 0 : (pg >= a.c.pool_pages ? a.c.pool_pages - 1 : pg); };
    const int32_t *table = a.c.page_table + (int64_t)b * a.c.table_pages;
    // (not paged) the rows of a tile's tokens: their pages are asked for a tile ahead
    struct Ahead { int n, in_page, page; };
    auto ask = [&](const PgTile &x) {
        Ahead p;
        p.n = pg_seen_token(sq, x, lane & 31);
        const int pi = (int)quotient((uint32_t)p.n, a.by_page);
        p.in_page = p.n - pi * (int)a.by_page.d;
        p.page = table[pi];
        return p;
    };
    auto park = [&](const Ahead &p) {
        if (lane < 32) rows_of[PAGED ? 0 : wave][lane] = in_pool(p.page) * a.c.stride_page + (int64_t)p.in_page * a.c.stride_token;
        asm volatile("" ::: "memory");                                   // the wavefront's LDS operations stay in this order
    };
    auto row_ptr = [&](const uint16_t *pool, const PgTile &x, int off) {
        if constexpr (PAGED) {
            const int n = pg_seen_token(sq, x, off) - x.page_index * (int)a.by_page.d;
            return reinterpret_cast<const uint16_t *>(reinterpret_cast<const char *>(pool + x.page * a.c.stride_page) + (uint64_t)((uint32_t)n) * row_bytes);
        } else return pool + rows_of[PAGED ? 0 : wave][off];
    };
    typedef uint32_t words __attribute__((ext_vector_type(W)));
    uint4 kr[2][KK];
    uint32_t vr[NS][8][W];
    auto load_k = [&](const PgTile &x) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint16_t *p = row_ptr(kp, x, 16 * hf + c) + 8 * kb;
#pragma unroll
            for (int i = 0; i < KK; ++i) kr[hf][i] = *reinterpret_cast<const uint4 *>(p + 32 * i);
        }
    };
    auto load_v = [&](const PgTile &x) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint16_t *p = row_ptr(vp, x, 16 * (e >> 2) + 4 * kb + (e & 3));
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int oct = min(16 * s + c, D / CH - 1);             // (octets beyond the head: results that nobody stores)
                const words *from = reinterpret_cast<const words *>(p + oct * CH);
                const words got = ONCE ? __builtin_nontemporal_load(from) : *from;
                __builtin_memcpy(vr[s][e], &got, sizeof(words));
            }
        }
    };

    floatx4_t O[RB][NS][CH];
    float m[RB], l[RB];
    const float lag = fminf(kPgLag / a.scale, 1e38f);                    // (any product is further than that above none)
    const float thin = fminf(kPgThin / a.scale, 1e38f);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kPgNoScore; l[rb] = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int j = 0; j < CH; ++j) O[rb][s][j] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // x is in registers, or on its way there; the one that follows it there is next, whose page is known or asked for.  (A wavefront asks for
    // tiles behind its last one too: behind a branch around the loads the waits for those before would be for all of them.)
    int v = lo_tile + wave;
    PgTile x, next;
    Ahead ahead;
    auto find = [&](int at) {
        PgTile y = pg_tile_at<PAGED>(a, sq, at, hi_tile);
        if constexpr (PAGED) y.page = in_pool(((const __attribute__((address_space(4))) int32_t *)table)[y.page_index]);
        else ahead = ask(y);
        return y;
    };
    if (v < hi_tile) {
        x = find(v);
        if (!PAGED) park(ahead);
        load_k(x);
        next = find(v + kPgWaves);
        load_v(x);
    }
    for (; v < hi_tile; v += kPgWaves) {
        // ---- S^T = K Q^T -------------------------------------------------------------------
        floatx4_t S[RB][2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                S[rb][hf] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < KK; ++i) S[rb][hf] = T::mfma(kr[hf][i], q[rb][i], S[rb][hf]);
            }
        __builtin_amdgcn_sched_barrier(0);                               // (loads before their registers' last use would need others)
        const PgTile now = x;
        x = next;
        if (!PAGED) park(ahead);
        next = find(v + 2 * kPgWaves);                                   // (behind these keys its page would be waited for with them)
        load_k(x);

        // ---- soft-max: the lane has tokens 16 hf + 4 kb + r of row c ------------------------
        const bool all = now.last - now.first == kPgTile && now.first >= all_low && now.last <= all_up;     // uniform
        uint4 ph[RB], pl[RB];
        float back[RB];                                                  // 2^-lift
        bool lifted = false;                                             // uniform
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = S[rb][e >> 2][e & 3];
            if (!all) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int n = now.first + 16 * (e >> 2) + 4 * kb + (e & 3);
                    p[e] = n < now.last && n < up[rb] && (n >= low[rb] || n < a.t.sink) ? p[e] : -INFINITY;
                }
            }
            float top = p[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, p[e]);
            if (__ballot(top - m[rb] > lag)) {                        // uniform: some row's reference moves
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float m_new = fmaxf(m[rb], top), alpha = __builtin_amdgcn_exp2f((m[rb] - m_new) * a.scale);
                l[rb] *= alpha; m[rb] = m_new;
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int j = 0; j < CH; ++j) O[rb][s][j] *= alpha;
            }
            if constexpr (T::kThin) {
                float up2 = kPgUp;
                back[rb] = 1.0f;
                const float under = m[rb] - top;                         // (infinite: nothing is seen)
                if (__ballot(under > thin && under < INFINITY)) {        // uniform: a lane's tokens, of some row, are that small
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    const float lift = __builtin_floorf(fminf(fmaxf((m[rb] - top) * a.scale, 0.0f), kPgMost)), ahead_by = __builtin_amdgcn_exp2f(lift);
                    up2 += lift; back[rb] = __builtin_amdgcn_exp2f(-lift);
                    lifted = true;
#pragma unroll
                    for (int s = 0; s < NS; ++s)
#pragma unroll
                        for (int j = 0; j < CH; ++j) O[rb][s][j] *= ahead_by;
                }
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) { p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[e] - m[rb], a.scale, up2)); sum += p[e]; }
                l[rb] = __builtin_fmaf(sum, back[rb], l[rb]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) { p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[e] - m[rb], a.scale, kPgUp)); l[rb] += p[e]; }
            }
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                hi[e] = T::pack(p[2 * e], p[2 * e + 1]);
                lo[e] = T::pack(__builtin_fmaf(T::lo(hi[e]), -1.0f, p[2 * e]), __builtin_fmaf(T::hi(hi[e]), -1.0f, p[2 * e + 1]));
            }
            ph[rb] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            pl[rb] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }

        // ---- O^T += V^T P ----------------------------------------------------------------------
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                uint32_t f[4];                                           // channel j: pairs of tokens
#pragma unroll
                for (int pr = 0; pr < 4; ++pr)
                    f[pr] = __builtin_amdgcn_perm(vr[s][2 * pr + 1][j / 2], vr[s][2 * pr][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
                const uint4 vf = make_uint4(f[0], f[1], f[2], f[3]);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    O[rb][s][j] = T::mfma(vf, ph[rb], O[rb][s][j]);
                    O[rb][s][j] = T::mfma(vf, pl[rb], O[rb][s][j]);
                }
            }
        if (T::kThin && lifted) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int j = 0; j < CH; ++j) O[rb][s][j] *= back[rb];
        }
        __builtin_amdgcn_sched_barrier(0);
        load_v(x);
    }

    // ---- the wavefronts' results meet ------------------------------------------------------
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        l[rb] += __shfl_xor(l[rb], 16, 64);
        l[rb] += __shfl_xor(l[rb], 32, 64);
        if (kb == 0) { ms[wave][rb * 16 + c] = m[rb]; ls[wave][rb * 16 + c] = l[rb]; }
    }
    __syncthreads();
    const int row = tid >> 4, oc = tid & 15;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float mm = ms[0][rb * 16 + c];
#pragma unroll
        for (int i = 1; i < kPgWaves; ++i) mm = fmaxf(mm, ms[i][rb * 16 + c]);
        const float f = __builtin_amdgcn_exp2f((m[rb] - mm) * a.scale);
        const int64_t r = (int64_t)rblk * kRows + rb * 16 + row;
        float mt = ms[0][rb * 16 + row], lt = 0.0f;
#pragma unroll
        for (int i = 1; i < kPgWaves; ++i) mt = fmaxf(mt, ms[i][rb * 16 + row]);
#pragma unroll
        for (int i = 0; i < kPgWaves; ++i) lt += ls[i][rb * 16 + row] * __builtin_amdgcn_exp2f((ms[i][rb * 16 + row] - mt) * a.scale);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if (rb + s > 0) __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < CH; j += 4)
                    *reinterpret_cast<float4 *>(&meet[wave][c][CH * (4 * kb + i) + j]) =
                        make_float4(O[rb][s][j][i] * f, O[rb][s][j + 1][i] * f, O[rb][s][j + 2][i] * f, O[rb][s][j + 3][i] * f);
            __syncthreads();
            float o[CH];
#pragma unroll
            for (int e = 0; e < CH; ++e) o[e] = 0.0f;
#pragma unroll
            for (int i = 0; i < kPgWaves; ++i)
#pragma unroll
                for (int e = 0; e < CH; ++e) o[e] += meet[i][row][CH * oc + e];
            const int ch = CH * (16 * s + oc);
            if (ch >= D) continue;
            if (parts > 1) {
                float *st = a.state + ((int64_t)unit * a.kept + first + part) * part_floats(kRows, D), *op = st + (rb * 16 + row) * D + ch;
#pragma unroll
                for (int e = 0; e < CH; e += 4) *reinterpret_cast<float4 *>(op + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                if (ch == 0) { st[kRows * D + rb * 16 + row] = mt; st[kRows * (D + 1) + rb * 16 + row] = lt; }
            } else if (r < rows) store_part<T, CH>(a, b, h, r, sq.live, ch, o, mt, lt);
        }
    }
}

// Joins query rows' parts: D / 4 lanes (four channels each) to a part, PER parts of a row at a time, as many rows to a workgroup as fit.
template <class T, int D, int PER>
__global__ __launch_bounds__(256)
void join_pages_kernel(PageAttnArgs a, int64_t n_rows) {
    constexpr int kLanes = D / 4, kRows = 256 / (kLanes * PER), kGroups = kRows * PER;
    __shared__ __attribute__((aligned(16))) float sums[kGroups][D];
    __shared__ float weights[kGroups], tops[kGroups];
    const int64_t rows = (int64_t)a.t.group * a.t.n_new;
    const int grp = (int)threadIdx.x / kLanes, c4 = (int)threadIdx.x - grp * kLanes, j = grp / PER;
    const int64_t at = (int64_t)blockIdx.x * kRows + j;
    const bool there = j < kRows && at < n_rows;
    const int64_t bh = (int64_t)((uint32_t)at / (uint32_t)rows), r = at - bh * rows;
    const int b = (int)(bh / a.c.n_heads), h = (int)(bh - (int64_t)b * a.c.n_heads);
    // a group's parts one after the other, their sums against the largest reference so far
    float m = kPgNoScore, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    int parts = 0;
    if (there) {
        const int2 place = a.places[b];                                  // first partial result, parts
        const int row = (int)(r % a.rows);
        const int64_t step = part_floats(a.rows, D);
        const float *st = a.state + (((int64_t)h * a.row_blocks + r / a.rows) * a.kept + place.x) * step;
        const float *mp = st + a.rows * D + row, *lp = mp + a.rows, *op = st + row * D + c4 * 4;
        parts = place.y > 1 ? place.y : 0;                               // (one: its workgroup has stored the row)
#pragma unroll 4
        for (int p = grp - j * PER; p < parts; p += PER) {
            const float mx = mp[p * step], lx = lp[p * step];
            const float4 x = *reinterpret_cast<const float4 *>(op + p * step);
            const float m_new = fmaxf(m, mx), f = __builtin_amdgcn_exp2f((mx - m_new) * a.scale), g = __builtin_amdgcn_exp2f((m - m_new) * a.scale);
            m = m_new;
            l = l * g + lx * f;
            o.x = o.x * g + x.x * f; o.y = o.y * g + x.y * f; o.z = o.z * g + x.z * f; o.w = o.w * g + x.w * f;
        }
    }
    if (there) {
        *reinterpret_cast<float4 *>(&sums[grp][c4 * 4]) = o;
        if (c4 == 0) { weights[grp] = l; tops[grp] = m; }
    }
    __syncthreads();
    if (!parts || grp != j * PER) return;
#pragma unroll
    for (int g = 0; g < PER; ++g) m = fmaxf(m, tops[grp + g]);
    l = 0.0f;
    o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int g = 0; g < PER; ++g) {
        const float4 x = *reinterpret_cast<const float4 *>(&sums[grp + g][c4 * 4]);
        const float f = __builtin_amdgcn_exp2f((tops[grp + g] - m) * a.scale);
        l += weights[grp + g] * f;
        o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f;
    }
    const float v[4] = {o.x, o.y, o.z, o.w};
    store_part<T, 4>(a, b, h, r, a.t.n_live ? max(0, min(a.t.n_live[b], a.t.n_new)) : a.t.n_new, c4 * 4, v, m, l);
}
template <class T, int D, int PER>
static void launch_join(const PageAttnArgs &a, int64_t n, hipStream_t s) {
    constexpr int kRows = 256 / (D / 4 * PER);
    join_pages_kernel<T, D, PER><<<dim3((unsigned)((n + kRows - 1) / kRows)), dim3(256), 0, s>>>(a, n);
}

bool page_attn_dim(int d) { return d == 64 || d == 96 || d == 128 || d == 192 || d == 256; }

template <class T, int D>
static void launch_dim(const PageAttnArgs &a, int blocks, hipStream_t s) {
    const int per_xcd = (blocks + 7) / 8;
    const dim3 grid((unsigned)(per_xcd * 8)), threads(kPgThreads);
    auto launch = [&](auto kernel) { kernel<<<grid, threads, 0, s>>>(a, blocks, per_xcd); };
    if (a.rows == 16) launch(a.paged ? attn_pages_kernel<T, D, 1, true, true> : attn_pages_kernel<T, D, 1, false, true>);
    else if (a.row_blocks == 1) launch(a.paged ? attn_pages_kernel<T, D, 2, true, true> : attn_pages_kernel<T, D, 2, false, true>);
    else launch(a.paged ? attn_pages_kernel<T, D, 2, true, false> : attn_pages_kernel<T, D, 2, false, false>);
    if (a.slots) {
        const int64_t n = (int64_t)a.c.n_seqs * a.c.n_heads * a.t.group * a.t.n_new;
        // (many rows have few parts)
        if (n > 512) launch_join<T, D, 2>(a, n, s);
        else launch_join<T, D, 1024 / D>(a, n, s);
    }
}
template <class T>
static void launch_type(const PageAttnArgs &a, int blocks, hipStream_t s) {
    switch (a.c.head_dim) {
        case 64: launch_dim<T, 64>(a, blocks, s); break;
        case 96: launch_dim<T, 96>(a, blocks, s); break;
        case 128: launch_dim<T, 128>(a, blocks, s); break;
        case 192: launch_dim<T, 192>(a, blocks, s); break;
        default: launch_dim<T, 256>(a, blocks, s); break;
    }
}
hipError_t launch_attn_pages(const PageAttnArgs &a, hipStream_t s) {
    const int blocks = (int)((int64_t)(a.slots ? a.slots : a.c.n_seqs) * a.c.n_heads * a.row_blocks);
    if (a.c.type == QVG_BF16) launch_type<PgBf16>(a, blocks, s);
    else launch_type<PgF16>(a, blocks, s);
    return hipGetLastError();
}

}  // namespace qvg
