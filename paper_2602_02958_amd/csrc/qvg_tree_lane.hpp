// What the kernels that attend over a paged cache share: a sequence's tiles, the decoding of a tile into the operands of the two
// contractions, and the way of a row's result to memory.
#pragma once
#include "qvg_tree.hpp"

namespace qvg {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4_t;

constexpr int kTrThreads = 256, kTrWaves = kTrThreads / 64;
constexpr float kTrNoScore = -3.402823466e38f;      // the running reference before any score (finite: see kNoScore)
// Probabilities are taken against a reference kTrBelow under the row's maximum and the reference moves when a score is
// kTrBelow + kTrLag above it: they stay below 2^14, and the small ones keep their bits in binary16 for longer.
constexpr float kTrBelow = 7.0f, kTrLag = 7.0f;
constexpr int kTrPitch = 132;                       // floats per row where the wavefronts' results meet

// One sequence's tiles: compressed ones page by page, then the tail's, then the new tokens'.
struct SeqTiles {
    int kv, tail, nodes;
    int per_page, kv_tiles, tail_tiles, total;
};
__device__ __forceinline__ SeqTiles tiles_of_sequence(const qvg_tree_step &t, int b) {
    SeqTiles s;
    const int kvmax = (int)(t.table_pages * t.page_len);
    auto clamp = [](int v, int hi) { return v < 0 ? 0 : (v > hi ? hi : v); };
    s.kv = t.table_pages ? clamp(t.kv_len[b], kvmax) : 0;
    s.tail = t.tail_capacity ? clamp(t.tail_len[b], t.tail_capacity) : 0;
    s.nodes = t.nodes ? clamp(t.nodes[b], t.n_nodes) : t.n_nodes;
    if (s.nodes == 0) s.kv = s.tail = 0;                                 // no row: nothing to read
    // (table_pages * page_len < 2^31, so a page that holds a token is shorter)
    const int L = s.kv ? (int)t.page_len : 1;
    s.per_page = tree_tiles(L);
    const int full = s.kv / L;
    s.kv_tiles = full * s.per_page + tree_tiles(s.kv - full * L);
    s.tail_tiles = tree_tiles(s.tail);
    s.total = s.kv_tiles + s.tail_tiles + tree_tiles(s.nodes);
    return s;
}

// the eight pairs' rotation, values not rounded before it
__device__ __forceinline__ void rotate_octet(float *acc, const uint4 &rp) {
    const uint32_t w[4] = {rp.x, rp.y, rp.z, rp.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const halfx2_t cs = __builtin_bit_cast(halfx2_t, w[i]);
        const float c = (float)cs[0], sn = (float)cs[1], x0 = acc[2 * i], x1 = acc[2 * i + 1];
        acc[2 * i] = __builtin_fmaf(x0, c, -(x1 * sn));
        acc[2 * i + 1] = __builtin_fmaf(x0, sn, x1 * c);
    }
}

__device__ __forceinline__ halfx8_t pack_f16x8(const float *v) {
    return __builtin_bit_cast(halfx8_t, make_uint4(pack_f16x2_rne(v[0], v[1]), pack_f16x2_rne(v[2], v[3]),
                                                   pack_f16x2_rne(v[4], v[5]), pack_f16x2_rne(v[6], v[7])));
}

// A block's partial result: [rows][128] sums, then the rows' references, then their sums of weights.
__host__ __device__ inline int64_t tree_state_floats(int rows) { return (int64_t)rows * (kHeadDim + 2); }

// How the slots of a divided call (a.slots of them, the same for every head and row block) are dealt to the sequences: a slot
// for every q tiles or part of them, and one at least, with the smallest q for which the slots suffice, or nearly: it lies between
// total / slots and total / (slots - n), since the sum of ceil(T / q) over n sequences is at most total / q + n, and is found in
// five halvings (16 ragged sequences on 64 slots, whose parts the upper end makes a third longer: 116 -> 109 us).  Every wavefront
// works that out for itself from the lengths, which only the device knows (n <= 256: a call of more sequences is not divided).
// Slots that are left over have nothing to do.
struct SlotPlace { int b, part, parts, first; };                         // first: the sequence's first slot; parts: 0, none
__device__ __forceinline__ int parts_of_tiles(int total, int q) {
    const int p = (int)(((uint32_t)total + (uint32_t)q - 1u) / (uint32_t)q);
    return p < 1 ? 1 : p;
}
template <typename N>
__device__ __forceinline__ N sum_of_lanes(N x) {
#pragma unroll
    for (int off = 1; off < 64; off *= 2) x += __shfl_xor(x, off, 64);
    return x;
}
// The place of slot `slot`.  Uniform over a wavefront.
__device__ __forceinline__ SlotPlace place_slot(const TreeArgs &a, int slot) {
    const int lane = threadIdx.x & 63, n = a.t.n_seqs;
    int tiles[4];                                                        // of sequences lane, 64 + lane, ..
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        tiles[k] = 0;
        if (64 * k < n && 64 * k + lane < n) tiles[k] = tiles_of_sequence(a.t, 64 * k + lane).total;
    }
    int q;
    if (n == 1) q = (__builtin_amdgcn_readfirstlane(tiles[0]) + a.slots - 1) / a.slots;
    else {
        const int64_t total = sum_of_lanes((int64_t)tiles[0] + tiles[1] + tiles[2] + tiles[3]);
        int lo = (int)((total + a.slots - 1) / a.slots);
        q = (int)((total + a.slots - n - 1) / (a.slots - n));
        for (int i = 0; i < 5 && lo < q; ++i) {                          // uniform
            const int mid = lo + (q - lo) / 2;
            int need = 0;
            if (mid > 0)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (64 * k < n) need += 64 * k + lane < n ? parts_of_tiles(tiles[k], mid) : 0;
            if (mid > 0 && sum_of_lanes(need) <= a.slots) q = mid; else lo = mid + 1;
        }
    }
    if (q < 2 * kTrWaves) q = 2 * kTrWaves;                              // two tiles to a wavefront
    SlotPlace p{0, 0, 0, 0};
    int before = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int base = 64 * k, i = base + lane;
        if (base >= n) break;                                            // uniform
        const int mine = i < n ? parts_of_tiles(tiles[k], q) : 0;
        int upto = mine;
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {
            const int x = __shfl_up(upto, off, 64);
            if (lane >= off) upto += x;
        }
        upto += before;
        const unsigned long long hit = __ballot(mine > 0 && slot >= upto - mine && slot < upto);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            p.b = base + at; p.parts = __shfl(mine, at, 64); p.first = __shfl(upto, at, 64) - p.parts;
            p.part = slot - p.first;
            break;
        }
        before = __shfl(upto, 63, 64);
    }
    p.b = __builtin_amdgcn_readfirstlane(p.b); p.part = __builtin_amdgcn_readfirstlane(p.part);
    p.parts = __builtin_amdgcn_readfirstlane(p.parts); p.first = __builtin_amdgcn_readfirstlane(p.first);
    if (a.share > 1 && p.parts >= 2 * a.share) p.parts = p.parts / a.share * a.share;       // whole groups
    return p;
}

// A workgroup's sequence, head, row block and part, from its number on its XCD (consecutive numbers run on one): the parts of one
// head together, whose pages' tables the L2 keeps, or with a rotation the same parts of all heads, which read the same rows of
// its table at about the same time.  parts: 0 where there is nothing to do.
struct BlockPlace { int b, h, rblk, part, parts; int64_t state; };       // state: floats of the part's place in a.state
__device__ __forceinline__ BlockPlace place_block(const TreeArgs &a, int w, bool rotated, int block_rows) {
    const int units = a.H * a.row_blocks;                                // of a sequence
    BlockPlace p;
    if (a.slots == 0) {
        p.b = w / units; p.part = 0; p.parts = 1; p.state = 0;
        const int unit = w - p.b * units;
        p.rblk = unit % a.row_blocks; p.h = unit / a.row_blocks;
        return p;
    }
    const int unit = rotated ? w % units : w / a.slots, slot = rotated ? w / units : w % a.slots;
    const SlotPlace s = place_slot(a, slot);
    p.b = s.b; p.part = s.part; p.parts = s.part < s.parts ? s.parts : 0;
    p.rblk = unit % a.row_blocks; p.h = unit / a.row_blocks;
    if (unit == 0 && p.part == 0 && p.parts > 0 && threadIdx.x == 0) a.places[p.b] = make_int2(s.first, s.parts);
    p.state = ((int64_t)unit * a.slots + slot) * tree_state_floats(block_rows);
    return p;
}

// The tiles of a part: range [lo, hi), of which the part's wavefronts take first, first + step, .. (a round of kTrWaves each).
// Parts that share a range walk it together: the tables of its pages, which they gather rows from, then stay in their XCD's L2.
struct PartTiles { int lo, hi, first, step; };
__device__ __forceinline__ PartTiles tiles_of_part(const TreeArgs &a, const SeqTiles &sq, int part, int parts) {
    const int share = a.slots && parts >= 2 * a.share ? a.share : 1, groups = parts / share, g = part / share;
    PartTiles p;
    p.lo = (int)((int64_t)sq.total * g / groups); p.hi = (int)((int64_t)sq.total * (g + 1) / groups);
    p.first = p.lo + (part - g * share) * kTrWaves; p.step = share * kTrWaves;
    return p;
}

// Where a query row of the batch lies: head h * group + r / n_nodes, node r % n_nodes.
struct RowPlace { int64_t head; int node; };
__device__ __forceinline__ RowPlace place_row(const TreeArgs &a, int h, int64_t r) {
    RowPlace p;
    const int u = (int)((uint32_t)r / (uint32_t)a.t.n_nodes);
    p.head = (int64_t)h * a.t.group + u; p.node = (int)r - u * a.t.n_nodes;
    return p;
}

// Store eight channels of a row: unnormalised sums o, the row's reference m and sum l of weights.
__device__ __forceinline__ void store_row8(const TreeArgs &a, int b, int h, int64_t r, int nodes, int c8, const float *o, float m,
                                           float l) {
    const RowPlace p = place_row(a, h, r);
    const bool seen = p.node < nodes && l > 0.0f;
    const float inv = seen ? 1.0f / l : 0.0f;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = seen ? o[e] * inv : 0.0f;
    bf16_t *out = static_cast<bf16_t *>(a.t.out) + b * a.t.out_stride_seq + p.head * a.t.out_stride_head + p.node * a.t.out_stride_node;
    *reinterpret_cast<uint4 *>(out + c8 * 8) = pack_bf16x8(v);
    if (a.t.lse && c8 == 0)
        a.t.lse[((int64_t)b * a.H * a.t.group + p.head) * a.t.n_nodes + p.node] =
            seen ? (m + __builtin_log2f(l)) * 0.6931471805599453f : -INFINITY;
}


constexpr int kTrRowPitch = 36;                     // 16-bit words per row of 32 tokens (72 bytes: 8-byte aligned, spread over the banks)

__device__ __forceinline__ halfx2_t as_half2(uint32_t w) { return __builtin_bit_cast(halfx2_t, w); }
__device__ __forceinline__ uint32_t as_bits(halfx2_t h) { return __builtin_bit_cast(uint32_t, h); }
// packed a * b + c, one rounding per element
__device__ __forceinline__ halfx2_t fma_half2(halfx2_t a, halfx2_t b, halfx2_t c) { return __builtin_elementwise_fma(a, b, c); }

// Two-bit levels of w's halves, field j from the top: (q, q') as (2q, 2q')
__device__ __forceinline__ halfx2_t level2(uint32_t w, int j) { return as_half2((w << (2 * j)) & 0xC000C000u); }
// Four-bit levels: x holds q + 8 in its nibbles; nibble k of both halves as (q, q').  With the exponent of 1024 in front a
// nibble is 1024 + u, or 1024 + 16 u from the second place of a byte.
__device__ __forceinline__ halfx2_t level4(uint32_t x, int k) {
    const uint32_t w = k < 2 ? x : x >> 8;
    const halfx2_t big = {(_Float16)1032.0f, (_Float16)1032.0f}, sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f},
                   off = {(_Float16)-72.0f, (_Float16)-72.0f};
    if (k & 1) return fma_half2(as_half2((w & 0x00F000F0u) | 0x64006400u), sixteenth, off);
    return as_half2((w & 0x000F000Fu) | 0x64006400u) - big;
}

// A stored format at compile time: with sizes that are known every load of the loop has one form, and nothing waits for it
// before it is used (with run-time branches between forms the loop waited for loads where the forms meet: one token over 12 heads
// x 187200 tokens of four rounds 239 us instead of 219).
template <int T_, int G_, bool FP8_, bool I4_, int S_>
struct TreeFormat {
    static constexpr int T = T_, G = G_, S = S_, TG = T * G;             // rounds, groups per token, smoothing stages
    static constexpr bool FP8 = FP8_, I4 = I4_;
    static constexpr int code = I4 ? 64 : 32;                            // code bytes per token and round
    static constexpr int record = TG * (FP8 ? 1 : 2);                    // scale bytes per token
    // bytes of a wavefront's LDS: V codes [T][16 octets][32 tokens], scales [2][T * G][32], row offsets [2][S][32]
    static constexpr int wave_bytes = T * 16 * kTrRowPitch * (I4 ? 4 : 2) + 2 * TG * kTrRowPitch * 2 + 2 * S * kTrTile * 4;
};


// Calls f(TreeFormat<..>{}) for the packed format of these parameters.
template <class Call>
inline hipError_t tree_format(int T, int G, int fmt, int S, Call f) {
#define QVG_TREE_CALL(t, g, fp8, i4, s) \
    if (T == t && G == g && S == s && fmt == ((fp8 ? kFmtE4M3 : 0) | (i4 ? kFmtInt4 : 0))) return f(TreeFormat<t, g, fp8, i4, s>{});
    QVG_TREE_FORMATS(QVG_TREE_CALL)
#undef QVG_TREE_CALL
    return hipErrorInvalidValue;
}

// A lane's part in decoding tiles of one sequence and KV head.  `own`: F::wave_bytes of LDS that are the wavefront's alone.
template <class F>
struct TreeLane {
    static constexpr int T = F::T, G = F::G, TG = F::TG, S = F::S, kCode = F::code, kRec = F::record;
    static constexpr bool I4 = F::I4, FP8 = F::FP8;
    static constexpr int kVPieces = T * kCode / 32, kTokPieces = T * kCode / 16;   // 16-byte pieces of the V codes: to a lane, of a token
    struct Where { int page_index, first, count; int64_t page, tok; };   // of a tile; tok: its first token in the pool
    // What a lane fetches of a tile: of tokens c and 16 + c the K codes of its 32 channels; 16-byte pieces of the V codes; the
    // scale record and the ids of one token (lanes 0..31: K, 32..63: V).
    struct Raw { uint4 kc4[2][I4 ? T : 1]; uint2 kc[2][I4 ? 1 : T]; uint4 vc[kVPieces]; uint32_t sc[(kRec + 3) / 4], id[S]; };

    const TreeArgs &a;
    const SeqTiles &sq;
    const int b, lane, c, kb, L, idb;
    const bool vside;
    PoolSide ks, vs;
    const uint8_t *side_scales, *side_ids;
    uint16_t *vcodes, *scales;
    uint32_t *offs;

    __device__ __forceinline__ TreeLane(const TreeArgs &args, const SeqTiles &tiles, int b_, int h, unsigned char *own)
        : a(args), sq(tiles), b(b_), lane(threadIdx.x & 63), c(threadIdx.x & 15), kb((threadIdx.x & 63) >> 4),
          L(tiles.kv ? (int)args.t.page_len : 1), idb(args.id_wide ? 2 : 1), vside((threadIdx.x & 63) >= 32), ks(args.k), vs(args.v) {
        const int64_t tok = (int64_t)h * a.t.pool_pages * a.t.page_len, tables = (int64_t)h * a.t.pool_pages * S * a.K * kHeadDim;
        ks.cent += tables;              vs.cent += tables;
        ks.ids += tok * S * idb;        vs.ids += tok * S * idb;
        ks.codes += tok * T * kCode;    vs.codes += tok * T * kCode;
        ks.scales += tok * kRec;        vs.scales += tok * kRec;
        side_scales = vside ? vs.scales : ks.scales;
        side_ids = vside ? vs.ids : ks.ids;
        vcodes = reinterpret_cast<uint16_t *>(own);
        scales = vcodes + T * 16 * kTrRowPitch * (I4 ? 2 : 1);
        offs = reinterpret_cast<uint32_t *>(scales + 2 * TG * kTrRowPitch);
    }
    // the wavefront's LDS operations stay in this order
    static __device__ __forceinline__ void order_lds() { asm volatile("" ::: "memory"); }
    static __device__ __forceinline__ uint4 load16(const void *base, uint32_t off) {
        return *reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(base) + off);
    }
    // Tile in_page of the sequence's page pi; `last`: the tile before (one of the same page needs no table).
    __device__ __forceinline__ Where place(int pi, int in_page, const Where &last) const {
        Where x;
        x.page_index = pi; x.first = in_page * kTrTile;
        x.count = min(kTrTile, min(L, sq.kv - pi * L) - x.first);
        x.page = last.page;
        if (pi != last.page_index) {
            const int64_t pg = __builtin_amdgcn_readfirstlane(a.t.page_table[(int64_t)b * a.t.table_pages + pi]);
            x.page = pg < 0 ? 0 : (pg >= a.t.pool_pages ? a.t.pool_pages - 1 : pg);
        }
        x.tok = x.page * L + x.first;
        return x;
    }
    // What belongs to tokens that are not there is read from the tile's last token instead, whatever piece of it that is: their
    // weights are zero.  Addresses are a uniform base and 32-bit offsets.
    __device__ __forceinline__ void fetch(const Where &x, Raw &f) const {
        const uint8_t *kbase = ks.codes + x.tok * (T * kCode), *vbase = vs.codes + x.tok * (T * kCode);
        const uint32_t n = min(lane & 31, x.count - 1);
        const uint8_t *ip = side_ids + x.tok * (S * idb) + n * (S * idb);
#pragma unroll
        for (int st = 0; st < S; ++st) f.id[st] = load_id(ip, st, a.id_wide);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint32_t off = (uint32_t)min(16 * hf + c, x.count - 1) * (T * kCode) + kb * (kCode / 4);
#pragma unroll
            for (int r = 0; r < T; ++r) {
                if (I4) f.kc4[hf][I4 ? r : 0] = load16(kbase, off + r * 64);
                else f.kc[hf][I4 ? 0 : r] = *reinterpret_cast<const uint2 *>(kbase + (off + r * 32));
            }
        }
        const uint32_t last = (uint32_t)x.count * (T * kCode) - 16;
#pragma unroll
        for (int i = 0; i < kVPieces; ++i) f.vc[i] = load16(vbase, min((uint32_t)(i * 64 + lane) * 16, last));
        __builtin_memcpy(f.sc, side_scales + x.tok * kRec + n * kRec, kRec);     // (E4M3 arrays may start anywhere)
    }
    // The tile's scales, row offsets and V codes into LDS, transposed; scales as binary16 (halved with 2-bit levels, which come as
    // 2q), K's rows' offsets in steps of `k_step` bytes
    __device__ __forceinline__ void park(const Raw &f, int k_step) const {
        const int n = lane & 31;
#pragma unroll
        for (int st = 0; st < S; ++st)
            offs[((vside ? S : 0) + st) * kTrTile + n] =
                (uint32_t)(st * a.K + min(f.id[st], (uint32_t)a.K - 1u)) * (uint32_t)(vside ? kHeadDim * 2 : k_step);
        uint16_t *sp = scales + (vside ? TG * kTrRowPitch : 0) + n;
#pragma unroll
        for (int i = 0; i < TG; ++i) {
            const uint32_t bits = FP8 ? f.sc[i / 4] >> (8 * (i & 3)) & 0x7fu : f.sc[i / 2] >> (16 * (i & 1)) & 0xffffu;
            // (E4M3 bits under binary16's exponent, seven places up, are the value times 2^-8)
            const _Float16 v = FP8 ? __builtin_bit_cast(_Float16, (uint16_t)(bits << 7)) * (_Float16)(I4 ? 256.0f : 128.0f)
                                   : __builtin_bit_cast(_Float16, (uint16_t)bits) * (_Float16)(I4 ? 1.0f : 0.5f);
            sp[i * kTrRowPitch] = __builtin_bit_cast(uint16_t, v);
        }
#pragma unroll
        for (int i = 0; i < kVPieces; ++i) {
            const int piece = i * 64 + lane, tokn = piece / kTokPieces, rest = piece - tokn * kTokPieces;
            const uint32_t wd[4] = {f.vc[i].x, f.vc[i].y, f.vc[i].z, f.vc[i].w};
            if (I4) {                                                    // four octets of a token and round
                const int r = rest / 4, oct = rest % 4 * 4;
                uint32_t *vp = reinterpret_cast<uint32_t *>(vcodes) + (r * 16 + oct) * kTrRowPitch + tokn;
#pragma unroll
                for (int e = 0; e < 4; ++e) vp[e * kTrRowPitch] = wd[e];
            } else {                                                     // eight octets
                const int r = rest / 2, oct = rest % 2 * 8;
                uint16_t *vp = vcodes + (r * 16 + oct) * kTrRowPitch + tokn;
#pragma unroll
                for (int e = 0; e < 8; ++e) vp[e * kTrRowPitch] = (uint16_t)(wd[e >> 1] >> (16 * (e & 1)));
            }
        }
    }
    // Centroid rows of tokens c and 16 + c, fragment i: channels 32 i + 8 kb + e (64 consecutive bytes of a token to four lanes), or
    // those of the residual's fragments, 32 kb + 8 i + e
    template <bool AS_RESIDUAL>
    __device__ __forceinline__ void gather_k(const Where &x, int st, uint4 (&row)[2][4]) const {
        const bf16_t *cent = ks.cent + x.page * S * a.K * kHeadDim;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint32_t off = offs[st * kTrTile + 16 * hf + c] + (AS_RESIDUAL ? 64 : 16) * kb;
#pragma unroll
            for (int i = 0; i < 4; ++i) row[hf][i] = load16(cent, off + (AS_RESIDUAL ? 16 : 64) * i);
        }
    }
    // All stages' rows of token 16 hf + c, its 32 channels 32 kb + .., and their sum in fp32
    __device__ __forceinline__ void gather_half(const Where &x, int hf, uint4 (&row)[S][4]) const {
        const bf16_t *cent = ks.cent + x.page * S * a.K * kHeadDim;
#pragma unroll
        for (int st = 0; st < S; ++st) {
            const uint32_t off = offs[st * kTrTile + 16 * hf + c] + 64 * kb;
#pragma unroll
            for (int i = 0; i < 4; ++i) row[st][i] = load16(cent, off + 16 * i);
        }
    }
    __device__ __forceinline__ void sum_rows(const uint4 (&row)[S][4], float (&v)[32]) const {
#pragma unroll
        for (int st = 0; st < S; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[8];
                unpack_bf16x8(row[st][i], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * i + e] = st ? v[8 * i + e] + x[e] : x[e];
            }
    }
    // the (cos, sin) pairs of that token and these channels
    __device__ __forceinline__ void gather_rope(const Where &x, int hf, uint4 (&rp)[4]) const {
        const int64_t at = min((int64_t)x.page_index * L + x.first + min(16 * hf + c, x.count - 1), a.t.rope_tokens - 1);
        const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const f16_t *>(a.t.k_rope_f16) + at * kHeadDim + 32 * kb);
#pragma unroll
        for (int i = 0; i < 4; ++i) rp[i] = p[i];
    }
    // Octet c of the rows of tokens 4 kb + r and 16 + 4 kb + r
    __device__ __forceinline__ void gather_v(const Where &x, int st, uint4 (&row)[8]) const {
        const bf16_t *cent = vs.cent + x.page * S * a.K * kHeadDim;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint4 o = *reinterpret_cast<const uint4 *>(offs + (S + st) * kTrTile + 16 * hf + 4 * kb);
            row[4 * hf + 0] = load16(cent, o.x + 16 * c);
            row[4 * hf + 1] = load16(cent, o.y + 16 * c);
            row[4 * hf + 2] = load16(cent, o.z + 16 * c);
            row[4 * hf + 3] = load16(cent, o.w + 16 * c);
        }
    }
    // The residual of tokens c and 16 + c as fragment i: pairs of a channel of two octets (2-bit levels), or of the halves of one.
    // Element e of a pair is channel channel(i, e), + pair_step in its upper half.
    static constexpr int pair_step = I4 ? 4 : 8;
    static __device__ __forceinline__ constexpr int channel(int i, int e) { return I4 ? 8 * i + e : 16 * (i >> 1) + 7 - 4 * (i & 1) - e; }
    // kStart: the values start from `start` (the rows' sums) instead of zero
    template <bool kStart>
    __device__ __forceinline__ void residual_k(const Raw &f, int hf, int i, const halfx2_t (&start)[4], uint4 &out) const {       // i: fragment
        const int d = i >> 1;                                            // 16 channels, which share a scale
        const uint16_t *sp = scales + ((32 * kb + 16 * d) * G / kHeadDim) * kTrRowPitch + 16 * hf + c;
        halfx2_t r[4];
#pragma unroll
        for (int rd = 0; rd < T; ++rd) {
            const _Float16 s1 = __builtin_bit_cast(_Float16, sp[rd * G * kTrRowPitch]);
            const halfx2_t s2 = {s1, s1};
            uint32_t wd;
            if (I4) { const uint4 &q4 = f.kc4[hf][I4 ? rd : 0]; wd = (i == 0 ? q4.x : i == 1 ? q4.y : i == 2 ? q4.z : q4.w) ^ 0x88888888u; }
            else { const uint2 &q2 = f.kc[hf][I4 ? 0 : rd]; wd = d ? q2.y : q2.x; }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const halfx2_t lv = I4 ? level4(wd, e) : level2(wd, 4 * (i & 1) + e);
                r[e] = rd ? fma_half2(lv, s2, r[e]) : kStart ? fma_half2(lv, s2, start[e]) : lv * s2;
            }
        }
        out = make_uint4(as_bits(r[0]), as_bits(r[1]), as_bits(r[2]), as_bits(r[3]));
    }
    // K_hat as fragments of the residual's order, rotated if ROPE: the rows' sums v and the residual meet in fp32
    template <bool ROPE>
    __device__ __forceinline__ void whole_k(const Raw &f, int hf, float (&v)[32], const uint4 (&rp)[4], uint4 (&out)[4]) const {
        const halfx2_t none[4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint4 res;
            residual_k<false>(f, hf, i, none, res);
            const uint32_t rw[4] = {res.x, res.y, res.z, res.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const halfx2_t r2 = as_half2(rw[e]);
                v[channel(i, e)] += (float)r2[0];
                v[channel(i, e) + pair_step] += (float)r2[1];
            }
        }
        if (ROPE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) rotate_octet(v + 8 * i, rp[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t x4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x4[e] = pack_f16x2_rne(v[channel(i, e)], v[channel(i, e) + pair_step]);
            out[i] = make_uint4(x4[0], x4[1], x4[2], x4[3]);
        }
    }
    // V's levels and scales of the lane's octet and tokens, and the values of channels 4 half .. 4 half + 3 as pairs of tokens
    // ([channel][pair]), from start(channel, pair)
    struct Levels { uint2 s4[T][2], w2[I4 ? 1 : T][2]; uint4 w4[I4 ? T : 1][2]; };
    __device__ __forceinline__ void read_levels(Levels &v) const {
        const uint16_t *sp = scales + (TG + 8 * c * G / kHeadDim) * kTrRowPitch + 4 * kb;
#pragma unroll
        for (int rd = 0; rd < T; ++rd)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                v.s4[rd][hf] = *reinterpret_cast<const uint2 *>(sp + rd * G * kTrRowPitch + 16 * hf);
                const int at = (rd * 16 + c) * kTrRowPitch + 16 * hf + 4 * kb;
                if (I4) v.w4[I4 ? rd : 0][hf] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint32_t *>(vcodes) + at);
                else v.w2[I4 ? 0 : rd][hf] = *reinterpret_cast<const uint2 *>(vcodes + at);
            }
    }
    template <bool kStart, class Start>
    __device__ __forceinline__ void values_v(const Levels &v, int half, Start start, uint32_t (&r)[4][4]) const {
#pragma unroll
        for (int rd = 0; rd < T; ++rd)
#pragma unroll
            for (int pr = 0; pr < 4; ++pr) {
                const uint2 &sv = v.s4[rd][pr >> 1];
                const halfx2_t s2 = as_half2(pr & 1 ? sv.y : sv.x);
                uint32_t x;
                if (I4) {
                    const uint4 &wv = v.w4[I4 ? rd : 0][pr >> 1];
                    x = __builtin_amdgcn_perm(pr & 1 ? wv.w : wv.y, pr & 1 ? wv.z : wv.x, half ? 0x07060302u : 0x05040100u) ^ 0x88888888u;
                } else {
                    const uint2 &wv = v.w2[I4 ? 0 : rd][pr >> 1];
                    x = pr & 1 ? wv.y : wv.x;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const halfx2_t lv = I4 ? level4(x, e) : level2(x, 7 - (4 * half + e));
                    r[e][pr] = as_bits(rd ? fma_half2(lv, s2, as_half2(r[e][pr])) : kStart ? fma_half2(lv, s2, start(4 * half + e, pr)) : lv * s2);
                }
            }
    }
    // the word of a row that holds channel j of the octet; channel j of two rows as binary16
    static __device__ __forceinline__ uint32_t word_of(const uint4 &row, int j) { return j < 2 ? row.x : j < 4 ? row.y : j < 6 ? row.z : row.w; }
    static __device__ __forceinline__ halfx2_t pair_f16(const uint4 &ra, const uint4 &rb, int j) {
        const uint32_t wa = word_of(ra, j), wb = word_of(rb, j);
        return as_half2(j & 1 ? pack_f16x2_rne(bf16_hi(wa), bf16_hi(wb)) : pack_f16x2_rne(bf16_lo(wa), bf16_lo(wb)));
    }
};

// The running soft-max of a lane's query rows: row c of RB blocks of 16, the scores of a tile's tokens 16 hf + 4 kb + r in s[.][hf][r],
// channels 32 kb + 8 r + j of the row's sums in o[.][j][r].
template <int RB>
struct TreeRows {
    floatx4_t o[RB][8], s[RB][2];
    float m[RB], l[RB], qs[RB];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            m[rb] = kTrNoScore; l[rb] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[rb][j] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
    __device__ __forceinline__ void clear_scores() {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) s[rb][hf] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // the row sees token i of the tile where bit i of see[rb] is set
    __device__ __forceinline__ void hide(const uint32_t (&see)[RB]) {
        const int kb = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s[rb][e >> 2][e & 3] = (see[rb] >> (16 * (e >> 2) + 4 * kb + (e & 3))) & 1u ? s[rb][e >> 2][e & 3] : -INFINITY;
    }
    // The weights of the tile's scores: use(rb, x) gets the eight of block rb.  A score is rounded before the reference is taken
    // from it, as the reference was, and the two are compared by their difference: fused, or against a rounded sum, a weight of
    // scores beyond 2^24 left binary16's range.
    template <class Use>
    __device__ __forceinline__ void weights(Use use) {
        float top[RB];
        bool move = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const floatx4_t &x = s[rb][0], &y = s[rb][1];
            top[rb] = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]))) * qs[rb];
            move |= top[rb] - m[rb] > kTrBelow + kTrLag;
        }
        if (__ballot(move)) {                                            // uniform: some row's reference moves
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float x = fmaxf(top[rb], __shfl_xor(top[rb], 16, 64));
                x = fmaxf(x, __shfl_xor(x, 32, 64));
                const float m_new = fmaxf(m[rb], x - kTrBelow), alpha = __builtin_amdgcn_exp2f(m[rb] - m_new);
                l[rb] *= alpha; m[rb] = m_new;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[rb][j] *= alpha;
            }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) { x[e] = __builtin_amdgcn_exp2f(s[rb][e >> 2][e & 3] * qs[rb] - m[rb]); l[rb] += x[e]; }
            use(rb, x);
        }
    }
};

// A query row's place and scale: the power of two (as 9 - its exponent) that brings the row's largest value to 2^8 .. 2^9, where
// binary16 holds all but what is 2^-22 of it; the row's scores are then times 2^(ex - 9).  v: the lane's 32 channels 32 kb + ..
struct QueryRow {
    const bf16_t *at; int node, ex;                                      // at: nullptr, node: -1 where there is no row
    __device__ __forceinline__ QueryRow(const TreeArgs &a, const SeqTiles &sq, int b, int h, int64_t r, float (&v)[32]) {
        const int kb = (threadIdx.x & 63) >> 4;
        at = nullptr; node = -1;
        if (r < (int64_t)a.t.group * a.t.n_nodes) {
            const RowPlace p = place_row(a, h, r);
            if (p.node < sq.nodes) {
                node = p.node;
                at = static_cast<const bf16_t *>(a.t.q) + b * a.t.q_stride_seq + p.head * a.t.q_stride_head + p.node * a.t.q_stride_node;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) octet(4 * kb + i, v + 8 * i);
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) top = fmaxf(top, __builtin_fabsf(v[i]));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        ex = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : 0;
    }
    __device__ __forceinline__ void octet(int oct, float *v) const {
        unpack_bf16x8(at ? *reinterpret_cast<const uint4 *>(at + 8 * oct) : make_uint4(0u, 0u, 0u, 0u), v);
    }
    // (never zero: a hidden token's score is -inf times it; scores that small are zero against any other)
    __device__ __forceinline__ float scale(const TreeArgs &a) const {
        return fmaxf(__builtin_amdgcn_ldexpf(a.scale * 1.4426950408889634f, ex - 9), 1.17549435e-38f);
    }
    // fragment i in the residual's order, of the lane's channels v (scaled already)
    template <class F>
    static __device__ __forceinline__ uint4 residual_fragment(const float (&v)[32], int i) {
        typedef TreeLane<F> Lane;
        uint32_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = pack_f16x2_rne(v[Lane::channel(i, e)], v[Lane::channel(i, e) + Lane::pair_step]);
        return make_uint4(x[0], x[1], x[2], x[3]);
    }
};

// The wavefronts' results meet: O, m and l of each (m the same in a row's four lanes, l a lane's share), the block's result
// to `state` or, undivided, to the output.  meet: [kTrWaves][16][kTrPitch] floats.
template <int RB>
__device__ __forceinline__ void finish_block(const TreeArgs &a, const BlockPlace &at, int nodes, float (*meet)[16][kTrPitch],
                                             float (*ms)[16 * RB], float (*ls)[16 * RB], const floatx4_t (&O)[RB][8], const float (&m)[RB], float (&l)[RB]) {
    constexpr int kRows = 16 * RB;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 15, kb = lane >> 4;
    const int64_t rows = (int64_t)a.t.group * a.t.n_nodes;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        l[rb] += __shfl_xor(l[rb], 16, 64);
        l[rb] += __shfl_xor(l[rb], 32, 64);
        if (kb == 0) { ms[wave][rb * 16 + c] = m[rb]; ls[wave][rb * 16 + c] = l[rb]; }
    }
    __syncthreads();
    const int row = tid >> 4, c8 = tid & 15;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float mm = ms[0][rb * 16 + c];
#pragma unroll
        for (int v = 1; v < kTrWaves; ++v) mm = fmaxf(mm, ms[v][rb * 16 + c]);
        const float f = __builtin_amdgcn_exp2f(m[rb] - mm);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 8; j += 4)
                *reinterpret_cast<float4 *>(&meet[wave][c][32 * kb + 8 * r + j]) =
                    make_float4(O[rb][j][r] * f, O[rb][j + 1][r] * f, O[rb][j + 2][r] * f, O[rb][j + 3][r] * f);
        __syncthreads();
        const int64_t r = (int64_t)at.rblk * kRows + rb * 16 + row;
        float o[8], mt = ms[0][rb * 16 + row], lt = 0.0f;
#pragma unroll
        for (int v = 1; v < kTrWaves; ++v) mt = fmaxf(mt, ms[v][rb * 16 + row]);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll
        for (int v = 0; v < kTrWaves; ++v) {
            lt += ls[v][rb * 16 + row] * __builtin_amdgcn_exp2f(ms[v][rb * 16 + row] - mt);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += meet[v][row][c8 * 8 + e];
        }
        if (a.slots) {
            float *st = a.state + at.state;
            float *op = st + (rb * 16 + row) * kHeadDim + c8 * 8;
            *reinterpret_cast<float4 *>(op) = make_float4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<float4 *>(op + 4) = make_float4(o[4], o[5], o[6], o[7]);
            if (c8 == 0) { st[kRows * kHeadDim + rb * 16 + row] = mt; st[kRows * (kHeadDim + 1) + rb * 16 + row] = lt; }
        } else if (r < rows) store_row8(a, at.b, at.h, r, nodes, c8, o, mt, lt);
        if (rb + 1 < RB) __syncthreads();
    }
}

// Which of the new tokens first .. first + 31 node i sees (`there`: those that are there).
__device__ __forceinline__ uint32_t node_sees(const qvg_tree_step &t, int b, int node, int first, uint32_t there) {
    if (node < 0) return 0u;
    if (t.mask) return there & t.mask[((int64_t)b * t.n_nodes + node) * ((t.n_nodes + 31) / 32) + first / 32];
    const int left = node - first;                                       // sees tokens first .. first + left
    return there & (left < 0 ? 0u : (left >= 31 ? 0xffffffffu : (2u << left) - 1u));
}

}  // namespace qvg
