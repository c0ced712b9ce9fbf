// Attention of the few new tokens of a step (one token, or a tree of drafted ones) over a sequence's compressed pages, its
// bf16 tail and the new tokens themselves:
//     o = sum_n w_n v_n / sum_n w_n,   w_n = exp(scale q.k_n),   k_n, v_n = sum_s c_s[id_s(n)] + sum_t s_t(n) q_t(n)  (Eq. 7)
// in one pass over the tokens with the running maximum and sum of the soft-max.
//
// A workgroup takes a block of 16, 32 or 64 query rows of one KV head (rows = group x new tokens) and a part of the
// sequence's tiles of 32 tokens; each of its wavefronts walks tiles of its own and nothing is exchanged before the end, so
// there is no barrier in the loop.  The contractions run on v_mfma_f32_16x16x32_f16 with the operands where the decoding
// puts them, so a decoded tile passes through registers only:
//   S^T = K Q^T:   lane (c, kb) decodes channels 32 kb .. 32 kb + 31 of tokens c and 16 + c; the order of a contraction is
//                  free, so MFMA i takes channels 32 kb + 8 i + e and Q's fragments are loaded the same way;
//   O^T += V^T P:  lane (c, kb) decodes the octet of channels 8 c .. 8 c + 7 of tokens 4 kb + r and 16 + 4 kb + r, which are
//                  the tokens whose scores S^T leaves in the lane: P needs no movement, and pairs of tokens are packed as
//                  they are rounded, which is the transposition.  MFMA j makes channels 8 c + j; the lane ends up with
//                  channels 32 kb .. 32 kb + 31 of query row c.
#include "qvg_tree.hpp"

namespace qvg {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4_t;

constexpr int kTrThreads = 256, kTrWaves = kTrThreads / 64, kTrTile = 32;
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
    s.per_page = (L + kTrTile - 1) / kTrTile;
    const int full = s.kv / L;
    s.kv_tiles = full * s.per_page + (s.kv - full * L + kTrTile - 1) / kTrTile;
    s.tail_tiles = (s.tail + kTrTile - 1) / kTrTile;
    s.total = s.kv_tiles + s.tail_tiles + (s.nodes + kTrTile - 1) / kTrTile;
    return s;
}

// fp32 values of channels 8 oct .. 8 oct + 7 of pool token n of the unit (in page `page`)
template <int FMT>
__device__ __forceinline__ void decode_octet(const TreeArgs &a, const PoolSide &s, int64_t page, int64_t n, int oct, float *acc) {
    constexpr bool FP8 = (FMT & kFmtE4M3) != 0, I4 = (FMT & kFmtInt4) != 0;
    const uint32_t kmax = (uint32_t)a.K - 1u;
    for (int st = 0; st < a.S; ++st) {
        const uint32_t id = min(load_id(s.ids, n * a.S + st, a.id_wide), kmax);
        float row[8];
        unpack_bf16x8(*reinterpret_cast<const uint4 *>(s.cent + ((page * a.S + st) * a.K + id) * kHeadDim + oct * 8), row);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = st ? acc[e] + row[e] : row[e];
    }
    const int G = kHeadDim / a.B, g = oct * 8 / a.B;
    for (int t = 0; t < a.T; ++t) {
        const int64_t rec = n * a.T + t;
        const float sc = FP8 ? e4m3_bits_to_f32(s.scales[rec * G + g])
                             : f16_bits_to_f32(reinterpret_cast<const f16_t *>(s.scales)[rec * G + g]);
        if (I4) add_stage_int4(acc, reinterpret_cast<const uint32_t *>(s.codes)[rec * 16 + oct], sc);
        else {
            const uint32_t w = reinterpret_cast<const uint16_t *>(s.codes)[rec * 16 + oct];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int q = ((int)(w << (30 - 2 * e))) >> 30;
                acc[e] = __builtin_fmaf(sc, (float)q, acc[e]);
            }
        }
    }
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

// A block's partial result: [rows][128] sums, then the rows' references, then their sums of weights.
__host__ __device__ inline int64_t tree_state_floats(int rows) { return (int64_t)rows * (kHeadDim + 2); }

// The wavefronts' results meet: O, m and l of each (m the same in a row's four lanes, l a lane's share), the block's result
// to `state` or, undivided, to the output.  meet: [kTrWaves][16][kTrPitch] floats.
template <int RB>
__device__ __forceinline__ void finish_block(const TreeArgs &a, int b, int h, int bh, int rblk, int part, int nodes, float (*meet)[16][kTrPitch],
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
        const int64_t r = (int64_t)rblk * kRows + rb * 16 + row;
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
        if (a.parts > 1) {
            float *st = a.state + (((int64_t)bh * a.row_blocks + rblk) * a.parts + part) * tree_state_floats(kRows);
            float *op = st + (rb * 16 + row) * kHeadDim + c8 * 8;
            *reinterpret_cast<float4 *>(op) = make_float4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<float4 *>(op + 4) = make_float4(o[4], o[5], o[6], o[7]);
            if (c8 == 0) { st[kRows * kHeadDim + rb * 16 + row] = mt; st[kRows * (kHeadDim + 1) + rb * 16 + row] = lt; }
        } else if (r < rows) store_row8(a, b, h, r, nodes, c8, o, mt, lt);
        if (rb + 1 < RB) __syncthreads();
    }
}

template <int FMT, int RB>
__global__ __launch_bounds__(kTrThreads, 2)
void tree_attn_kernel(TreeArgs a, int blocks, int per_xcd) {
    constexpr int kRows = 16 * RB;
    __shared__ float meet[kTrWaves][16][kTrPitch];
    __shared__ float ms[kTrWaves][kRows], ls[kTrWaves][kRows];
    // workgroups are dealt to the 8 XCDs round-robin: the parts of one KV head run on one, whose L2 then keeps its tables
    const int w = (int)(blockIdx.x % 8u) * per_xcd + (int)(blockIdx.x / 8u);
    if (w >= blocks) return;                                             // uniform, before any barrier
    const int part = w % a.parts, rblk = w / a.parts % a.row_blocks, bh = w / a.parts / a.row_blocks;
    const int b = bh / a.H, h = bh - b * a.H;
    const qvg_tree_step &t = a.t;
    const SeqTiles sq = tiles_of_sequence(t, b);
    const int lo = (int)((int64_t)sq.total * part / a.parts), hi = (int)((int64_t)sq.total * (part + 1) / a.parts);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, kb = lane >> 4;
    const int64_t rows = (int64_t)t.group * t.n_nodes;

    // Q: the row's values times a power of two that brings its largest to 2^8 .. 2^9, as binary16 (exact, but for what is
    // 2^-22 of the largest or less)
    halfx8_t q[RB][4];
    float qs[RB];
    int node[RB];                                                        // -1: no such row
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int64_t r = (int64_t)rblk * kRows + rb * 16 + c;
        node[rb] = -1; qs[rb] = 0.0f;
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
        if (r < rows) {
            const RowPlace p = place_row(a, h, r);
            if (p.node < sq.nodes) {
                node[rb] = p.node;
                const bf16_t *qp = static_cast<const bf16_t *>(t.q) + b * t.q_stride_seq + p.head * t.q_stride_head + p.node * t.q_stride_node + 32 * kb;
#pragma unroll
                for (int i = 0; i < 4; ++i) unpack_bf16x8(*reinterpret_cast<const uint4 *>(qp + 8 * i), v[i]);
            }
        }
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, __builtin_fabsf(v[i][e]));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const int ex = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = __builtin_amdgcn_ldexpf(v[i][e], 9 - ex);
            q[rb][i] = pack_f16x8(v[i]);
        }
        qs[rb] = __builtin_amdgcn_ldexpf(a.scale * 1.4426950408889634f, ex - 9);
    }

    PoolSide ks = a.k, vs = a.v;
    {
        const int64_t tok = (int64_t)h * t.pool_pages * t.page_len;
        const int idb = a.id_wide ? 2 : 1, cb = (FMT & kFmtInt4) ? 64 : 32, sb = (FMT & kFmtE4M3) ? 1 : 2;
        ks.cent += (int64_t)h * t.pool_pages * a.S * a.K * kHeadDim;  vs.cent += (int64_t)h * t.pool_pages * a.S * a.K * kHeadDim;
        ks.ids += tok * a.S * idb;                                      vs.ids += tok * a.S * idb;
        ks.codes += tok * a.T * cb;                                     vs.codes += tok * a.T * cb;
        ks.scales += tok * a.T * (kHeadDim / a.B) * sb;                 vs.scales += tok * a.T * (kHeadDim / a.B) * sb;
    }

    floatx4_t O[RB][8];
    float m[RB], l[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kTrNoScore; l[rb] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) O[rb][j] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    for (int ti = lo + wave; ti < hi; ti += kTrWaves) {
        // the tile: its first token (in the page, the tail or the new tokens) and how many it has
        int kind = 0, first, count;
        int64_t page = 0, pool_tok = 0;
        int place = 0;                                                   // of its first token in the sequence (compressed)
        if (ti < sq.kv_tiles) {
            const int pi = ti / sq.per_page;
            first = (ti - pi * sq.per_page) * kTrTile;
            const int in_page = min((int)t.page_len, sq.kv - pi * (int)t.page_len);
            count = min(kTrTile, in_page - first);
            int64_t pg = t.page_table[(int64_t)b * t.table_pages + pi];
            page = pg < 0 ? 0 : (pg >= t.pool_pages ? t.pool_pages - 1 : pg);
            pool_tok = page * t.page_len + first;
            place = pi * (int)t.page_len + first;
        } else if (ti < sq.kv_tiles + sq.tail_tiles) {
            kind = 1; first = (ti - sq.kv_tiles) * kTrTile; count = min(kTrTile, sq.tail - first);
        } else {
            kind = 2; first = (ti - sq.kv_tiles - sq.tail_tiles) * kTrTile; count = min(kTrTile, sq.nodes - first);
        }
        const uint32_t there = count >= 32 ? 0xffffffffu : (1u << count) - 1u;
        // which of the tile's tokens each row sees, and which any row of the block sees
        uint32_t see[RB], any = there;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) see[rb] = node[rb] >= 0 ? there : 0u;
        if (kind == 2) {
            any = 0u;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                if (node[rb] >= 0) {
                    if (t.mask) see[rb] &= t.mask[((int64_t)b * t.n_nodes + node[rb]) * ((t.n_nodes + 31) / 32) + first / 32];
                    else {
                        const int left = node[rb] - first;                 // sees tokens first .. first + left
                        see[rb] &= left < 0 ? 0u : (left >= 31 ? 0xffffffffu : (2u << left) - 1u);
                    }
                }
                any |= see[rb];
            }
#pragma unroll
            for (int off = 1; off < 16; off *= 2) any |= __shfl_xor(any, off, 64);
        }

        const bf16_t *kr, *vr;                                           // bf16 tokens: first row and stride
        int64_t stride;
        if (kind == 1) {
            stride = t.tail_stride_token;
            const int64_t off = b * t.tail_stride_seq + h * t.tail_stride_head + first * stride;
            kr = static_cast<const bf16_t *>(t.k_tail) + off; vr = static_cast<const bf16_t *>(t.v_tail) + off;
        } else {
            stride = t.new_stride_node;
            const int64_t off = b * t.new_stride_seq + h * t.new_stride_head + first * stride;
            kr = static_cast<const bf16_t *>(t.k_new) + off; vr = static_cast<const bf16_t *>(t.v_new) + off;
        }

        // ---- S^T = K Q^T -------------------------------------------------------------------
        floatx4_t S[RB][2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int tok = min(16 * hf + c, count - 1);                 // a token that is not there reads the last one
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) S[rb][hf] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float acc[8];
                if (kind == 0) {
                    decode_octet<FMT>(a, ks, page, pool_tok + tok, 4 * kb + i, acc);
                    if (t.k_rope_f16) {
                        const int64_t at = min((int64_t)place + tok, t.rope_tokens - 1);
                        rotate_octet(acc, *reinterpret_cast<const uint4 *>(static_cast<const f16_t *>(t.k_rope_f16) + at * kHeadDim + (4 * kb + i) * 8));
                    }
                } else unpack_bf16x8(*reinterpret_cast<const uint4 *>(kr + tok * stride + (4 * kb + i) * 8), acc);
                const halfx8_t kf = pack_f16x8(acc);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) S[rb][hf] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, q[rb][i], S[rb][hf], 0, 0, 0);
            }
        }

        // ---- soft-max: the lane has tokens 16 hf + 4 kb + r of row c ------------------------
        halfx8_t P[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int tok = 16 * (e >> 2) + 4 * kb + (e & 3);
                x[e] = (see[rb] >> tok) & 1u ? S[rb][e >> 2][e & 3] * qs[rb] : -INFINITY;
            }
            float top = x[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
            if (__ballot(top > m[rb] + (kTrBelow + kTrLag))) {            // uniform: some row's reference moves
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float m_new = fmaxf(m[rb], top - kTrBelow), alpha = __builtin_amdgcn_exp2f(m[rb] - m_new);
                l[rb] *= alpha; m[rb] = m_new;
#pragma unroll
                for (int j = 0; j < 8; ++j) O[rb][j] *= alpha;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) { x[e] = __builtin_amdgcn_exp2f(x[e] - m[rb]); l[rb] += x[e]; }
            P[rb] = pack_f16x8(x);
        }

        // ---- O^T += V^T P ----------------------------------------------------------------------
        uint32_t vp[8][4];                                               // channel j: pairs of tokens
#pragma unroll
        for (int pr = 0; pr < 4; ++pr) {
            float acc[2][8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int slot = 16 * (pr >> 1) + 4 * kb + 2 * (pr & 1) + e, tok = min(slot, count - 1);
                if (kind == 0) decode_octet<FMT>(a, vs, page, pool_tok + tok, c, acc[e]);
                else {
                    unpack_bf16x8(*reinterpret_cast<const uint4 *>(vr + tok * stride + c * 8), acc[e]);
                    // (a new token that no row sees may be no number)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[e][j] = (any >> slot) & 1u ? acc[e][j] : 0.0f;
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) vp[j][pr] = pack_f16x2_rne(acc[0][j], acc[1][j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const halfx8_t vf = __builtin_bit_cast(halfx8_t, make_uint4(vp[j][0], vp[j][1], vp[j][2], vp[j][3]));
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) O[rb][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, P[rb], O[rb][j], 0, 0, 0);
        }
    }

    finish_block<RB>(a, b, h, bh, rblk, part, sq.nodes, meet, ms, ls, O, m, l);
}

// ---- the packed form ------------------------------------------------------------------------------
// Up to four rounds of 2-bit levels, or one of 4-bit levels (any scale format, id width and number of smoothing stages).
// The sum over Eq. 7's parts is left to the contractions where that saves vector instructions, of which the decoding is
// made: the centroid rows go to the matrix cores as they are stored, as bf16, and only the residual of the rounds,
// sum_t s_t q_t, is formed, two elements at a time in packed binary16 arithmetic (one round: exact).  So S^T = C Q^T + R Q^T
// with Q as bf16 and as binary16, and O^T = C^T P + R^T P with P as a sum of two bf16 numbers (16 significant bits; one would
// cost 2^-9 of every weight) and as binary16.
// A token's part q.c of a score depends on its centroid alone: at the start of a page the workgroup contracts the page's tables
// with its queries once and keeps the scores of all rows in LDS, where the tokens' accumulators start from what their ids name.
// (Gathering K's rows as well, 256 bytes per token and side, the loop was bound by what the L2s give to gathers, about 10 TB/s:
// one token over 12 heads x 187200 tokens of one round 125 us instead of ... .)  V's rows are gathered, 16 bytes per lane, row and octet.
// A tile's codes and scales come in with a few wide loads a tile ahead; the V side's codes, all scales and ids pass through a few KB of LDS that are the wavefront's own, where they are
// transposed: tokens become contiguous, so that a lane reads four tokens' levels or scales, already paired, at once.
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
// before it is used (as run-time branches between forms the loop took 1.0 instead of ... us).
template <int RB> __host__ __device__ constexpr int tree_query_bytes() { return RB * 8 * 1024; }
template <int T_, int G_, bool FP8_, bool I4_, int S_>
struct TreeFormat {
    static constexpr int T = T_, G = G_, S = S_, TG = T * G;             // rounds, groups per token, smoothing stages
    static constexpr bool FP8 = FP8_, I4 = I4_;
    static constexpr int code = I4 ? 64 : 32;                            // code bytes per token and round
    static constexpr int record = TG * (FP8 ? 1 : 2);                    // scale bytes per token
    // bytes of a wavefront's LDS: V codes [T][16 octets][32 tokens], scales [2][T * G][32], row offsets [2][S][32]
    static constexpr int wave_bytes = T * 16 * kTrRowPitch * (I4 ? 4 : 2) + 2 * TG * kTrRowPitch * 2 + 2 * S * kTrTile * 4;
};
constexpr int kTrMeetBytes = kTrWaves * 16 * kTrPitch * 4;

template <class F, bool ROPE, int RB>
__global__ __launch_bounds__(kTrThreads, 2)
void tree_attn_packed(TreeArgs a, int blocks, int per_xcd) {
    constexpr int T = F::T, G = F::G, TG = F::TG, S = F::S, kCode = F::code, kRec = F::record;
    constexpr bool I4 = F::I4, FP8 = F::FP8;
    constexpr int kRows = 16 * RB;
    // One block of 16 rows takes V's rows as they are and P twice; for more rows the values are put together in binary16, 96
    // instructions a tile, and P is taken once, which saves 24 instructions, eight registers and 16 contractions a block
    constexpr bool kSplitV = RB == 1;
    constexpr int kVPieces = T * kCode / 32, kTokPieces = T * kCode / 16;   // 16-byte pieces of the V codes: to a lane, of a token
    // the scores of the centroids in LDS; not where keys are rotated, nor where four stages' tables and 32 rows would leave a
    // CU one workgroup
    constexpr bool kTable = !ROPE && (S == 1 || RB == 1);
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float ms[kTrWaves][kRows], ls[kTrWaves][kRows];
    const int w = (int)(blockIdx.x % 8u) * per_xcd + (int)(blockIdx.x / 8u);
    if (w >= blocks) return;                                             // uniform, before any barrier
    const int part = w % a.parts, rblk = w / a.parts % a.row_blocks, bh = w / a.parts / a.row_blocks;
    const int b = bh / a.H, h = bh - b * a.H;
    const qvg_tree_step &t = a.t;
    const SeqTiles sq = tiles_of_sequence(t, b);
    const int lo = (int)((int64_t)sq.total * part / a.parts), hi = (int)((int64_t)sq.total * (part + 1) / a.parts);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, kb = lane >> 4;
    const int64_t rows = (int64_t)t.group * t.n_nodes;
    uint4 *qlds = reinterpret_cast<uint4 *>(smem);                       // [RB][8][64] fragments
    unsigned char *own = smem + tree_query_bytes<RB>() + wave * F::wave_bytes;
    uint16_t *vcodes = reinterpret_cast<uint16_t *>(own);
    uint16_t *scales = vcodes + T * 16 * kTrRowPitch * (I4 ? 2 : 1);
    uint32_t *offs = reinterpret_cast<uint32_t *>(scales + 2 * TG * kTrRowPitch);
    float *table = reinterpret_cast<float *>(smem + tree_query_bytes<RB>() + kTrWaves * F::wave_bytes);   // [S * K][kRows], kTable

    // ---- Q: fragments 0..3 as bf16 (channels 32 i + 8 kb + e: a row's gathers then read 64 consecutive bytes of a token with four
    // lanes), 4..7 as binary16 in the order of the residual's fragments (channels 32 kb + ..) ----
    float qs[RB];
    int node[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int64_t r = (int64_t)rblk * kRows + rb * 16 + c;
        node[rb] = -1;
        const bf16_t *qp = nullptr;
        if (r < rows) {
            const RowPlace p = place_row(a, h, r);
            if (p.node < sq.nodes) {
                node[rb] = p.node;
                qp = static_cast<const bf16_t *>(t.q) + b * t.q_stride_seq + p.head * t.q_stride_head + p.node * t.q_stride_node;
            }
        }
        auto octet = [&](int oct, float *v) {
            unpack_bf16x8(qp ? *reinterpret_cast<const uint4 *>(qp + 8 * oct) : make_uint4(0u, 0u, 0u, 0u), v);
        };
        float v[32], top = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) octet(4 * kb + i, v + 8 * i);
#pragma unroll
        for (int i = 0; i < 32; ++i) top = fmaxf(top, __builtin_fabsf(v[i]));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const int ex = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : 0;
        qs[rb] = __builtin_amdgcn_ldexpf(a.scale * 1.4426950408889634f, ex - 9);
        if (wave == rb % kTrWaves) {                                     // one wavefront leaves them for all
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __builtin_amdgcn_ldexpf(v[i], 9 - ex);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] = I4 ? pack_f16x2_rne(v[8 * i + e], v[8 * i + 4 + e])
                              : pack_f16x2_rne(v[16 * (i >> 1) + 7 - 4 * (i & 1) - e], v[16 * (i >> 1) + 15 - 4 * (i & 1) - e]);
                qlds[(rb * 8 + 4 + i) * 64 + lane] = make_uint4(x[0], x[1], x[2], x[3]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                octet(4 * i + kb, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __builtin_amdgcn_ldexpf(v[e], 9 - ex);
                qlds[(rb * 8 + i) * 64 + lane] = pack_bf16x8(v);
            }
        }
    }
    __syncthreads();
    auto qfrag = [&](int rb, int i) { return qlds[(rb * 8 + i) * 64 + lane]; };

    PoolSide ks = a.k, vs = a.v;
    const int idb = a.id_wide ? 2 : 1;
    {
        const int64_t tok = (int64_t)h * t.pool_pages * t.page_len, tables = (int64_t)h * t.pool_pages * S * a.K * kHeadDim;
        ks.cent += tables;              vs.cent += tables;
        ks.ids += tok * S * idb;        vs.ids += tok * S * idb;
        ks.codes += tok * T * kCode;    vs.codes += tok * T * kCode;
        ks.scales += tok * kRec;        vs.scales += tok * kRec;
    }

    floatx4_t O[RB][8];
    float m[RB], l[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kTrNoScore; l[rb] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) O[rb][j] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    floatx4_t Sc[RB][2];
    auto clear_scores = [&]() {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) Sc[rb][hf] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
    };
    // bf16 rows: fragment i of both halves of the tile's tokens
    auto scores_of_rows = [&](const uint4 (&row)[2][4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const bf16x8_t q = __builtin_bit_cast(bf16x8_t, qfrag(rb, i));
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                    Sc[rb][hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, row[hf][i]), q, Sc[rb][hf], 0, 0, 0);
            }
    };
    uint4 Phi[1], Plo[1], Ph[RB];
    // the lane's row sees token i of the tile where bit i of see[rb] is set
    auto hide = [&](const uint32_t (&see)[RB]) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                Sc[rb][e >> 2][e & 3] = (see[rb] >> (16 * (e >> 2) + 4 * kb + (e & 3))) & 1u ? Sc[rb][e >> 2][e & 3] : -INFINITY;
    };
    // soft-max of the tile's scores
    auto weights = [&]() {
        float top[RB];
        bool move = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const floatx4_t &x = Sc[rb][0], &y = Sc[rb][1];
            top[rb] = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]))) * qs[rb];
            move |= top[rb] > m[rb] + (kTrBelow + kTrLag);
        }
        if (__ballot(move)) {                                            // uniform: some row's reference moves
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float x = fmaxf(top[rb], __shfl_xor(top[rb], 16, 64));
                x = fmaxf(x, __shfl_xor(x, 32, 64));
                const float m_new = fmaxf(m[rb], x - kTrBelow), alpha = __builtin_amdgcn_exp2f(m[rb] - m_new);
                l[rb] *= alpha; m[rb] = m_new;
#pragma unroll
                for (int j = 0; j < 8; ++j) O[rb][j] *= alpha;
            }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float x[8];
            uint32_t ph[4], pl[4], pf[4];
#pragma unroll
            for (int e = 0; e < 8; ++e) { x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(Sc[rb][e >> 2][e & 3], qs[rb], -m[rb])); l[rb] += x[e]; }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pf[e] = pack_f16x2_rne(x[2 * e], x[2 * e + 1]);
                if (!kSplitV) continue;
                ph[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
                pl[e] = pack_bf16x2(x[2 * e] - bf16_lo(ph[e]), x[2 * e + 1] - bf16_hi(ph[e]));
            }
            Ph[rb] = make_uint4(pf[0], pf[1], pf[2], pf[3]);
            if (kSplitV) {
                Phi[0] = make_uint4(ph[0], ph[1], ph[2], ph[3]);
                Plo[0] = make_uint4(pl[0], pl[1], pl[2], pl[3]);
            }
        }
    };
    // the word of a row that holds channel j of the lane's octet; channel j of a pair of rows, as bf16 and as binary16
    auto word_of = [](const uint4 &row, int j) { return j < 2 ? row.x : j < 4 ? row.y : j < 6 ? row.z : row.w; };
    auto pair_f16 = [&](const uint4 &ra, const uint4 &rb_, int j) {
        const uint32_t wa = word_of(ra, j), wb = word_of(rb_, j);
        return as_half2(j & 1 ? pack_f16x2_rne(bf16_hi(wa), bf16_hi(wb)) : pack_f16x2_rne(bf16_lo(wa), bf16_lo(wb)));
    };
    auto add_pv = [&](int j, const uint32_t (&x)[4]) {
        const halfx8_t v = __builtin_bit_cast(halfx8_t, make_uint4(x[0], x[1], x[2], x[3]));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) O[rb][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, __builtin_bit_cast(halfx8_t, Ph[rb]), O[rb][j], 0, 0, 0);
    };
    // O^T += (bf16 rows of the lane's eight tokens)^T P
    auto add_rows = [&](const uint4 (&row)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t x[4];
            if (kSplitV) {
#pragma unroll
                for (int pr = 0; pr < 4; ++pr)
                    x[pr] = __builtin_amdgcn_perm(word_of(row[2 * pr + 1], j), word_of(row[2 * pr], j), j & 1 ? 0x07060302u : 0x05040100u);
                const bf16x8_t v = __builtin_bit_cast(bf16x8_t, make_uint4(x[0], x[1], x[2], x[3]));
                O[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, Phi[0]), O[0][j], 0, 0, 0);
                O[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, Plo[0]), O[0][j], 0, 0, 0);
            } else {
#pragma unroll
                for (int pr = 0; pr < 4; ++pr) x[pr] = as_bits(pair_f16(row[2 * pr], row[2 * pr + 1], j));
                add_pv(j, x);
            }
        }
    };
    auto order_lds = []() { asm volatile("" ::: "memory"); };             // the wavefront's LDS operations stay in this order

    // ---- compressed tiles ----------------------------------------------------------------------
    struct Where { int page_index, first, count; int64_t page, tok; };    // of a tile; tok: its first token in the pool
    const int L = sq.kv ? (int)t.page_len : 1;
    auto place = [&](int pi, int in_page, const Where &last) {            // (a tile of the page before needs no table)
        Where x;
        x.page_index = pi; x.first = in_page * kTrTile;
        x.count = min(kTrTile, min(L, sq.kv - pi * L) - x.first);
        x.page = last.page;
        if (pi != last.page_index) {
            const int64_t pg = __builtin_amdgcn_readfirstlane(t.page_table[(int64_t)b * t.table_pages + pi]);
            x.page = pg < 0 ? 0 : (pg >= t.pool_pages ? t.pool_pages - 1 : pg);
        }
        x.tok = x.page * L + x.first;
        return x;
    };
    // What a lane fetches of a tile: of tokens c and 16 + c the K codes of its 32 channels; 16-byte pieces of the V codes; the
    // scale record and the ids of one token (lanes 0..31: K, 32..63: V).  What belongs to tokens that are not there is read from
    // the tile's last token instead, whatever piece of it that is: their weights are zero.  Addresses are a uniform base and
    // 32-bit offsets.
    struct Raw { uint4 kc4[2][I4 ? T : 1]; uint2 kc[2][I4 ? 1 : T]; uint4 vc[kVPieces]; uint32_t sc[(kRec + 3) / 4], id[S]; };
    const bool vside = lane >= 32;
    const uint8_t *side_scales = vside ? vs.scales : ks.scales, *side_ids = vside ? vs.ids : ks.ids;
    auto load16 = [](const void *base, uint32_t off) { return *reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(base) + off); };
    auto fetch = [&](const Where &x, Raw &f) {
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
    };
    // The tile's scales, row offsets and V codes into LDS, transposed; scales as binary16 (halved with 2-bit levels, which come as 2q)
    auto park = [&](const Raw &f) {
        const int n = lane & 31;
#pragma unroll
        for (int st = 0; st < S; ++st)
            offs[((vside ? S : 0) + st) * kTrTile + n] =
                (uint32_t)(st * a.K + min(f.id[st], (uint32_t)a.K - 1u)) * (uint32_t)(kTable && !vside ? kRows * 4 : kHeadDim * 2);
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
    };
    auto gather_k = [&](const Where &x, int st, uint4 (&row)[2][4]) {
        const bf16_t *cent = ks.cent + x.page * S * a.K * kHeadDim;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            // (as Q's fragments take them; the rotation wants them as the residual is)
            const uint32_t off = offs[st * kTrTile + 16 * hf + c] + (ROPE ? 64 : 16) * kb;
#pragma unroll
            for (int i = 0; i < 4; ++i) row[hf][i] = load16(cent, off + (ROPE ? 16 : 64) * i);
        }
    };
    auto gather_v = [&](const Where &x, int st, uint4 (&row)[8]) {
        const bf16_t *cent = vs.cent + x.page * S * a.K * kHeadDim;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const uint4 o = *reinterpret_cast<const uint4 *>(offs + (S + st) * kTrTile + 16 * hf + 4 * kb);
            row[4 * hf + 0] = load16(cent, o.x + 16 * c);
            row[4 * hf + 1] = load16(cent, o.y + 16 * c);
            row[4 * hf + 2] = load16(cent, o.z + 16 * c);
            row[4 * hf + 3] = load16(cent, o.w + 16 * c);
        }
    };
    // the residual of tokens c and 16 + c as fragments 0..3 (in the order of Q's fragments 4..7)
    auto residual_k = [&](const Raw &f, int hf, int i, uint4 &out) {       // i: fragment
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
                r[e] = rd ? fma_half2(lv, s2, r[e]) : lv * s2;
            }
        }
        out = make_uint4(as_bits(r[0]), as_bits(r[1]), as_bits(r[2]), as_bits(r[3]));
    };
    // K_hat rotated, as fragments of the residual's order: the values meet in binary16 (rows of all stages in fp32 first)
    auto rotated_k = [&](const Where &x, int hf, const uint4 (&res)[4], const float (&cen)[32], uint4 (&out)[4]) {
        const int64_t at = min((int64_t)x.page_index * L + x.first + min(16 * hf + c, x.count - 1), t.rope_tokens - 1);
        const uint4 *rp = reinterpret_cast<const uint4 *>(static_cast<const f16_t *>(t.k_rope_f16) + at * kHeadDim + 32 * kb);
        float v[32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t rw[4] = {res[i].x, res[i].y, res[i].z, res[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int ca = I4 ? 8 * i + e : 16 * (i >> 1) + 7 - 4 * (i & 1) - e, cb = ca + (I4 ? 4 : 8);
                const halfx2_t r2 = as_half2(rw[e]);
                v[ca] = cen[ca] + (float)r2[0];
                v[cb] = cen[cb] + (float)r2[1];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) rotate_octet(v + 8 * i, rp[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t x4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int ca = I4 ? 8 * i + e : 16 * (i >> 1) + 7 - 4 * (i & 1) - e, cb = ca + (I4 ? 4 : 8);
                x4[e] = pack_f16x2_rne(v[ca], v[cb]);
            }
            out[i] = make_uint4(x4[0], x4[1], x4[2], x4[3]);
        }
    };
    auto scores_of_residual = [&](int i, const uint4 &r0, const uint4 &r1) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const halfx8_t q = __builtin_bit_cast(halfx8_t, qfrag(rb, 4 + i));
            Sc[rb][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8_t, r0), q, Sc[rb][0], 0, 0, 0);
            Sc[rb][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8_t, r1), q, Sc[rb][1], 0, 0, 0);
        }
    };
    // O^T += R^T P (kSplitV), or (C + R)^T P with the sums of the rows in `start` ([channel][pair of tokens]), four channels of the
    // lane's octet at a time (registers are what the loop is short of)
    auto add_residual = [&](auto start) {
        const uint16_t *sp = scales + (TG + 8 * c * G / kHeadDim) * kTrRowPitch + 4 * kb;
        uint2 s4[T][2], w2[I4 ? 1 : T][2];
        uint4 w4[I4 ? T : 1][2];
#pragma unroll
        for (int rd = 0; rd < T; ++rd)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                s4[rd][hf] = *reinterpret_cast<const uint2 *>(sp + rd * G * kTrRowPitch + 16 * hf);
                const int at = (rd * 16 + c) * kTrRowPitch + 16 * hf + 4 * kb;
                if (I4) w4[I4 ? rd : 0][hf] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint32_t *>(vcodes) + at);
                else w2[I4 ? 0 : rd][hf] = *reinterpret_cast<const uint2 *>(vcodes + at);
            }
#pragma unroll
        for (int half = 0; half < 2; ++half) {                           // channels 4 half .. 4 half + 3
            uint32_t r[4][4];                                            // [channel][pair of tokens]
#pragma unroll
            for (int rd = 0; rd < T; ++rd)
#pragma unroll
                for (int pr = 0; pr < 4; ++pr) {
                    const uint2 &sv = s4[rd][pr >> 1];
                    const halfx2_t s2 = as_half2(pr & 1 ? sv.y : sv.x);
                    uint32_t x;
                    if (I4) {
                        const uint4 &wv = w4[I4 ? rd : 0][pr >> 1];
                        x = __builtin_amdgcn_perm(pr & 1 ? wv.w : wv.y, pr & 1 ? wv.z : wv.x, half ? 0x07060302u : 0x05040100u) ^ 0x88888888u;
                    } else {
                        const uint2 &wv = w2[I4 ? 0 : rd][pr >> 1];
                        x = pr & 1 ? wv.y : wv.x;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const halfx2_t lv = I4 ? level4(x, e) : level2(x, 7 - (4 * half + e));
                        r[e][pr] = as_bits(rd ? fma_half2(lv, s2, as_half2(r[e][pr])) : kSplitV ? lv * s2 : fma_half2(lv, s2, start(4 * half + e, pr)));
                    }
                }
#pragma unroll
            for (int e = 0; e < 4; ++e) add_pv(4 * half + e, r[e]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // the centroids' scores: q . c of every row of the page's tables, 16 rows to a contraction
    auto build_table = [&](int64_t page) {
        const bf16_t *cent = ks.cent + page * S * a.K * kHeadDim;
        const int n = S * a.K;
        for (int r0 = wave * 16; r0 < n; r0 += kTrWaves * 16) {
            const uint32_t off = (uint32_t)min(r0 + c, n - 1) * (kHeadDim * 2) + 16 * kb;
            uint4 row[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) row[i] = load16(cent, off + 64 * i);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                floatx4_t x = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, row[i]), __builtin_bit_cast(bf16x8_t, qfrag(rb, i)), x, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) table[(r0 + 4 * kb + r) * kRows + rb * 16 + c] = x[r];
            }
        }
    };
    auto scores_of_ids = [&]() {
#pragma unroll
        for (int st = 0; st < S; ++st)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint4 o = *reinterpret_cast<const uint4 *>(offs + st * kTrTile + 16 * hf + 4 * kb);
                const uint32_t at[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = *reinterpret_cast<const float *>(reinterpret_cast<const unsigned char *>(table) + at[r] + (rb * 16 + c) * 4);
                        Sc[rb][hf][r] = st ? Sc[rb][hf][r] + x : x;
                    }
            }
    };

    const int stop = min(hi, sq.kv_tiles);
    if (lo < stop) {                                                     // uniform over the workgroup
        int ti = lo + wave, pi = ti / sq.per_page, in_page = ti - pi * sq.per_page;
        Where cur{-1, 0, 0, 0, 0};
        Raw f;
        if (ti < stop) {
            cur = place(pi, in_page, cur);
            fetch(cur, f);
        }
        // page by page; a wavefront without tiles in a page still helps with its table
        Where held{-1, 0, 0, 0, 0};
        for (int pg = lo / sq.per_page; pg * sq.per_page < stop; ++pg) {
            if (kTable) {
                held = place(pg, 0, held);
                __syncthreads();
                build_table(held.page);
                __syncthreads();
            }
            const int page_end = min(stop, (pg + 1) * sq.per_page);
            while (ti < page_end) {
            park(f);
            order_lds();
            uint4 krow[2][4], vrow[8];
            if (!kTable) gather_k(cur, 0, krow);
            const bool more = ti + kTrWaves < stop;                      // uniform
            Where nxt = cur;
            if (more) {
                in_page += kTrWaves;
                while (in_page >= sq.per_page) { in_page -= sq.per_page; ++pi; }
                nxt = place(pi, in_page, cur);
            }
            // The load counter is in order: the rows that this tile still needs are asked for before the next tile's data, which
            // then has the rest of the tile to arrive
            auto ahead = [&]() {
                gather_v(cur, 0, vrow);
                if (more) fetch(nxt, f);
            };
            if (kTable) scores_of_ids(); else clear_scores();
            if (ROPE) {
                uint4 res[2][4];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                    for (int i = 0; i < 4; ++i) residual_k(f, hf, i, res[hf][i]);
                if (S == 1) ahead();
                float cen[2][32];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                    for (int i = 0; i < 4; ++i) unpack_bf16x8(krow[hf][i], cen[hf] + 8 * i);
                for (int st = 1; st < S; ++st) {
                    gather_k(cur, st, krow);
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float x[8];
                            unpack_bf16x8(krow[hf][i], x);
#pragma unroll
                            for (int e = 0; e < 8; ++e) cen[hf][8 * i + e] += x[e];
                        }
                }
                uint4 rot[2][4];
                if (S > 1) ahead();
                rotated_k(cur, 0, res[0], cen[0], rot[0]);
                rotated_k(cur, 1, res[1], cen[1], rot[1]);
#pragma unroll
                for (int i = 0; i < 4; ++i) scores_of_residual(i, rot[0][i], rot[1][i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint4 r0, r1;
                    residual_k(f, 0, i, r0);
                    residual_k(f, 1, i, r1);
                    scores_of_residual(i, r0, r1);
                }
                if (!kTable) {
                    scores_of_rows(krow);
                    for (int st = 1; st < S; ++st) {
                        gather_k(cur, st, krow);
                        scores_of_rows(krow);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                ahead();
            }
            __builtin_amdgcn_sched_barrier(0);
            if (cur.count < kTrTile) {                                   // uniform: the page's last tile
                uint32_t see[RB];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) see[rb] = (1u << cur.count) - 1u;
                hide(see);
            }
            weights();
            __builtin_amdgcn_sched_barrier(0);
            if (kSplitV) {
                add_residual([&](int, int) { return halfx2_t{}; });
                __builtin_amdgcn_sched_barrier(0);
                add_rows(vrow);
                for (int st = 1; st < S; ++st) {
                    gather_v(cur, st, vrow);
                    add_rows(vrow);
                }
            } else if (S == 1) {
                add_residual([&](int j, int pr) { return pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j); });
            } else {
                halfx2_t sum[8][4];
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int pr = 0; pr < 4; ++pr) sum[j][pr] = pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j);
                for (int st = 1; st < S; ++st) {
                    gather_v(cur, st, vrow);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int pr = 0; pr < 4; ++pr) sum[j][pr] += pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j);
                }
                add_residual([&](int j, int pr) { return sum[j][pr]; });
            }
            order_lds();
            ti += kTrWaves;
            cur = nxt;
            }
        }
    }

    // ---- the tail's and the new tokens' tiles ---------------------------------------------------
    for (int ti = max(lo, sq.kv_tiles) + wave; ti < hi; ti += kTrWaves) {
        const bool fresh = ti >= sq.kv_tiles + sq.tail_tiles;
        const int first = (ti - sq.kv_tiles - (fresh ? sq.tail_tiles : 0)) * kTrTile;
        const int count = min(kTrTile, (fresh ? sq.nodes : sq.tail) - first);
        const uint32_t there = count >= 32 ? 0xffffffffu : (1u << count) - 1u;
        uint32_t see[RB], any = there;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) see[rb] = node[rb] >= 0 ? there : 0u;
        if (fresh) {
            any = 0u;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                if (node[rb] >= 0) {
                    if (t.mask) see[rb] &= t.mask[((int64_t)b * t.n_nodes + node[rb]) * ((t.n_nodes + 31) / 32) + first / 32];
                    else {
                        const int left = node[rb] - first;                 // sees tokens first .. first + left
                        see[rb] &= left < 0 ? 0u : (left >= 31 ? 0xffffffffu : (2u << left) - 1u);
                    }
                }
                any |= see[rb];
            }
#pragma unroll
            for (int off = 1; off < 16; off *= 2) any |= __shfl_xor(any, off, 64);
        }
        const int64_t stride = fresh ? t.new_stride_node : t.tail_stride_token;
        const int64_t off = fresh ? b * t.new_stride_seq + h * t.new_stride_head + first * stride
                                  : b * t.tail_stride_seq + h * t.tail_stride_head + first * stride;
        const bf16_t *kr = static_cast<const bf16_t *>(fresh ? t.k_new : t.k_tail) + off + 8 * kb;
        const bf16_t *vr = static_cast<const bf16_t *>(fresh ? t.v_new : t.v_tail) + off + 8 * c;
        uint4 krow[2][4], vrow[8];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                krow[hf][i] = *reinterpret_cast<const uint4 *>(kr + min(16 * hf + c, count - 1) * stride + 32 * i);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            vrow[e] = *reinterpret_cast<const uint4 *>(vr + min(16 * (e >> 2) + 4 * kb + (e & 3), count - 1) * stride);
        clear_scores();
        scores_of_rows(krow);
        hide(see);
        weights();
        // (a new token that no row sees may be no number)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!((any >> (16 * (e >> 2) + 4 * kb + (e & 3))) & 1u)) vrow[e] = make_uint4(0u, 0u, 0u, 0u);
        add_rows(vrow);
    }
    __syncthreads();                                                     // (the meeting place lies over the wavefronts' own LDS)
    finish_block<RB>(a, b, h, bh, rblk, part, sq.nodes, reinterpret_cast<float (*)[16][kTrPitch]>(smem), ms, ls, O, m, l);
}

// Joins a query row's parts: a workgroup to a row, 16 lanes (8 channels each) to a part, so that 16 parts are read at a time.
__global__ __launch_bounds__(256)
void tree_join_kernel(TreeArgs a, int block_rows) {
    __shared__ float sums[16][kTrPitch], weights[16];
    const int64_t rows = (int64_t)a.t.group * a.t.n_nodes;
    const int64_t bh = (int64_t)(blockIdx.x / (unsigned)rows), r = (int64_t)blockIdx.x - bh * rows;
    const int b = (int)(bh / a.H), h = (int)(bh - (int64_t)b * a.H);
    const int64_t block = bh * a.row_blocks + r / block_rows;
    const int row = (int)(r % block_rows), grp = threadIdx.x >> 4, c8 = threadIdx.x & 15;
    const int step = (int)tree_state_floats(block_rows);
    const float *st = a.state + block * a.parts * step;
    const float *mp = st + block_rows * kHeadDim + row, *lp = mp + block_rows, *op = st + row * kHeadDim + c8 * 8;
    float m = kTrNoScore, l = 0.0f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
    // every lane finds the maximum over all parts: lane i of 64 looks at parts i, i + 64, ..
    for (int p = threadIdx.x & 63; p < a.parts; p += 64) m = fmaxf(m, mp[(int64_t)p * step]);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
#pragma unroll 4
    for (int p = grp; p < a.parts; p += 16) {
        const float f = __builtin_amdgcn_exp2f(mp[(int64_t)p * step] - m);
        const float4 x = *reinterpret_cast<const float4 *>(op + (int64_t)p * step), y = *reinterpret_cast<const float4 *>(op + (int64_t)p * step + 4);
        l += lp[(int64_t)p * step] * f;
        o[0] += x.x * f; o[1] += x.y * f; o[2] += x.z * f; o[3] += x.w * f;
        o[4] += y.x * f; o[5] += y.y * f; o[6] += y.z * f; o[7] += y.w * f;
    }
    *reinterpret_cast<float4 *>(&sums[grp][c8 * 8]) = make_float4(o[0], o[1], o[2], o[3]);
    *reinterpret_cast<float4 *>(&sums[grp][c8 * 8 + 4]) = make_float4(o[4], o[5], o[6], o[7]);
    if (c8 == 0) weights[grp] = l;
    __syncthreads();
    if (grp) return;
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll
    for (int g = 0; g < 16; ++g) {
        l += weights[g];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += sums[g][c8 * 8 + e];
    }
    int nodes = a.t.n_nodes;
    if (a.t.nodes) { nodes = a.t.nodes[b]; nodes = nodes < 0 ? 0 : (nodes > a.t.n_nodes ? a.t.n_nodes : nodes); }
    store_row8(a, b, h, r, nodes, c8, o, m, l);
}

TreePlan tree_plan(int H, const qvg_tree_step &t) {
    TreePlan p{1, 1, 0};
    const int64_t rows = (int64_t)t.group * t.n_nodes;
    const int br = tree_block_rows(rows);
    p.row_blocks = (int)((rows + br - 1) / br);
    const int64_t units = (int64_t)t.n_seqs * H * p.row_blocks;
    if (units < 1) return p;
    const int64_t tiles = t.table_pages * ((t.page_len + kTrTile - 1) / kTrTile) + (t.tail_capacity + kTrTile - 1) / kTrTile +
                          (t.n_nodes + kTrTile - 1) / kTrTile;
    // as many workgroups as the chip holds at once (two to a CU, three with blocks of 16 rows), two tiles to a wavefront at least
    int64_t parts = 512 / units;
    const int64_t most = tiles / (2 * kTrWaves);
    if (parts > most) parts = most;
    if (parts > 1) {
        p.parts = (int)parts;
        p.state_bytes = (size_t)units * parts * tree_state_floats(br) * sizeof(float);
    }
    return p;
}

template <int FMT, int RB>
static void launch_rb(const TreeArgs &a, int blocks, hipStream_t s) {
    const int per_xcd = (blocks + 7) / 8;
    tree_attn_kernel<FMT, RB><<<dim3((unsigned)(per_xcd * 8)), dim3(kTrThreads), 0, s>>>(a, blocks, per_xcd);
}
template <int FMT>
static void launch_fmt(const TreeArgs &a, int blocks, int block_rows, hipStream_t s) {
    if (block_rows == 16) launch_rb<FMT, 1>(a, blocks, s);
    else launch_rb<FMT, 2>(a, blocks, s);
}
template <class F, bool ROPE, int RB>
static hipError_t launch_packed_rb(const TreeArgs &a, int blocks, hipStream_t s) {
    const int per_xcd = (blocks + 7) / 8;
    constexpr bool table = !ROPE && (F::S == 1 || RB == 1);               // (as in the kernel)
    constexpr int own = tree_query_bytes<RB>() + kTrWaves * F::wave_bytes;
    int lds = own + (table ? (F::S * a.K + 15) / 16 * 16 * 16 * RB * 4 : 0);
    if (lds < kTrMeetBytes) lds = kTrMeetBytes;
    if (lds > 64 * 1024) {
        static LdsHighWater mark;
        const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(tree_attn_packed<F, ROPE, RB>), (size_t)lds, mark);
        if (e != hipSuccess) return e;
    }
    tree_attn_packed<F, ROPE, RB><<<dim3((unsigned)(per_xcd * 8)), dim3(kTrThreads), (size_t)lds, s>>>(a, blocks, per_xcd);
    return hipSuccess;
}
template <int T, int G, bool FP8, bool I4, int S>
static bool launch_packed(const TreeArgs &a, int blocks, int br, hipStream_t s, hipError_t &e) {
    if (a.T != T || kHeadDim / a.B != G || a.S != S || a.fmt != ((FP8 ? kFmtE4M3 : 0) | (I4 ? kFmtInt4 : 0))) return false;
    typedef TreeFormat<T, G, FP8, I4, S> F;
    if (a.t.k_rope_f16)
        e = br == 16 ? launch_packed_rb<F, true, 1>(a, blocks, s) : launch_packed_rb<F, true, 2>(a, blocks, s);
    else
        e = br == 16 ? launch_packed_rb<F, false, 1>(a, blocks, s) : launch_packed_rb<F, false, 2>(a, blocks, s);
    return true;
}
hipError_t launch_attn_tree(const TreeArgs &a, hipStream_t s) {
    const int br = tree_block_rows((int64_t)a.t.group * a.t.n_nodes);
    const int64_t units = (int64_t)a.t.n_seqs * a.H * a.row_blocks;
    const int blocks = (int)(units * a.parts);
    // The packed form is built for the formats of the package's configurations and of the paper's presets, and their
    // neighbours in group size; any other one is decoded element by element.
    hipError_t e = hipSuccess;
    const bool packed = launch_packed<1, 2, true, false, 1>(a, blocks, br, s, e) || launch_packed<1, 8, true, false, 1>(a, blocks, br, s, e) ||
                        launch_packed<1, 8, true, false, 4>(a, blocks, br, s, e) || launch_packed<1, 2, true, true, 1>(a, blocks, br, s, e) ||
                        launch_packed<1, 8, true, true, 4>(a, blocks, br, s, e) || launch_packed<1, 2, false, false, 1>(a, blocks, br, s, e) ||
                        launch_packed<2, 2, false, false, 1>(a, blocks, br, s, e) || launch_packed<2, 4, false, false, 1>(a, blocks, br, s, e) ||
                        launch_packed<3, 2, false, false, 1>(a, blocks, br, s, e) || launch_packed<3, 4, false, false, 1>(a, blocks, br, s, e) ||
                        launch_packed<4, 2, false, false, 1>(a, blocks, br, s, e) || launch_packed<4, 4, false, false, 1>(a, blocks, br, s, e);
    if (e != hipSuccess) return e;
    if (!packed) switch (a.fmt) {
        case 0: launch_fmt<0>(a, blocks, br, s); break;
        case kFmtE4M3: launch_fmt<kFmtE4M3>(a, blocks, br, s); break;
        case kFmtInt4: launch_fmt<kFmtInt4>(a, blocks, br, s); break;
        default: launch_fmt<kFmtE4M3 | kFmtInt4>(a, blocks, br, s); break;
    }
    if (a.parts > 1) {
        const int64_t n = (int64_t)a.t.n_seqs * a.H * a.t.group * a.t.n_nodes;
        tree_join_kernel<<<dim3((unsigned)n), dim3(256), 0, s>>>(a, br);
    }
    return hipGetLastError();
}

}  // namespace qvg
