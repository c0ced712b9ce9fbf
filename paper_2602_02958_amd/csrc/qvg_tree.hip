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

    // ---- the wavefronts' results meet ---------------------------------------------------------
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
        } else if (r < rows) store_row8(a, b, h, r, sq.nodes, c8, o, mt, lt);
        if (rb + 1 < RB) __syncthreads();
    }
}

// Joins the parts of a block: 16 lanes to a row, 8 channels each.
__global__ __launch_bounds__(256)
void tree_join_kernel(TreeArgs a, int block_rows) {
    const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);      // block row
    const int c8 = threadIdx.x & 15;
    const int64_t total = (int64_t)a.t.n_seqs * a.H * a.row_blocks * block_rows;
    if (i >= total) return;
    const int64_t block = i / block_rows;
    const int row = (int)(i - block * block_rows);
    const int64_t bh = block / a.row_blocks;
    const int b = (int)(bh / a.H), h = (int)(bh - (int64_t)b * a.H);
    const int64_t r = (block - bh * a.row_blocks) * block_rows + row;
    if (r >= (int64_t)a.t.group * a.t.n_nodes) return;
    const float *st = a.state + block * a.parts * tree_state_floats(block_rows);
    const float *mp = st + block_rows * kHeadDim + row, *lp = mp + block_rows;
    const int64_t step = tree_state_floats(block_rows);
    float m = kTrNoScore, l = 0.0f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
    for (int p = 0; p < a.parts; ++p) m = fmaxf(m, mp[p * step]);
    for (int p = 0; p < a.parts; ++p) {
        const float f = __builtin_amdgcn_exp2f(mp[p * step] - m);
        const float *op = st + p * step + row * kHeadDim + c8 * 8;
        const float4 x = *reinterpret_cast<const float4 *>(op), y = *reinterpret_cast<const float4 *>(op + 4);
        l += lp[p * step] * f;
        o[0] += x.x * f; o[1] += x.y * f; o[2] += x.z * f; o[3] += x.w * f;
        o[4] += y.x * f; o[5] += y.y * f; o[6] += y.z * f; o[7] += y.w * f;
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
    // about a thousand workgroups (four to a CU), two tiles to a wavefront at least
    int64_t parts = (1024 + units - 1) / units;
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
    else if (block_rows == 32) launch_rb<FMT, 2>(a, blocks, s);
    else launch_rb<FMT, 4>(a, blocks, s);
}
hipError_t launch_attn_tree(const TreeArgs &a, hipStream_t s) {
    const int br = tree_block_rows((int64_t)a.t.group * a.t.n_nodes);
    const int64_t units = (int64_t)a.t.n_seqs * a.H * a.row_blocks;
    const int blocks = (int)(units * a.parts);
    switch (a.fmt) {
        case 0: launch_fmt<0>(a, blocks, br, s); break;
        case kFmtE4M3: launch_fmt<kFmtE4M3>(a, blocks, br, s); break;
        case kFmtInt4: launch_fmt<kFmtInt4>(a, blocks, br, s); break;
        default: launch_fmt<kFmtE4M3 | kFmtInt4>(a, blocks, br, s); break;
    }
    if (a.parts > 1) {
        const int64_t n = units * br;
        tree_join_kernel<<<dim3((unsigned)((n + 15) / 16)), dim3(256), 0, s>>>(a, br);
    }
    return hipGetLastError();
}

}  // namespace qvg
