// Attention of the few new tokens of a step (one token, or a tree of drafted ones) over a sequence's compressed pages, its
// bf16 tail and the new tokens themselves:
//     o = sum_n w_n v_n / sum_n w_n,   w_n = exp(scale q.k_n),   k_n, v_n = sum_s c_s[id_s(n)] + sum_t s_t(n) q_t(n)  (Eq. 7)
// in one pass over the tokens with the running maximum and sum of the soft-max.
//
// A workgroup takes a block of 16 or 32 query rows of one KV head (rows = group x new tokens; 64 or 128 in qvg_tree_wide.hip)
// and a part of the sequence's tiles of 32 tokens; each of its wavefronts walks tiles of its own, so a tile costs no barrier.
// The contractions run on v_mfma_f32_16x16x32_f16 with the operands where the decoding puts them, so a decoded tile passes
// through registers only:
//   S^T = K Q^T:   lane (c, kb) decodes channels 32 kb .. 32 kb + 31 of tokens c and 16 + c; the order of a contraction is
//                  free, so MFMA i takes channels 32 kb + 8 i + e and Q's fragments are loaded the same way;
//   O^T += V^T P:  lane (c, kb) decodes the octet of channels 8 c .. 8 c + 7 of tokens 4 kb + r and 16 + 4 kb + r, which are
//                  the tokens whose scores S^T leaves in the lane: P needs no movement, and pairs of tokens are packed as
//                  they are rounded, which is the transposition.  MFMA j makes channels 8 c + j; the lane ends up with
//                  channels 32 kb .. 32 kb + 31 of query row c.
// Tokens that are not there, and new ones that a row does not see, get the score -inf; the row's reference is finite from the
// start, so their weights are zero whatever comes first.
//
// The kernel here decodes a tile element by element with the format's sizes at run time: any format that the encoder
// writes.  Its vector instructions bound it: five to ten times the packed form's time (qvg_tree.hpp).  The formats of the package's
// configurations and presets have qvg_tree_packed.hip and qvg_tree_wide.hip.
#include "qvg_tree_lane.hpp"

namespace qvg {

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

template <int FMT, int RB>
__global__ __launch_bounds__(kTrThreads, 2)
void tree_attn_kernel(TreeArgs a, int blocks, int per_xcd) {
    constexpr int kRows = 16 * RB;
    __shared__ float meet[kTrWaves][16][kTrPitch];
    __shared__ float ms[kTrWaves][kRows], ls[kTrWaves][kRows];
    // workgroups are dealt to the 8 XCDs round-robin: the parts of one KV head run on one, whose L2 then keeps its tables
    const int w = (int)(blockIdx.x % 8u) * per_xcd + (int)(blockIdx.x / 8u);
    if (w >= blocks) return;                                             // uniform, before any barrier
    const BlockPlace at = place_block(a, w, a.t.k_rope_f16 != nullptr, kRows);
    if (at.parts == 0) return;                                           // uniform, before any barrier
    const int b = at.b, h = at.h, rblk = at.rblk;
    const qvg_tree_step &t = a.t;
    const SeqTiles sq = tiles_of_sequence(t, b);
    const PartTiles pt = tiles_of_part(a, sq, at.part, at.parts);
    const int hi = pt.hi;
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

    for (int ti = pt.first + wave; ti < hi; ti += pt.step) {
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
            for (int rb = 0; rb < RB; ++rb) any |= see[rb] = node_sees(t, b, node[rb], first, there);
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
            if (__ballot(top - m[rb] > kTrBelow + kTrLag)) {            // uniform: some row's reference moves
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

    finish_block<RB>(a, at, sq.nodes, meet, ms, ls, O, m, l);
}

// Joins a query row's parts: a workgroup to a row, 16 lanes (8 channels each) to a part, so that GROUPS parts are read at a time.
// One wavefront to a row where there are many rows of few parts: shuffles alone, and all rows at once.
template <int GROUPS>
__global__ __launch_bounds__(16 * GROUPS)
void tree_join_kernel(TreeArgs a, int block_rows) {
    const int64_t rows = (int64_t)a.t.group * a.t.n_nodes;
    const int64_t bh = (int64_t)(blockIdx.x / (unsigned)rows), r = (int64_t)blockIdx.x - bh * rows;
    const int b = (int)(bh / a.H), h = (int)(bh - (int64_t)b * a.H);
    const int row = (int)(r % block_rows), grp = threadIdx.x >> 4, c8 = threadIdx.x & 15;
    const int step = (int)tree_state_floats(block_rows);
    const int2 place = a.places[b];                                      // first slot, parts
    int nodes = a.t.n_nodes;
    if (a.t.nodes) { nodes = a.t.nodes[b]; nodes = nodes < 0 ? 0 : (nodes > a.t.n_nodes ? a.t.n_nodes : nodes); }
    const float *st = a.state + (((int64_t)h * a.row_blocks + r / block_rows) * a.slots + place.x) * step;
    const float *mp = st + block_rows * kHeadDim + row, *lp = mp + block_rows, *op = st + row * kHeadDim + c8 * 8;
    float m = kTrNoScore, l = 0.0f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
    // every lane finds the maximum over all parts: lane i of 64 looks at parts i, i + 64, ..
    for (int p = threadIdx.x & 63; p < place.y; p += 64) m = fmaxf(m, mp[(int64_t)p * step]);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
#pragma unroll 4
    for (int p = grp; p < place.y; p += GROUPS) {
        const float f = __builtin_amdgcn_exp2f(mp[(int64_t)p * step] - m);
        const float4 x = *reinterpret_cast<const float4 *>(op + (int64_t)p * step);
        const float4 y = *reinterpret_cast<const float4 *>(op + (int64_t)p * step + 4);
        l += lp[(int64_t)p * step] * f;
        o[0] += x.x * f; o[1] += x.y * f; o[2] += x.z * f; o[3] += x.w * f;
        o[4] += y.x * f; o[5] += y.y * f; o[6] += y.z * f; o[7] += y.w * f;
    }
    // the four parts of a wavefront, then the wavefronts
#pragma unroll
    for (int off = 16; off < 64; off *= 2) {
        l += __shfl_xor(l, off, 64);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += __shfl_xor(o[e], off, 64);
    }
    if constexpr (GROUPS > 4) {
        constexpr int W = GROUPS / 4;
        __shared__ float sums[W][kTrPitch], weights[W];
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) < 16) {
            *reinterpret_cast<float4 *>(&sums[wave][c8 * 8]) = make_float4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<float4 *>(&sums[wave][c8 * 8 + 4]) = make_float4(o[4], o[5], o[6], o[7]);
            if (c8 == 0) weights[wave] = l;
        }
        __syncthreads();
        l = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll
        for (int g = 0; g < W; ++g) {
            l += weights[g];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += sums[g][c8 * 8 + e];
        }
    }
    if (grp == 0) store_row8(a, b, h, r, nodes, c8, o, m, l);
}

static bool packed_format(const qvg_params &p) {
    return tree_packed(p.n_stages, kHeadDim / p.group_size, (p.bits == 4 ? kFmtInt4 : 0) | (p.scale_format == QVG_SCALE_E4M3 ? kFmtE4M3 : 0),
                       p.n_smooth_stages);
}
TreePlan tree_plan(const qvg_params &prm, const qvg_tree_step &t, bool rotated) {
    TreePlan p{16, 1, 0, 1, 0};
    const int64_t rows = (int64_t)t.group * t.n_nodes;
    const int br = p.rows = tree_block_rows(rows, packed_format(prm), rotated);
    p.row_blocks = (int)((rows + br - 1) / br);
    const int64_t units = (int64_t)prm.n_heads * p.row_blocks;           // of a sequence
    if (t.n_seqs < 1 || rows < 1) return p;
    const int64_t tiles = (int64_t)t.table_pages * tree_tiles((int)t.page_len) + tree_tiles(t.tail_capacity) + tree_tiles(t.n_nodes);
    // As many workgroups as the chip holds at once (two to a CU), two tiles to a wavefront at least; not divided where that is
    // less than two workgroups to a sequence
    int64_t slots = 512 / units;
    const int64_t most = t.n_seqs * (tiles / (2 * kTrWaves));
    if (slots > most) slots = most;
    if (slots >= 2 * (int64_t)t.n_seqs) {
        p.slots = (int)slots;
        p.state_bytes = (size_t)(units * slots * tree_state_floats(br)) * sizeof(float) + (size_t)t.n_seqs * sizeof(int2);
        // Several smoothing stages' rows gathered for both sides (with a rotation, or beyond 16 rows) are more than an XCD's L2
        // holds for 64 workgroups in pages of their own: 12 heads x 187200 tokens, four stages, 736 -> 560 us rotated, 32 rows
        // 528 -> 435 us.  Elsewhere sharing costs more tables than it saves (one token, one round: 92 -> 114 us).
        if (prm.n_smooth_stages > 1 && (rotated || rows > 16)) p.share = 8;
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
hipError_t launch_attn_tree(const TreeArgs &a, hipStream_t s) {
    const bool packed = tree_packed(a.T, kHeadDim / a.B, a.fmt, a.S);
    const int br = a.rows;
    const int blocks = (int)((int64_t)(a.slots ? a.slots : a.t.n_seqs) * a.H * a.row_blocks);
    hipError_t e = hipSuccess;
    if (packed) e = br > 32 ? launch_tree_wide(a, blocks, br, s) : launch_tree_packed(a, blocks, br, s);
    else switch (a.fmt) {
        case 0: launch_fmt<0>(a, blocks, br, s); break;
        case kFmtE4M3: launch_fmt<kFmtE4M3>(a, blocks, br, s); break;
        case kFmtInt4: launch_fmt<kFmtInt4>(a, blocks, br, s); break;
        default: launch_fmt<kFmtE4M3 | kFmtInt4>(a, blocks, br, s); break;
    }
    if (e != hipSuccess) return e;
    if (a.slots) {
        const int64_t n = (int64_t)a.t.n_seqs * a.H * a.t.group * a.t.n_nodes;
        // (more rows than the chip holds workgroups of 256: 4960 rows of 13 parts 9.0 us so and 13.8; 12 of 42 parts 7.9 and 7.1)
        if (n > 2048) tree_join_kernel<4><<<dim3((unsigned)n), dim3(64), 0, s>>>(a, br);
        else tree_join_kernel<16><<<dim3((unsigned)n), dim3(256), 0, s>>>(a, br);
    }
    return hipGetLastError();
}

}  // namespace qvg
