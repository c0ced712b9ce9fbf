// Attention over a paged cache for more than 64 query rows of a KV head (32 where keys are rotated): the wavefronts of a workgroup
// share what they decode.
//
// A workgroup takes 64 or 128 rows, RS wavefronts of 32 rows each, and walks its tiles in rounds of four: every wavefront decodes
// one of them into the fragments of both contractions (8 KB each, K_hat and V_hat as binary16) in LDS, and then contracts
// its rows with the fragments of all four tiles (RS = 4), or of two while another wavefront has the same rows and the other two
// (RS = 2).  Decoding costs about 300 vector instructions a side, whatever the number of rows; a wavefront that decodes for 32
// rows alone does it four times for 128.  While one workgroup of a CU decodes, the other contracts.
// Between the barriers the V codes, scales and ids of the tile that is decoded lie where its V fragments will.
// What bounds it: two workgroups of 64 KB to a CU, two wavefronts to a SIMD, which do not hide all waits (two rounds over 12 heads x
// 187200 tokens: with 128 rows vector instructions 48 % of the SIMDs' time and the matrix pipe 19 %, with 64 rotated rows 42 and 8 %).
// 128 rows take 258 us in one round and 312 in two, rotated 439 in two; 64 rotated rows 281 and 360.
#include "qvg_tree_lane.hpp"

namespace qvg {

constexpr int kTwFragBytes = 16 * 64 * 16;          // of a tile: 8 fragments of K, 8 of V
constexpr int kTwSmem = kTrWaves * kTwFragBytes;

template <class F, bool ROPE, int RS>
__global__ __launch_bounds__(kTrThreads, 2)
void tree_attn_wide(TreeArgs a, int blocks, int per_xcd) {
    constexpr int S = F::S, RB = 2, kRows = 32 * RS, TS = kTrWaves / RS;
    static_assert(F::wave_bytes <= kTwFragBytes / 2, "a tile's staging must fit the place of its V fragments");
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float ms[kTrWaves][32], ls[kTrWaves][32];
    __shared__ int tile_first[kTrWaves], tile_count[kTrWaves];           // first: of a tile of new tokens, else -1
    const int w = (int)(blockIdx.x % 8u) * per_xcd + (int)(blockIdx.x / 8u);
    if (w >= blocks) return;                                             // uniform, before any barrier
    const BlockPlace at = place_block(a, w, ROPE, kRows);
    if (at.parts == 0) return;                                           // uniform, before any barrier
    const int b = at.b, h = at.h, rblk = at.rblk;
    const qvg_tree_step &t = a.t;
    const SeqTiles sq = tiles_of_sequence(t, b);
    const PartTiles pt = tiles_of_part(a, sq, at.part, at.parts);
    const int hi = pt.hi;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, kb = lane >> 4, rs = wave % RS, ts = wave / RS;
    const int64_t row0 = (int64_t)rblk * kRows;
    uint4 *frags = reinterpret_cast<uint4 *>(smem);                      // [wavefront][K: half * 4 + i, V: 8 + channel][64]
    uint4 *mine = frags + wave * 16 * 64 + lane;

    TreeRows<RB> R;
    uint4 q[RB][4];
    int node[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float v[32];
        const QueryRow row(a, sq, b, h, row0 + rs * 32 + rb * 16 + c, v);
        node[rb] = row.node; R.qs[rb] = row.scale(a);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __builtin_amdgcn_ldexpf(v[i], 9 - row.ex);
#pragma unroll
        for (int i = 0; i < 4; ++i) q[rb][i] = QueryRow::residual_fragment<F>(v, i);
    }
    R.clear();

    typedef TreeLane<F> Lane;
    const Lane D(a, sq, b, h, smem + wave * kTwFragBytes + kTwFragBytes / 2);
    typename Lane::Where cur{-1, 0, 0, 0, 0};
    typename Lane::Raw f;
    const int stop = min(hi, sq.kv_tiles);
    int pi = (pt.first + wave) / sq.per_page, in_page = pt.first + wave - pi * sq.per_page;
    if (pt.first + wave < stop) {
        cur = D.place(pi, in_page, cur);
        D.fetch(cur, f);
    }
    // pairs of channels of bf16 rows (in the residual's order), as binary16
    auto row_pairs = [&](const uint4 (&row)[4], int i, halfx2_t (&x)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int ca = Lane::channel(i, e), cb = ca + Lane::pair_step;
            const uint32_t wa = D.word_of(row[ca >> 3], ca & 7), wb = D.word_of(row[cb >> 3], cb & 7);
            x[e] = as_half2(pack_f16x2_rne(ca & 1 ? bf16_hi(wa) : bf16_lo(wa), cb & 1 ? bf16_hi(wb) : bf16_lo(wb)));
        }
    };

    for (int r0 = pt.first; r0 < hi; r0 += pt.step) {
        // ---- decode: the wavefront's tile -------------------------------------------------------
        const int ti = r0 + wave;
        if (ti < stop) {
            D.park(f, kHeadDim * 2);
            D.order_lds();
            uint4 vrow[8];
            const bool more = ti + pt.step < stop;                      // uniform
            typename Lane::Where nxt = cur;
            if (more) {
                in_page += pt.step;
                while (in_page >= sq.per_page) { in_page -= sq.per_page; ++pi; }
                nxt = D.place(pi, in_page, cur);
            }
            if (ROPE || S > 1) {                                         // rows and residual meet in fp32
                uint4 row[S][4], rp[2][4];
                D.gather_half(cur, 0, row);
                if (ROPE) { D.gather_rope(cur, 0, rp[0]); D.gather_rope(cur, 1, rp[1]); }
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    float v[32];
                    uint4 out[4];
                    D.sum_rows(row, v);
                    if (hf == 0) D.gather_half(cur, 1, row);
                    else D.gather_v(cur, 0, vrow);
                    D.template whole_k<ROPE>(f, hf, v, rp[hf], out);
#pragma unroll
                    for (int i = 0; i < 4; ++i) mine[(hf * 4 + i) * 64] = out[i];
                }
            } else {
                uint4 krow[2][4];
                D.template gather_k<true>(cur, 0, krow);
                D.gather_v(cur, 0, vrow);
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        halfx2_t x[4];
                        uint4 out;
                        row_pairs(krow[hf], i, x);
                        D.template residual_k<true>(f, hf, i, x, out);
                        mine[(hf * 4 + i) * 64] = out;
                    }
            }
            // (the loads that this tile still needs are asked for; the next tile's have the rest of the round to arrive)
            typename Lane::Levels lv;
            D.read_levels(lv);
            halfx2_t sum[S > 1 ? 8 : 1][4];
            if (S > 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int pr = 0; pr < 4; ++pr) sum[S > 1 ? j : 0][pr] = D.pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j);
                for (int st = 1; st < S; ++st) {
                    D.gather_v(cur, st, vrow);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int pr = 0; pr < 4; ++pr) sum[S > 1 ? j : 0][pr] += D.pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j);
                }
            }
            D.order_lds();                                               // (staging is read before the fragments go over it)
            if (more) D.fetch(nxt, f);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t r[4][4];
                if (S > 1) D.template values_v<true>(lv, half, [&](int j, int pr) { return sum[S > 1 ? j : 0][pr]; }, r);
                else D.template values_v<true>(lv, half, [&](int j, int pr) { return D.pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j); }, r);
#pragma unroll
                for (int e = 0; e < 4; ++e) mine[(8 + 4 * half + e) * 64] = make_uint4(r[e][0], r[e][1], r[e][2], r[e][3]);
            }
            if (lane == 0) { tile_first[wave] = -1; tile_count[wave] = cur.count; }
            cur = nxt;
        } else if (ti < hi) {
            const bool fresh = ti >= sq.kv_tiles + sq.tail_tiles;
            const int first = (ti - sq.kv_tiles - (fresh ? sq.tail_tiles : 0)) * kTrTile;
            const int count = min(kTrTile, (fresh ? sq.nodes : sq.tail) - first);
            const uint32_t there = count >= 32 ? 0xffffffffu : (1u << count) - 1u;
            uint32_t any = there;
            if (fresh) {                                                 // what any row of the block sees
                any = 0u;
                for (int i = lane; i < kRows; i += 64) {
                    const int64_t r = row0 + i;
                    if (r < (int64_t)t.group * t.n_nodes) {
                        const int nd = place_row(a, h, r).node;
                        any |= node_sees(t, b, nd < sq.nodes ? nd : -1, first, there);
                    }
                }
#pragma unroll
                for (int off = 1; off < 64; off *= 2) any |= __shfl_xor(any, off, 64);
            }
            const int64_t stride = fresh ? t.new_stride_node : t.tail_stride_token;
            const int64_t off = fresh ? b * t.new_stride_seq + h * t.new_stride_head + first * stride
                                      : b * t.tail_stride_seq + h * t.tail_stride_head + first * stride;
            const bf16_t *kr = static_cast<const bf16_t *>(fresh ? t.k_new : t.k_tail) + off + 32 * kb;
            const bf16_t *vr = static_cast<const bf16_t *>(fresh ? t.v_new : t.v_tail) + off + 8 * c;
            uint4 krow[2][4], vrow[8];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int i = 0; i < 4; ++i) krow[hf][i] = *reinterpret_cast<const uint4 *>(kr + min(16 * hf + c, count - 1) * stride + 8 * i);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                vrow[e] = *reinterpret_cast<const uint4 *>(vr + min(16 * (e >> 2) + 4 * kb + (e & 3), count - 1) * stride);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    halfx2_t x[4];
                    row_pairs(krow[hf], i, x);
                    mine[(hf * 4 + i) * 64] = make_uint4(as_bits(x[0]), as_bits(x[1]), as_bits(x[2]), as_bits(x[3]));
                }
            // (a new token that no row sees may be no number)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!((any >> (16 * (e >> 2) + 4 * kb + (e & 3))) & 1u)) vrow[e] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                mine[(8 + j) * 64] = make_uint4(as_bits(D.pair_f16(vrow[0], vrow[1], j)), as_bits(D.pair_f16(vrow[2], vrow[3], j)),
                                                as_bits(D.pair_f16(vrow[4], vrow[5], j)), as_bits(D.pair_f16(vrow[6], vrow[7], j)));
            if (lane == 0) { tile_first[wave] = fresh ? first : -1; tile_count[wave] = count; }
        }
        __syncthreads();
        // ---- contract: the wavefront's rows with its tiles of the round -----------------------------
#pragma unroll 1
        for (int k = ts * RS; k < ts * RS + RS && r0 + k < hi; ++k) {    // uniform
            const uint4 *fr = frags + k * 16 * 64 + lane;
            R.clear_scores();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const halfx8_t k0 = __builtin_bit_cast(halfx8_t, fr[i * 64]), k1 = __builtin_bit_cast(halfx8_t, fr[(4 + i) * 64]);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    R.s[rb][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, __builtin_bit_cast(halfx8_t, q[rb][i]), R.s[rb][0], 0, 0, 0);
                    R.s[rb][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, __builtin_bit_cast(halfx8_t, q[rb][i]), R.s[rb][1], 0, 0, 0);
                }
            }
            const int count = __builtin_amdgcn_readfirstlane(tile_count[k]), first = __builtin_amdgcn_readfirstlane(tile_first[k]);
            if (count < kTrTile || first >= 0) {                         // uniform
                const uint32_t there = count >= 32 ? 0xffffffffu : (1u << count) - 1u;
                uint32_t see[RB];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) see[rb] = first >= 0 ? node_sees(t, b, node[rb], first, there) : there;
                R.hide(see);
            }
            uint4 P[RB];
            R.weights([&](int rb, const float (&x)[8]) {
                P[rb] = make_uint4(pack_f16x2_rne(x[0], x[1]), pack_f16x2_rne(x[2], x[3]), pack_f16x2_rne(x[4], x[5]), pack_f16x2_rne(x[6], x[7]));
            });
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const halfx8_t v = __builtin_bit_cast(halfx8_t, fr[(8 + j) * 64]);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    R.o[rb][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, __builtin_bit_cast(halfx8_t, P[rb]), R.o[rb][j], 0, 0, 0);
            }
        }
        __syncthreads();
    }

    // ---- the wavefronts of the same rows meet (wavefronts rs, rs + RS, ..), 16 rows of each at a time -------
    float (*meet)[16][kTrPitch] = reinterpret_cast<float (*)[16][kTrPitch]>(smem);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        R.l[rb] += __shfl_xor(R.l[rb], 16, 64);
        R.l[rb] += __shfl_xor(R.l[rb], 32, 64);
        if (kb == 0) { ms[wave][rb * 16 + c] = R.m[rb]; ls[wave][rb * 16 + c] = R.l[rb]; }
    }
    __syncthreads();
    const int row = tid >> 4, c8 = tid & 15;
    const int64_t rows = (int64_t)t.group * t.n_nodes;
    float *st = a.state + at.state;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float mm = ms[rs][rb * 16 + c];
#pragma unroll
        for (int v = 1; v < TS; ++v) mm = fmaxf(mm, ms[rs + v * RS][rb * 16 + c]);
        const float f16 = __builtin_amdgcn_exp2f(R.m[rb] - mm);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < 8; j += 4)
                *reinterpret_cast<float4 *>(&meet[wave][c][32 * kb + 8 * r + j]) =
                    make_float4(R.o[rb][j][r] * f16, R.o[rb][j + 1][r] * f16, R.o[rb][j + 2][r] * f16, R.o[rb][j + 3][r] * f16);
        __syncthreads();
#pragma unroll
        for (int g = 0; g < RS; ++g) {                                   // the rows of wavefronts g, g + RS, ..
            const int br = g * 32 + rb * 16 + row;                       // in the block
            float o[8], mt = ms[g][rb * 16 + row], lt = 0.0f;
#pragma unroll
            for (int v = 1; v < TS; ++v) mt = fmaxf(mt, ms[g + v * RS][rb * 16 + row]);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll
            for (int v = 0; v < TS; ++v) {
                lt += ls[g + v * RS][rb * 16 + row] * __builtin_amdgcn_exp2f(ms[g + v * RS][rb * 16 + row] - mt);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += meet[g + v * RS][row][c8 * 8 + e];
            }
            if (a.slots) {
                float *op = st + br * kHeadDim + c8 * 8;
                *reinterpret_cast<float4 *>(op) = make_float4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<float4 *>(op + 4) = make_float4(o[4], o[5], o[6], o[7]);
                if (c8 == 0) { st[kRows * kHeadDim + br] = mt; st[kRows * (kHeadDim + 1) + br] = lt; }
            } else if (row0 + br < rows) store_row8(a, b, h, row0 + br, sq.nodes, c8, o, mt, lt);
        }
        __syncthreads();
    }
}

template <class F, bool ROPE, int RS>
static hipError_t launch_wide_rs(const TreeArgs &a, int blocks, hipStream_t s) {
    const int per_xcd = (blocks + 7) / 8;
    tree_attn_wide<F, ROPE, RS><<<dim3((unsigned)(per_xcd * 8)), dim3(kTrThreads), kTwSmem, s>>>(a, blocks, per_xcd);
    return hipSuccess;
}
hipError_t launch_tree_wide(const TreeArgs &a, int blocks, int block_rows, hipStream_t s) {
    return tree_format(a.T, kHeadDim / a.B, a.fmt, a.S, [&](auto f) {
        typedef decltype(f) F;
        if (a.t.k_rope_f16) return block_rows == 64 ? launch_wide_rs<F, true, 2>(a, blocks, s) : launch_wide_rs<F, true, 4>(a, blocks, s);
        return launch_wide_rs<F, false, 4>(a, blocks, s);
    });
}

}  // namespace qvg
