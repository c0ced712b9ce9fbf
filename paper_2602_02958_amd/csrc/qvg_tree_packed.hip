// Attention over a paged cache, packed form: up to 32 query rows to a block (qvg_tree.hip has the layout that all forms share).
#include "qvg_tree_lane.hpp"

namespace qvg {

// The formats of QVG_TREE_FORMATS: up to four rounds of 2-bit levels, or one of 4-bit levels; any id width.
// The sum over Eq. 7's parts is left to the contractions where that saves vector instructions, of which the decoding is
// made: the centroid rows go to the matrix cores as they are stored, as bf16, and only the residual of the rounds,
// sum_t s_t q_t, is formed, two elements at a time in packed binary16 arithmetic (one round: exact).  So S^T = C Q^T + R Q^T
// with Q as bf16 and as binary16, and O^T = C^T P + R^T P with P as a sum of two bf16 numbers (16 significant bits; one would
// cost 2^-9 of every weight) and as binary16.
// A token's part q.c of a score depends on its centroid alone: at the start of a page the workgroup contracts the page's tables
// with its queries once and keeps the scores of all rows in LDS, where the tokens' accumulators start from what their ids name.
// (Gathering K's rows as well, 256 bytes per token and side, the loop was bound by what the L2s give to gathers, about 10 TB/s:
// one token over 12 heads x 187200 tokens of one round 125 us instead of 91.)  V's rows are gathered, 16 bytes per lane, row and
// octet.  A tile's codes and scales come in with a few wide loads a tile ahead; the V side's codes, all scales and ids pass
// through a few KB of LDS that are the wavefront's own, where they are transposed: tokens become contiguous, so that a lane
// reads four tokens' levels or scales, already paired, at once.
// What bounds it: without a rotation the vector instructions, 378 a tile for 16 rows of one round, two wavefronts to a SIMD
// (registers); one token over 12 heads x 187200 tokens takes 93 us in one round (2.4 TB/s of stored bytes and tables), 133 in two,
// 188 in four (3.8 TB/s).  With a rotation its rows, 256 bytes a token, of which the L2s miss three quarters: 192 us in one round.
template <int RB> __host__ __device__ constexpr int tree_query_bytes() { return RB * 8 * 1024; }
constexpr int kTrMeetBytes = kTrWaves * 16 * kTrPitch * 4;

// Where the centroids' scores may lie in LDS: not where keys are rotated, nor where four stages' tables and 32 rows would leave a
// CU one workgroup.
template <class F, bool ROPE, int RB> __host__ __device__ constexpr bool table_fits() { return !ROPE && (F::S == 1 || RB == 1); }

template <class F, bool ROPE, int RB, bool kTable>
__global__ __launch_bounds__(kTrThreads, 2)
void tree_attn_packed(TreeArgs a, int blocks, int per_xcd) {
    constexpr int S = F::S;
    constexpr int kRows = 16 * RB;
    // One block of 16 rows takes V's rows as they are and P twice; for more rows the values are put together in binary16, 96
    // instructions a tile, and P is taken once, which saves 24 instructions, eight registers and 16 contractions a block
    constexpr bool kSplitV = RB == 1;
    static_assert(!kTable || table_fits<F, ROPE, RB>(), "");
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float ms[kTrWaves][kRows], ls[kTrWaves][kRows];
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
    const int c = lane & 15, kb = lane >> 4;
    uint4 *qlds = reinterpret_cast<uint4 *>(smem);                       // [RB][8][64] fragments
    float *table = reinterpret_cast<float *>(smem + tree_query_bytes<RB>() + kTrWaves * F::wave_bytes);   // [S * K][cols], kTable
    const int cols = S > 1 ? a.table_cols : kRows, col = S > 1 ? c & (cols - 1) : c;

    // ---- Q: fragments 0..3 as bf16 in the order of gather_k, 4..7 as binary16 in the order of the residual's ----
    TreeRows<RB> R;
    int node[RB];                                                        // -1: no such row
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float v[32];
        const QueryRow q(a, sq, b, h, (int64_t)rblk * kRows + rb * 16 + c, v);
        node[rb] = q.node; R.qs[rb] = q.scale(a);
        if (wave == rb % kTrWaves) {                                     // one wavefront leaves them for all
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __builtin_amdgcn_ldexpf(v[i], 9 - q.ex);
#pragma unroll
            for (int i = 0; i < 4; ++i) qlds[(rb * 8 + 4 + i) * 64 + lane] = QueryRow::residual_fragment<F>(v, i);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                q.octet(4 * i + kb, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __builtin_amdgcn_ldexpf(v[e], 9 - q.ex);
                qlds[(rb * 8 + i) * 64 + lane] = pack_bf16x8(v);
            }
        }
    }
    __syncthreads();
    auto qfrag = [&](int rb, int i) { return qlds[(rb * 8 + i) * 64 + lane]; };

    R.clear();
    const TreeLane<F> D(a, sq, b, h, smem + tree_query_bytes<RB>() + wave * F::wave_bytes);
    typedef typename TreeLane<F>::Where Where;
    typedef typename TreeLane<F>::Raw Raw;
    typedef typename TreeLane<F>::Levels Levels;
    floatx4_t (&Sc)[RB][2] = R.s;
    floatx4_t (&O)[RB][8] = R.o;
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
    auto weights = [&]() {
        R.weights([&](int rb, const float (&x)[8]) {
            uint32_t ph[4], pl[4], pf[4];
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
        });
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
                    x[pr] = __builtin_amdgcn_perm(D.word_of(row[2 * pr + 1], j), D.word_of(row[2 * pr], j), j & 1 ? 0x07060302u : 0x05040100u);
                const bf16x8_t v = __builtin_bit_cast(bf16x8_t, make_uint4(x[0], x[1], x[2], x[3]));
                O[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, Phi[0]), O[0][j], 0, 0, 0);
                O[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8_t, Plo[0]), O[0][j], 0, 0, 0);
            } else {
#pragma unroll
                for (int pr = 0; pr < 4; ++pr) x[pr] = as_bits(D.pair_f16(row[2 * pr], row[2 * pr + 1], j));
                add_pv(j, x);
            }
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
    // O^T += R^T P (kSplitV), or (C + R)^T P with the sums of the rows in `start`, four channels of the lane's octet at a time
    // (registers are what the loop is short of)
    auto add_residual = [&](auto start) {
        Levels v;
        D.read_levels(v);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t r[4][4];
            D.template values_v<!kSplitV>(v, half, start, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) add_pv(4 * half + e, r[e]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // the centroids' scores: q . c of every row of the page's tables, 16 rows to a contraction
    auto build_table = [&](int64_t page) {
        const bf16_t *cent = D.ks.cent + page * S * a.K * kHeadDim;
        const int n = S * a.K;
        for (int r0 = wave * 16; r0 < n; r0 += kTrWaves * 16) {
            const uint32_t off = (uint32_t)min(r0 + c, n - 1) * (kHeadDim * 2) + 16 * kb;
            uint4 row[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) row[i] = D.load16(cent, off + 64 * i);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                floatx4_t x = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, row[i]), __builtin_bit_cast(bf16x8_t, qfrag(rb, i)), x, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (S == 1 || c < cols) table[(r0 + 4 * kb + r) * cols + rb * 16 + c] = x[r];
            }
        }
    };
    auto scores_of_ids = [&]() {
#pragma unroll
        for (int st = 0; st < S; ++st)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint4 o = *reinterpret_cast<const uint4 *>(D.offs + st * kTrTile + 16 * hf + 4 * kb);
                const uint32_t at[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = *reinterpret_cast<const float *>(reinterpret_cast<const unsigned char *>(table) + at[r] + (rb * 16 + col) * 4);
                        Sc[rb][hf][r] = st ? Sc[rb][hf][r] + x : x;
                    }
            }
    };

    const halfx2_t none[4] = {};
    const int stop = min(hi, sq.kv_tiles);
    if (pt.lo < stop) {                                                     // uniform over the workgroup
        int ti = pt.first + wave, pi = ti / sq.per_page, in_page = ti - pi * sq.per_page;
        Where cur{-1, 0, 0, 0, 0};
        Raw f;
        if (ti < stop) {
            cur = D.place(pi, in_page, cur);
            D.fetch(cur, f);
        }
        // page by page; a wavefront without tiles in a page still helps with its table
        Where held{-1, 0, 0, 0, 0};
        for (int pg = pt.lo / sq.per_page; pg * sq.per_page < stop; ++pg) {
            if (kTable) {
                held = D.place(pg, 0, held);
                __syncthreads();
                build_table(held.page);
                __syncthreads();
            }
            const int page_end = min(stop, (pg + 1) * sq.per_page);
            while (ti < page_end) {
            D.park(f, kTable ? cols * 4 : kHeadDim * 2);
            D.order_lds();
            uint4 krow[2][4], vrow[8];
            if (!kTable && !ROPE) D.template gather_k<false>(cur, 0, krow);
            const bool more = ti + pt.step < stop;                      // uniform
            Where nxt = cur;
            if (more) {
                in_page += pt.step;
                while (in_page >= sq.per_page) { in_page -= sq.per_page; ++pi; }
                nxt = D.place(pi, in_page, cur);
            }
            // The load counter is in order: the rows that this tile still needs are asked for before the next tile's data, which
            // then has the rest of the tile to arrive
            // (rows of V: at once where all of a tile's rows fit the registers)
            constexpr bool kEarlyV = S == 1;
            auto ahead = [&]() {
                if (!kEarlyV) D.gather_v(cur, 0, vrow);
                if (more) D.fetch(nxt, f);
            };
            uint4 kh[2][S][4], rp[2][4];
            if (ROPE) {
                D.gather_half(cur, 0, kh[0]);
                D.gather_rope(cur, 0, rp[0]);
                D.gather_rope(cur, 1, rp[1]);
                if (S == 1) D.gather_half(cur, 1, kh[1]);
            }
            if (kEarlyV) D.gather_v(cur, 0, vrow);
            if (kTable) scores_of_ids(); else R.clear_scores();
            if (ROPE) {
                uint4 kf[2][4];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    float v[32];
                    D.sum_rows(kh[S == 1 ? hf : 0], v);
                    if (S > 1 && hf == 0) D.gather_half(cur, 1, kh[0]);
                    D.template whole_k<true>(f, hf, v, rp[hf], kf[hf]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) scores_of_residual(i, kf[0][i], kf[1][i]);
                __builtin_amdgcn_sched_barrier(0);
                ahead();
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint4 r0, r1;
                    D.template residual_k<false>(f, 0, i, none, r0);
                    D.template residual_k<false>(f, 1, i, none, r1);
                    scores_of_residual(i, r0, r1);
                }
                if (!kTable) {
                    scores_of_rows(krow);
                    for (int st = 1; st < S; ++st) {
                        D.template gather_k<false>(cur, st, krow);
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
                R.hide(see);
            }
            weights();
            __builtin_amdgcn_sched_barrier(0);
            if (kSplitV) {
                add_residual([&](int, int) { return halfx2_t{}; });
                __builtin_amdgcn_sched_barrier(0);
                add_rows(vrow);
                for (int st = 1; st < S; ++st) {
                    D.gather_v(cur, st, vrow);
                    add_rows(vrow);
                }
            } else if (S == 1) {
                add_residual([&](int j, int pr) { return D.pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j); });
            } else {
                halfx2_t sum[8][4];
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int pr = 0; pr < 4; ++pr) sum[j][pr] = D.pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j);
                for (int st = 1; st < S; ++st) {
                    D.gather_v(cur, st, vrow);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int pr = 0; pr < 4; ++pr) sum[j][pr] += D.pair_f16(vrow[2 * pr], vrow[2 * pr + 1], j);
                }
                add_residual([&](int j, int pr) { return sum[j][pr]; });
            }
            D.order_lds();
            ti += pt.step;
            cur = nxt;
            }
        }
    }

    // ---- the tail's and the new tokens' tiles ---------------------------------------------------
    int tail_at = pt.first + wave;
    if (tail_at < sq.kv_tiles) tail_at += (sq.kv_tiles - tail_at + pt.step - 1) / pt.step * pt.step;
    for (int ti = tail_at; ti < hi; ti += pt.step) {
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
            for (int rb = 0; rb < RB; ++rb) any |= see[rb] = node_sees(t, b, node[rb], first, there);
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
        R.clear_scores();
        scores_of_rows(krow);
        R.hide(see);
        weights();
        // (a new token that no row sees may be no number)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!((any >> (16 * (e >> 2) + 4 * kb + (e & 3))) & 1u)) vrow[e] = make_uint4(0u, 0u, 0u, 0u);
        add_rows(vrow);
    }
    __syncthreads();                                                     // (the meeting place lies over the wavefronts' own LDS)
    finish_block<RB>(a, at, sq.nodes, reinterpret_cast<float (*)[16][kTrPitch]>(smem), ms, ls, R.o, R.m, R.l);
}

template <class F, bool ROPE, int RB, bool TABLE>
static hipError_t launch_packed_form(const TreeArgs &a, int blocks, int lds, hipStream_t s) {
    const int per_xcd = (blocks + 7) / 8;
    if (lds < kTrMeetBytes) lds = kTrMeetBytes;
    if (lds > 64 * 1024) {
        static LdsHighWater mark;
        const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(tree_attn_packed<F, ROPE, RB, TABLE>), (size_t)lds, mark);
        if (e != hipSuccess) return e;
    }
    tree_attn_packed<F, ROPE, RB, TABLE><<<dim3((unsigned)(per_xcd * 8)), dim3(kTrThreads), (size_t)lds, s>>>(a, blocks, per_xcd);
    return hipSuccess;
}
// A table costs a contraction for each 16 of its rows, and saves a row's gather for each token that a workgroup meets in a page:
// those of the page, or of the workgroup's part where that is shorter.  One token over 12 heads x 187200 tokens, K = 256, one
// round: pages of 512 tokens 158 us with tables and 153 gathered, of 1024 124 and 141, of 4680 91 and 124; four stages,
// 1024 tokens, 391 and 538.  For 32 rows, whose tables are twice as large, 1024 tokens 140 and 148, four rounds 267 and 261,
// and not where a CU holds one workgroup (K = 512, 4680 tokens: 164 and 162, 1024 tokens 251 and 172).
template <class F, bool ROPE, int RB>
static hipError_t launch_packed_rb(TreeArgs a, int blocks, hipStream_t s) {
    constexpr int own = tree_query_bytes<RB>() + kTrWaves * F::wave_bytes;
    // (two workgroups to a CU: 79 KB each and what the kernel declares itself)
    if constexpr (table_fits<F, ROPE, RB>()) {
        static_assert(own + F::S * kMaxClusters * 16 * RB * 4 + kTrWaves * 16 * RB * 8 <= 160 * 1024, "the largest table must fit a CU");
        int64_t met = a.t.page_len;
        const int64_t pages = (int64_t)a.t.n_seqs * a.t.table_pages;
        if (a.slots && pages < a.slots) met = pages * a.t.page_len / a.slots;
        // Several stages' tables: columns for the rows that there are, where 16 would leave a CU one workgroup (one token, four
        // stages, 495 -> 391 us)
        const int64_t rows = (int64_t)a.t.group * a.t.n_nodes;
        auto bytes = [&](int cols) { return own + (F::S * a.K + 15) / 16 * 16 * cols * 4; };
        a.table_cols = 16 * RB;
        while (F::S > 1 && a.table_cols / 2 >= rows && bytes(a.table_cols) > 79 * 1024) a.table_cols /= 2;
        const int lds = bytes(a.table_cols);
        if (met >= (RB == 1 ? 3 : 4) * (int64_t)a.K && (RB == 1 || lds <= 79 * 1024)) return launch_packed_form<F, ROPE, RB, true>(a, blocks, lds, s);
    }
    return launch_packed_form<F, ROPE, RB, false>(a, blocks, own, s);
}
template <class F>
static hipError_t launch_packed(const TreeArgs &a, int blocks, int br, hipStream_t s) {
    if (a.t.k_rope_f16)
        return br == 16 ? launch_packed_rb<F, true, 1>(a, blocks, s) : launch_packed_rb<F, true, 2>(a, blocks, s);
    return br == 16 ? launch_packed_rb<F, false, 1>(a, blocks, s) : launch_packed_rb<F, false, 2>(a, blocks, s);
}
hipError_t launch_tree_packed(const TreeArgs &a, int blocks, int block_rows, hipStream_t s) {
    return tree_format(a.T, kHeadDim / a.B, a.fmt, a.S, [&](auto f) { return launch_packed<decltype(f)>(a, blocks, block_rows, s); });
}

}  // namespace qvg
