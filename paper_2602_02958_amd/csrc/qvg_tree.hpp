// Arguments of the operators over paged caches (qvg_tree.hip: attention of a step's new tokens; qvg_pages.hip: tree
// masks, kept tokens, page copies) and their launchers.
#pragma once
#include "qvg_internal.hpp"

namespace qvg {

constexpr int kTrTile = 32;        // tokens of a tile
// Tiles of 0 .. 2^31 - 1 tokens (the sum that rounds up may pass 31 bits).
__host__ __device__ inline int tree_tiles(int tokens) { return (int)(((uint32_t)tokens + (uint32_t)(kTrTile - 1)) / (uint32_t)kTrTile); }

struct PoolSide {                  // K or V pool: [H] units of pool_tokens tokens, pool_pages tables
    const bf16_t *cent; const uint8_t *ids; const uint8_t *codes; const uint8_t *scales;
};
struct TreeArgs {
    PoolSide k, v;
    int H, K, B, T, S, fmt, id_wide;
    qvg_tree_step t;
    float scale;
    int rows, row_blocks;          // rows of a block of a KV head's query rows, and the blocks
    int slots;                     // workgroups of a block of all sequences, dealt to them by their lengths; 0: one to each, undivided
    int share;                     // consecutive parts of a sequence that walk the same range of tiles together, a round each in turn
    int table_cols;                // query rows of a table of the centroids' scores: a power of two
    float *state;                  // partial results of the slots
    int2 *places;                  // [n_seqs] a sequence's first slot and its parts, for the joining launch
};
// The stored formats of the package's configurations and of the paper's presets, and their neighbours in group size: X(rounds,
// groups per token, E4M3 scales, 4-bit levels, smoothing stages).  They have kernels of their own; any other one is decoded
// element by element (one token over 12 heads x 187200 tokens: two rounds 133 us in the packed form and, with E4M3 scales, 1.1 ms so;
// one round of 4-bit levels with binary16 scales 0.7 ms, two smoothing stages 1.15 ms).
#define QVG_TREE_FORMATS(X)                                                                                              \
    X(1, 2, true, false, 1) X(1, 8, true, false, 1) X(1, 8, true, false, 4) X(1, 2, true, true, 1) X(1, 8, true, true, 4) \
    X(1, 2, false, false, 1) X(2, 2, false, false, 1) X(2, 4, false, false, 1) X(3, 2, false, false, 1)                   \
    X(3, 4, false, false, 1) X(4, 2, false, false, 1) X(4, 4, false, false, 1)
inline bool tree_packed(int T, int G, int fmt, int S) {
#define QVG_TREE_IS(t, g, fp8, i4, s) if (T == t && G == g && S == s && fmt == ((fp8 ? kFmtE4M3 : 0) | (i4 ? kFmtInt4 : 0))) return true;
    QVG_TREE_FORMATS(QVG_TREE_IS)
#undef QVG_TREE_IS
    return false;
}
// Rows of a KV head (group * n_nodes) are taken in blocks of 16 or 32, which a wavefront holds, and in the packed formats of 64 or
// 128, whose wavefronts share what they decode: beyond 64 rows (12 heads x 187200 tokens, two rounds, each pair timed on one box:
// 128 rows shared 335 us and 503 in blocks of 32; 64 rows 272 and 255), with a rotation, which costs more, beyond 32 (64 rows 355
// and 460).  As they are now: 128 rows 312 us, 64 rows in two blocks 245, rotated 64 rows 360.
inline int tree_block_rows(int64_t rows, bool packed, bool rotated) {
    return rows <= 16 ? 16 : rows <= 32 || !packed ? 32 : rows > 64 ? 128 : rotated ? 64 : 32;
}
struct TreePlan { int rows, row_blocks, slots, share; size_t state_bytes; };      // (as in TreeArgs)
TreePlan tree_plan(const qvg_params &p, const qvg_tree_step &t, bool rotated);
hipError_t launch_tree_packed(const TreeArgs &a, int blocks, int block_rows, hipStream_t s);
hipError_t launch_tree_wide(const TreeArgs &a, int blocks, int block_rows, hipStream_t s);
hipError_t launch_attn_tree(const TreeArgs &a, hipStream_t s);

hipError_t launch_tree_mask(int n_seqs, int n_nodes, const int32_t *parents, const int32_t *nodes, uint32_t *mask, int32_t *depth,
                            hipStream_t s);

struct KeepArgs {
    const bf16_t *k_new, *v_new; int64_t new_seq, new_head, new_node;
    bf16_t *k_tail, *v_tail; int64_t tail_seq, tail_head, tail_token;
    const int32_t *path, *keep, *tail_len; int32_t *tail_len_out;
    int H, n_seqs, n_nodes, n_path, capacity;
    int blocks;                    // of 16 rows of a path
    int lengths_here;              // the rows' launch writes tail_len_out too
};
hipError_t launch_keep_nodes(const KeepArgs &a, hipStream_t s);

struct PageArray {                 // one of a pool's four arrays
    const uint8_t *src; uint8_t *dst;
    int64_t bytes;                 // of a page
    int64_t src_unit, dst_unit;    // bytes of a unit
};
hipError_t launch_copy_pages(const PageArray (&arrays)[4], int units, int64_t n_pairs, const int32_t *src, const int32_t *dst,
                             hipStream_t s);

}  // namespace qvg
