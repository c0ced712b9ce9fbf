// Arguments of the rotary operators and of the caches of 16-bit pages (qvg_rope.hip: tables, turned rows, appending;
// qvg_attn_pages.hip: attention), and their launchers.
#pragma once
#include "qvg_internal.hpp"

namespace qvg {

// n / d for n below 2^31 as a multiplication, (mulhi(n, mul) + n) >> shift: division by an invariant number after Granlund and Montgomery (1994)
struct FastDiv { uint32_t d, mul, shift; };
inline FastDiv fast_div(uint32_t d) {
    uint32_t s = 0;
    while (s < 31 && (1u << s) < d) ++s;
    return {d, (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << s) - d)) / d + 1), s};
}
__host__ __device__ __forceinline__ uint32_t quotient(uint32_t n, const FastDiv &f) {
    return ((uint32_t)(((uint64_t)n * f.mul) >> 32) + n) >> f.shift;
}

struct RopeTableArgs {
    int64_t n_rows; int n_pairs, n_axes; int64_t first;
    const double *freq; const int32_t *positions; float amplitude; void *out;
    uint8_t axis[256];
    int64_t first_block;                          // of a launch
};
hipError_t launch_rope_table(const RopeTableArgs &a, bool f32, hipStream_t s);

// Rows of x to out, or of k_new and v_new to pages
struct TurnArgs {
    const void *x, *v;                            // v: appending
    void *out;
    int64_t x_seq, x_head, x_tok, o_seq, o_head, o_tok;
    qvg_rotary r;                                 // table nullptr: rows stay as they are
    const int32_t *first; int backward;
    int H, d, n_tokens; int64_t tokens;           // tokens: of all sequences
    int units;                                    // pieces of a row (launch_rope, launch_append)
    FastDiv by_units, by_tokens;
    int64_t first_block;                          // of a launch
    // appending
    void *k_pages, *v_pages; int64_t head, page, tok;     // strides
    const int32_t *table, *kv_len, *live; int32_t *len_out;
    int table_pages, capacity, lengths_here;
    uint32_t pool_pages; FastDiv by_page;
};
hipError_t launch_rope(TurnArgs &a, int type, hipStream_t s);
hipError_t launch_append(TurnArgs &a, int n_seqs, int type, hipStream_t s);

constexpr int kPgTile = 32;                       // tokens of a tile
__host__ __device__ inline int page_tiles(int tokens) { return (int)(((uint32_t)tokens + (uint32_t)(kPgTile - 1)) / (uint32_t)kPgTile); }
struct PageAttnArgs {
    qvg_page_cache c;
    qvg_page_step t;
    float scale;                                  // times log2(e)
    int paged;                                    // tiles end where pages do (else they run on over them)
    FastDiv by_page, by_tiles, by_units, by_blocks, by_new;      // tokens of a page, tiles of one; heads x row blocks, row blocks, new tokens
    int rows, row_blocks;                         // rows of a block of a KV head's query rows, and the blocks
    int slots;                                    // workgroups of a block of all sequences, dealt to them by their lengths; 0: one to each
    int extra, kept;                              // slots beyond one to a sequence; partial results of a block, at most
    float *state;                                 // [blocks of all sequences][kept] partial results
    int2 *places;                                 // [n_seqs] a sequence's first partial result and its parts, for the joining launch
};
struct PagePlan { int rows, row_blocks, slots, extra, kept, paged; size_t state_bytes; };      // (as in PageAttnArgs)
bool page_attn_dim(int d);
hipError_t launch_attn_pages(const PageAttnArgs &a, hipStream_t s);

}  // namespace qvg
