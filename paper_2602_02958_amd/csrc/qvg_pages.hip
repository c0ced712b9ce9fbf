// What a paged cache needs beside its attention: the masks of draft trees, the kept tokens' way into the tail, page copies.
#include "qvg_tree.hpp"

namespace qvg {

// ---- tree masks ----------------------------------------------------------------------------------
// A node's row is its parent's row and its own bit.  One workgroup to a tree.  First every node finds, inside its block of 32
// nodes, its ancestors and the parent of the topmost one (five pointer doublings by lane exchange, all blocks at once);
// then the blocks take turns: the rows of a block are complete below its own word once the row of that outside ancestor is
// copied, which lies in an earlier block.  So a tree of n nodes takes n / 32 steps however deep it is.
__global__ __launch_bounds__(1024)
void tree_mask_kernel(int n, int words, const int32_t *parents, const int32_t *nodes, uint32_t *mask, int32_t *depth) {
    extern __shared__ uint32_t lds[];
    uint32_t *rows = lds;                                   // [n][words]
    int *exit_of = reinterpret_cast<int *>(rows + n * words);          // [words * 32] outside ancestor, -1: none, -2: a hole
    uint32_t *inside = reinterpret_cast<uint32_t *>(exit_of + words * 32);   // [words * 32]
    const int b = blockIdx.x, tid = threadIdx.x;
    int live = n;
    if (nodes) { live = nodes[b]; live = live < 0 ? 0 : (live > n ? n : live); }
    for (int i = tid; i < words * 32; i += blockDim.x) {               // (a multiple of 64 threads and 32 nodes: halves of a wavefront agree)
        int up = i < live ? parents[(int64_t)b * n + i] : -2;
        if (up < -1 || up >= i) up = -2;
        const int base = i & ~31;
        uint32_t bits = 1u << (i & 31);
#pragma unroll
        for (int step = 0; step < 5; ++step) {
            const bool in = up >= base;
            const int from = (tid & 32) | (in ? up - base : tid & 31);
            const uint32_t obits = __shfl(bits, from, 64);
            const int oup = __shfl(up, from, 64);
            if (in) { bits |= obits; up = oup; }
        }
        exit_of[i] = up; inside[i] = bits;
    }
    __syncthreads();
    for (int w = 0; w < words; ++w) {
        // 32 rows of w + 1 words
        for (int e = tid; e < 32 * words; e += blockDim.x) {
            const int i = w * 32 + e / words, k = e - e / words * words;
            if (i < n) {
                const int up = exit_of[i];
                // (a hole's row is empty: the outside ancestor's own word tells)
                const bool hole = up == -2 || (up >= 0 && rows[up * words + (up >> 5)] == 0u);
                const uint32_t v = hole || k > w ? 0u : k == w ? inside[i] : (up >= 0 ? rows[up * words + k] : 0u);
                rows[i * words + k] = v;
                mask[((int64_t)b * n + i) * words + k] = v;
            }
        }
        __syncthreads();
    }
    if (depth)
        for (int i = tid; i < n; i += blockDim.x) {
            int d = -1;
            for (int k = 0; k < words; ++k) d += __builtin_popcount(rows[i * words + k]);
            depth[(int64_t)b * n + i] = d;
        }
}

hipError_t launch_tree_mask(int n_seqs, int n_nodes, const int32_t *parents, const int32_t *nodes, uint32_t *mask, int32_t *depth,
                            hipStream_t s) {
    const int words = (n_nodes + 31) / 32;
    const size_t lds = ((size_t)n_nodes * words + 2 * (size_t)words * 32) * sizeof(uint32_t);
    static LdsHighWater mark;
    if (lds > 64 * 1024) {
        const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(tree_mask_kernel), lds, mark);
        if (e != hipSuccess) return e;
    }
    const int threads = words <= 2 ? 64 : words <= 8 ? 256 : 1024;
    tree_mask_kernel<<<dim3((unsigned)n_seqs), dim3((unsigned)threads), lds, s>>>(n_nodes, words, parents, nodes, mask, depth);
    return hipGetLastError();
}

// ---- kept tokens --------------------------------------------------------------------------------------
// 16 lanes to a row of 128 bf16, both sides.
__global__ __launch_bounds__(256)
void keep_nodes_kernel(KeepArgs a) {
    const unsigned unit = blockIdx.x / (unsigned)a.blocks;                // sequence and unit (K heads, then V heads)
    const int i = (int)(blockIdx.x - unit * (unsigned)a.blocks) * 16 + (int)(threadIdx.x >> 4), c8 = threadIdx.x & 15;
    const int b = (int)(unit / (unsigned)(2 * a.H)), u = (int)(unit - (unsigned)b * (unsigned)(2 * a.H));
    const int side = u >= a.H, h = u - side * a.H;
    int keep = a.keep[b], len = a.tail_len[b];
    keep = keep < 0 ? 0 : (keep > a.n_path ? a.n_path : keep);
    len = len < 0 ? 0 : (len > a.capacity ? a.capacity : len);
    if (i >= keep || len + i >= a.capacity) return;
    const int from = a.path[(int64_t)b * a.n_path + i];
    if (from < 0 || from >= a.n_nodes) return;
    const bf16_t *src = (side ? a.v_new : a.k_new) + b * a.new_seq + h * a.new_head + from * a.new_node;
    bf16_t *dst = (side ? a.v_tail : a.k_tail) + b * a.tail_seq + h * a.tail_head + (int64_t)(len + i) * a.tail_token;
    reinterpret_cast<uint4 *>(dst)[c8] = reinterpret_cast<const uint4 *>(src)[c8];
}
// (in a launch of its own, behind the rows: tail_len_out may be tail_len)
__global__ __launch_bounds__(256)
void keep_lengths_kernel(KeepArgs a) {
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= a.n_seqs) return;
    int keep = a.keep[b], len = a.tail_len[b];
    keep = keep < 0 ? 0 : (keep > a.n_path ? a.n_path : keep);
    len = len < 0 ? 0 : (len > a.capacity ? a.capacity : len);
    a.tail_len_out[b] = len + keep > a.capacity ? a.capacity : len + keep;
}
hipError_t launch_keep_nodes(const KeepArgs &a, hipStream_t s) {
    if (a.n_path > 0)
        keep_nodes_kernel<<<dim3((unsigned)((int64_t)a.n_seqs * 2 * a.H * a.blocks)), dim3(256), 0, s>>>(a);
    if (a.tail_len_out) keep_lengths_kernel<<<dim3((unsigned)((a.n_seqs + 255) / 256)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

// ---- page copies -----------------------------------------------------------------------------------------
constexpr int kCpPairs = 192;                 // pairs of a launch: they travel in its arguments
constexpr int kCpBlock = 256 * 64;            // bytes a workgroup copies: four 16-byte pieces to a thread
struct CopyArgs {
    PageArray array[4];
    int width[4];                             // bytes of a piece: what the array's pages are all aligned to, up to 16
    int first_block[5];                       // workgroups of a page, array by array
    int units;
    int32_t src[kCpPairs], dst[kCpPairs];
};
template <typename W>
__device__ __forceinline__ void copy_pieces(const uint8_t *src, uint8_t *dst, int64_t from, int64_t bytes) {
    const int64_t end = from + kCpBlock < bytes ? from + kCpBlock : bytes;
    const W *s = reinterpret_cast<const W *>(src);
    W *d = reinterpret_cast<W *>(dst);
    for (int64_t i = from / (int64_t)sizeof(W) + threadIdx.x; i < end / (int64_t)sizeof(W); i += 4 * 256) {
        W v[4];
        const int64_t n = end / (int64_t)sizeof(W);
#pragma unroll
        for (int k = 0; k < 4; ++k) if (i + k * 256 < n) v[k] = s[i + k * 256];
#pragma unroll
        for (int k = 0; k < 4; ++k) if (i + k * 256 < n) d[i + k * 256] = v[k];
    }
}
__global__ __launch_bounds__(256)
void copy_pages_kernel(CopyArgs a) {
    const int pair = blockIdx.z, unit = blockIdx.y, blk = blockIdx.x;
    int k = 0;
    while (blk >= a.first_block[k + 1]) ++k;                             // (the last entry is the grid's width)
    const PageArray p = a.array[k];
    const uint8_t *src = p.src + unit * p.src_unit + a.src[pair] * p.bytes;
    uint8_t *dst = p.dst + unit * p.dst_unit + a.dst[pair] * p.bytes;
    const int64_t from = (int64_t)(blk - a.first_block[k]) * kCpBlock;
    switch (a.width[k]) {
        case 16: copy_pieces<uint4>(src, dst, from, p.bytes); break;
        case 8: copy_pieces<uint2>(src, dst, from, p.bytes); break;
        case 4: copy_pieces<uint32_t>(src, dst, from, p.bytes); break;
        case 2: copy_pieces<uint16_t>(src, dst, from, p.bytes); break;
        default: copy_pieces<uint8_t>(src, dst, from, p.bytes); break;
    }
}
hipError_t launch_copy_pages(const PageArray (&arrays)[4], int units, int64_t n_pairs, const int32_t *src, const int32_t *dst,
                             hipStream_t s) {
    CopyArgs a{};
    a.units = units;
    for (int k = 0; k < 4; ++k) {
        a.array[k] = arrays[k];
        const uint64_t all = (uint64_t)reinterpret_cast<uintptr_t>(arrays[k].src) | (uint64_t)reinterpret_cast<uintptr_t>(arrays[k].dst) |
                             (uint64_t)arrays[k].bytes | (uint64_t)arrays[k].src_unit | (uint64_t)arrays[k].dst_unit | 16u;
        a.width[k] = (int)(all & (~all + 1));
        a.first_block[k + 1] = a.first_block[k] + (int)((arrays[k].bytes + kCpBlock - 1) / kCpBlock);
    }
    for (int64_t at = 0; at < n_pairs; at += kCpPairs) {
        const int n = (int)(n_pairs - at < kCpPairs ? n_pairs - at : kCpPairs);
        for (int i = 0; i < n; ++i) { a.src[i] = src[at + i]; a.dst[i] = dst[at + i]; }
        copy_pages_kernel<<<dim3((unsigned)a.first_block[4], (unsigned)units, (unsigned)n), dim3(256), 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace qvg
