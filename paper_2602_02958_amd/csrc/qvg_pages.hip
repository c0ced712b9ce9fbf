// What a paged cache needs beside its attention: the masks of draft trees, the kept tokens' way into the tail, page copies.
#include "qvg_tree.hpp"

namespace qvg {

// ---- tree masks ----------------------------------------------------------------------------------
// A node's row is its parent's row and its own bit.  One workgroup to a tree.  First every node finds, inside its block of 32
// nodes, its ancestors and the parent of the topmost one (five pointer doublings by lane exchange, all blocks at once);
// then the blocks take turns: the rows of a block are complete below its own word once the row of that outside ancestor is
// copied, which lies in an earlier block.  So a tree of n nodes takes n / 32 steps however deep it is.  The rows go out at the
// end: a store in every step made its barrier wait for memory (64 trees of 1000 nodes 36 us instead of 22; the rows
// that they write, 8 MB, take 2 us at the rate of a copy: what bounds a tree is its 32 steps of a barrier and two LDS accesses).
__global__ __launch_bounds__(1024)
void tree_mask_kernel(int n, int words, const int32_t *parents, const int32_t *nodes, uint32_t *mask, int32_t *depth) {
    extern __shared__ uint32_t lds[];
    uint32_t *rows = lds;                                   // [n][words]
    int *exit_of = reinterpret_cast<int *>(rows + n * words);          // [words * 32] outside ancestor, -1: none, -2: a hole
    uint32_t *inside = reinterpret_cast<uint32_t *>(exit_of + words * 32);   // [words * 32]
    int *deep = reinterpret_cast<int *>(inside + words * 32);          // [words * 32] depths, -1: a hole
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
    // lanes of a wavefront have neighbouring words of a row; `shift`: words rounded up to a power of two
    int shift = 0;
    while ((1 << shift) < words) ++shift;
    for (int w = 0; w < words; ++w) {
        for (int e = tid; e < 32 << shift; e += blockDim.x) {
            const int i = w * 32 + (e >> shift), k = e & ((1 << shift) - 1);
            if (i < n && k < words) {
                const int up = exit_of[i];
                const bool hole = up == -2 || (up >= 0 && deep[up] < 0);
                rows[i * words + k] = hole || k > w ? 0u : k == w ? inside[i] : (up >= 0 ? rows[up * words + k] : 0u);
                if (k == 0) deep[i] = hole ? -1 : __builtin_popcount(inside[i]) + (up >= 0 ? deep[up] : -1);
            }
        }
        __syncthreads();
    }
    uint32_t *out = mask + (int64_t)b * n * words;
    for (int e = tid; e < n * words; e += blockDim.x) out[e] = rows[e];
    if (depth)
        for (int i = tid; i < n; i += blockDim.x) depth[(int64_t)b * n + i] = deep[i];
}

hipError_t launch_tree_mask(int n_seqs, int n_nodes, const int32_t *parents, const int32_t *nodes, uint32_t *mask, int32_t *depth,
                            hipStream_t s) {
    const int words = (n_nodes + 31) / 32;
    const size_t lds = ((size_t)n_nodes * words + 3 * (size_t)words * 32) * sizeof(uint32_t);
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
// 16 lanes to a row of 128 bf16, 16 rows of a path in one unit of a sequence to a workgroup.  64 paths over 40 heads, 31 MB both
// ways, which a large copy takes 6 us for: 11.8 us, three loads one after the other in 15360 small workgroups (eight units to one
// with all their loads in flight: 12.8).  A sequence alone takes 2.7 us (4.6).
__global__ __launch_bounds__(256)
void keep_nodes_kernel(KeepArgs a) {
    const unsigned unit = blockIdx.x / (unsigned)a.blocks;                // sequence and unit (K heads, then V heads)
    const int i = (int)(blockIdx.x - unit * (unsigned)a.blocks) * 16 + (int)(threadIdx.x >> 4), c8 = threadIdx.x & 15;
    const int b = (int)(unit / (unsigned)(2 * a.H)), u = (int)(unit - (unsigned)b * (unsigned)(2 * a.H));
    const int side = u >= a.H, h = u - side * a.H;
    int keep = a.keep[b], len = a.tail_len[b];
    keep = keep < 0 ? 0 : (keep > a.n_path ? a.n_path : keep);
    len = len < 0 ? 0 : (len > a.capacity ? a.capacity : len);
    // (where the new lengths have a place of their own; else they wait for the rows to be done with the old ones)
    const int room = a.capacity - len;                                  // (len + keep may pass 31 bits)
    if (a.lengths_here && u == 0 && i == 0 && c8 == 0) a.tail_len_out[b] = len + (keep < room ? keep : room);
    if (i >= keep || i >= room) return;
    const int from = a.path[(int64_t)b * a.n_path + i];
    if (from < 0 || from >= a.n_nodes) return;
    const bf16_t *src = (side ? a.v_new : a.k_new) + b * a.new_seq + h * a.new_head + from * a.new_node;
    bf16_t *dst = (side ? a.v_tail : a.k_tail) + b * a.tail_seq + h * a.tail_head + (int64_t)(len + i) * a.tail_token;
    reinterpret_cast<uint4 *>(dst)[c8] = reinterpret_cast<const uint4 *>(src)[c8];
}
// (in a launch of its own, behind the rows, when tail_len_out may be tail_len)
__global__ __launch_bounds__(256)
void keep_lengths_kernel(KeepArgs a) {
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= a.n_seqs) return;
    int keep = a.keep[b], len = a.tail_len[b];
    keep = keep < 0 ? 0 : (keep > a.n_path ? a.n_path : keep);
    len = len < 0 ? 0 : (len > a.capacity ? a.capacity : len);
    a.tail_len_out[b] = len + (keep < a.capacity - len ? keep : a.capacity - len);
}
hipError_t launch_keep_nodes(const KeepArgs &a, hipStream_t s) {
    if (a.blocks > 0)
        keep_nodes_kernel<<<dim3((unsigned)((int64_t)a.n_seqs * 2 * a.H * a.blocks)), dim3(256), 0, s>>>(a);
    if (a.tail_len_out && !a.lengths_here) keep_lengths_kernel<<<dim3((unsigned)((a.n_seqs + 255) / 256)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

// ---- page copies -----------------------------------------------------------------------------------------
constexpr int kCpPairs = 192;                 // pairs of a launch: they travel in its arguments
constexpr int kCpBlock = 256 * 64;            // bytes a workgroup copies: four 16-byte pieces to a thread
struct CopyArgs {
    PageArray array[4];
    int width[4];                             // bytes of a piece: what the array's pages are all aligned to, up to 16
    int first_block[5];                       // workgroups of a page, array by array
    int32_t src[kCpPairs], dst[kCpPairs];
};
template <typename W>
__device__ __forceinline__ void copy_pieces(const uint8_t *src, uint8_t *dst, int64_t from, int64_t bytes) {
    const int n = (int)((from + kCpBlock < bytes ? (int64_t)kCpBlock : bytes - from) / (int64_t)sizeof(W));
    const W *s = reinterpret_cast<const W *>(src + from);
    W *d = reinterpret_cast<W *>(dst + from);
    const int i = (int)threadIdx.x;
    if (i + 3 * 256 < n) {                                               // four pieces at a time (all there is of 16-byte ones)
        for (int j = i; j + 3 * 256 < n; j += 4 * 256) {
            const W x0 = s[j], x1 = s[j + 256], x2 = s[j + 512], x3 = s[j + 768];
            d[j] = x0; d[j + 256] = x1; d[j + 512] = x2; d[j + 768] = x3;
        }
    }
    for (int j = i + (n - i > 0 ? (n - i + 255) / 256 / 4 * 4 * 256 : 0); j < n; j += 256) d[j] = s[j];
}
// Every field that a workgroup needs is asked for at once, the arrays' four descriptions among them: the arguments lie in memory
// that is far away, and one after the other (or as a value, which indexed at run time every thread keeps in scratch memory)
// they took 16 us of a copy of 1 MB, which takes 3 us so.  20 pages of 4680 tokens of 24 units, 714 MB both ways: 141 us,
// 5.1 TB/s, the rate of a large copy.
__global__ __launch_bounds__(256)
void copy_pages_kernel(CopyArgs) {
    const CopyArgs &a = *(const CopyArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    const int pair = blockIdx.z, unit = blockIdx.y, blk = blockIdx.x;
    const int64_t from_page = a.src[pair], to_page = a.dst[pair];
    const PageArray p0 = a.array[0], p1 = a.array[1], p2 = a.array[2], p3 = a.array[3];
    const int f1 = a.first_block[1], f2 = a.first_block[2], f3 = a.first_block[3];
    const int w0 = a.width[0], w1 = a.width[1], w2 = a.width[2], w3 = a.width[3];
    auto pick = [&](auto x0, auto x1, auto x2, auto x3) { return blk < f1 ? x0 : blk < f2 ? x1 : blk < f3 ? x2 : x3; };
    const int64_t bytes = pick(p0.bytes, p1.bytes, p2.bytes, p3.bytes);
    const uint8_t *src = pick(p0.src, p1.src, p2.src, p3.src) + unit * pick(p0.src_unit, p1.src_unit, p2.src_unit, p3.src_unit) + from_page * bytes;
    uint8_t *dst = pick(p0.dst, p1.dst, p2.dst, p3.dst) + unit * pick(p0.dst_unit, p1.dst_unit, p2.dst_unit, p3.dst_unit) + to_page * bytes;
    const int64_t from = (int64_t)(blk - pick(0, f1, f2, f3)) * kCpBlock;
    switch (pick(w0, w1, w2, w3)) {
        case 16: copy_pieces<uint4>(src, dst, from, bytes); break;
        case 8: copy_pieces<uint2>(src, dst, from, bytes); break;
        case 4: copy_pieces<uint32_t>(src, dst, from, bytes); break;
        case 2: copy_pieces<uint16_t>(src, dst, from, bytes); break;
        default: copy_pieces<uint8_t>(src, dst, from, bytes); break;
    }
}
hipError_t launch_copy_pages(const PageArray (&arrays)[4], int units, int64_t n_pairs, const int32_t *src, const int32_t *dst,
                             hipStream_t s) {
    CopyArgs a{};
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
