// C ABI of libqvg: argument validation and the order in which kernels are enqueued.
// Compiled as HIP host code; holds no kernel and no arithmetic of the method.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <mutex>
#include <new>

#include "qvg.h"
#include "qvg_attn_pages.hpp"
#include "qvg_internal.hpp"
#include "qvg_tree.hpp"

using namespace qvg;

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t v) { return (v + 255u) & ~(size_t)255u; }
// Chunk counts and lengths: any chunk_len >= 1 is accepted (one that is not shorter than the cache, up to
// INT64_MAX, means one chunk), so no sum with it may overflow.  The kernels and the size rules
// get a length of at most 2^36, beyond every token count, which leaves them room for theirs.
inline int64_t chunk_count(int64_t n_tokens, int64_t chunk_len) { return n_tokens / chunk_len + (n_tokens % chunk_len != 0); }
inline int64_t bounded_chunk_len(int64_t chunk_len) { return chunk_len < ((int64_t)1 << 36) ? chunk_len : (int64_t)1 << 36; }

int check_params(const qvg_params *p) {
    if (!p) return QVG_ERR_NULL;
    if (p->n_heads < 1 || p->n_heads > 65535) return QVG_ERR_BAD_PARAM;
    if (p->n_clusters < 1 || p->n_clusters > kMaxClusters) return QVG_ERR_BAD_PARAM;
    if (p->n_stages < 1 || p->n_stages > kMaxStages) return QVG_ERR_BAD_PARAM;
    if (p->kmeans_iters < 0) return QVG_ERR_BAD_PARAM;
    if (p->head_dim < 1 || p->n_smooth_stages < 1) return QVG_ERR_BAD_PARAM;
    if (p->group_size < 1 || p->head_dim % p->group_size != 0) return QVG_ERR_BAD_PARAM;
    if (p->bits != 2 && p->bits != 4) return QVG_ERR_BAD_PARAM;
    if (p->scale_format != QVG_SCALE_F16 && p->scale_format != QVG_SCALE_E4M3) return QVG_ERR_BAD_PARAM;
    // valid in the paper, not built here
    if (p->head_dim != kHeadDim) return QVG_ERR_UNSUPPORTED;
    if (p->n_smooth_stages > kMaxSmooth) return QVG_ERR_UNSUPPORTED;
    const int B = p->group_size;
    if (B != 16 && B != 32 && B != 64 && B != 128) return QVG_ERR_UNSUPPORTED;
    return QVG_OK;
}

// more than 256 centroids: an id is a 16-bit word (2-byte aligned arrays)
inline int id_wide(const qvg_params *p) { return p->n_clusters > 256 ? 1 : 0; }
inline bool ids_aligned(const qvg_params *p, const void *ids) {
    return !id_wide(p) || (reinterpret_cast<uintptr_t>(ids) & 1u) == 0;
}
inline int format_of(const qvg_params *p) {
    return (p->bits == 4 ? kFmtInt4 : 0) | (p->scale_format == QVG_SCALE_E4M3 ? kFmtE4M3 : 0);
}
// scale arrays: binary16 arrays follow the 16-byte rule, E4M3 bytes may start anywhere
inline bool scales_aligned(const qvg_params *p, const void *sc) {
    return p->scale_format == QVG_SCALE_E4M3 || aligned16(sc);
}

struct EncodeWs { size_t init_norms, norms; size_t cent[2]; size_t perm; size_t seg; size_t resid[2]; size_t total; };

// with_assign: split norms of the start tables (one per smoothing stage); with_tables: two centroid
// tables for the Lloyd loop and the split norms of the newer one; with_update: the member lists
EncodeWs encode_ws(const qvg_params *p, int64_t N, bool with_assign, bool with_tables, bool with_update = true) {
    EncodeWs w{};
    size_t o = 0;
    const size_t norms = round256((size_t)p->n_heads * k_padded(p->n_clusters) * sizeof(uint2));
    // (one more word per unit than the norms take: the size that callers were told from the start)
    if (with_assign) { w.init_norms = o; o += norms * (size_t)p->n_smooth_stages + round256((size_t)p->n_heads * sizeof(float)); }
    const size_t table = round256((size_t)p->n_heads * p->n_clusters * kHeadDim * sizeof(bf16_t));
    if (with_tables) { w.norms = o; o += norms; w.cent[0] = o; o += table; w.cent[1] = o; o += table; }
    if (with_update) {
        const int64_t block = member_block(p->n_heads, N), n_blocks = N > 0 ? (N + block - 1) / block : 1;
        w.perm = o; o += round256((size_t)p->n_heads * (size_t)(n_blocks * block) * sizeof(uint16_t));
        // (a workspace must serve every call of fewer tokens or units)
        w.seg = o; o += round256((size_t)member_blocks_bound(p->n_heads, N) * (size_t)p->n_clusters * sizeof(uint32_t));
    }
    // bf16 residual tensors that carry the data from one smoothing stage to the next
    if (with_assign && p->n_smooth_stages > 1) {
        const size_t r = round256((size_t)p->n_heads * (size_t)(N > 0 ? N : 1) * kHeadDim * sizeof(bf16_t));
        w.resid[0] = o; o += r;
        if (p->n_smooth_stages > 2) { w.resid[1] = o; o += r; }
    }
    w.total = o;
    return w;
}

MemberLists member_lists(const qvg_params *p, int64_t N, unsigned char *ws, const EncodeWs &w) {
    MemberLists l;
    l.perm = reinterpret_cast<uint16_t *>(ws + w.perm);
    l.seg = reinterpret_cast<uint32_t *>(ws + w.seg);
    l.block = member_block(p->n_heads, N);
    l.n_blocks = (int)((N + l.block - 1) / l.block);
    return l;
}

int check_view(const void *base, int64_t stride_head, int64_t stride_token, int64_t N) {
    if (!aligned16(base)) return QVG_ERR_ALIGN;
    if (stride_token < kHeadDim || (stride_token & 7) || (stride_head & 7)) return QVG_ERR_ALIGN;
    if (stride_head < 0 || (N > 0 && stride_head < stride_token)) return QVG_ERR_BAD_PARAM;
    return QVG_OK;
}

// Whether the start tables and the tables' place in the output share memory.
bool tables_overlap(const qvg_params *p, const void *init, const void *out, int64_t out_stride) {
    const uintptr_t unit = (uintptr_t)p->n_smooth_stages * p->n_clusters * kHeadDim * sizeof(bf16_t);
    const uintptr_t a = reinterpret_cast<uintptr_t>(init), b = reinterpret_cast<uintptr_t>(out);
    return a < b + (uintptr_t)(p->n_heads - 1) * out_stride * sizeof(bf16_t) + unit && b < a + (uintptr_t)p->n_heads * unit;
}

// wanted: how many workgroups a unit's first barrier waits for in the one-launch form, 0: all
int encode_call(const qvg_params *p, int64_t n_tokens, const void *x, int64_t stride_head,
                int64_t stride_token, const void *init_centroids, void *centroids_out,
                int64_t cent_out_stride_head, uint8_t *ids_out, uint8_t *codes_out,
                void *scales_out, int64_t out_stride_head_tokens, void *workspace,
                size_t workspace_bytes, int wanted, void *stream) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (n_tokens < 0 || n_tokens > kMaxTokensPerChunk) return QVG_ERR_BAD_PARAM;
    if (!init_centroids || !centroids_out) return QVG_ERR_NULL;
    if (!aligned16(init_centroids) || !aligned16(centroids_out)) return QVG_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const size_t row = (size_t)p->n_clusters * kHeadDim * sizeof(bf16_t);    // one unit's table
    if (cent_out_stride_head == 0) cent_out_stride_head = (int64_t)p->n_smooth_stages * p->n_clusters * kHeadDim;
    if (out_stride_head_tokens == 0) out_stride_head_tokens = n_tokens;
    if (cent_out_stride_head < (int64_t)p->n_smooth_stages * p->n_clusters * kHeadDim || (cent_out_stride_head & 7))
        return QVG_ERR_ALIGN;
    if (out_stride_head_tokens < n_tokens) return QVG_ERR_BAD_PARAM;
    // n_tokens == 0: the start tables go out unchanged, H rows of S*K*d bf16 with the caller's pitch
    auto copy_out = [&](const void *src) -> int {
        const size_t all = row * (size_t)p->n_smooth_stages;
        if (src == centroids_out && cent_out_stride_head == (int64_t)p->n_smooth_stages * p->n_clusters * kHeadDim) return QVG_OK;
        return hipMemcpy2DAsync(centroids_out, (size_t)cent_out_stride_head * sizeof(bf16_t), src, all, all,
                                (size_t)p->n_heads, hipMemcpyDeviceToDevice, s) == hipSuccess
                   ? QVG_OK : QVG_ERR_LAUNCH;
    };
    if (n_tokens == 0) return copy_out(init_centroids);
    if (!x || !ids_out || !codes_out || !scales_out) return QVG_ERR_NULL;
    if ((st = check_view(x, stride_head, stride_token, n_tokens)) != QVG_OK) return st;
    if (!aligned16(codes_out) || !scales_aligned(p, scales_out) || !ids_aligned(p, ids_out)) return QVG_ERR_ALIGN;
    const int I = p->kmeans_iters;
    const int fmt = format_of(p);
    const int S = p->n_smooth_stages;
    const EncodeWs w = encode_ws(p, n_tokens, true, I > 0, I > 0);
    if (!workspace || workspace_bytes < w.total) return QVG_ERR_WORKSPACE;
    if (!aligned16(workspace)) return QVG_ERR_ALIGN;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    const int64_t table = (int64_t)p->n_clusters * kHeadDim, kpad = k_padded(p->n_clusters);
    // small enough that all its workgroups run at the same time: one launch for all iterations and stages (its start
    // tables must outlast the first results)
    const int groups = tables_overlap(p, init_centroids, centroids_out, cent_out_stride_head) ? 0
                           : lloyd_groups(p->n_heads, p->n_clusters, n_tokens, stride_token, I);
    if (groups > 0) {
        LloydArgs l{};
        l.x = static_cast<const bf16_t *>(x); l.stride_head = stride_head; l.stride_token = stride_token;
        l.n_tokens = (int)n_tokens; l.init = static_cast<const bf16_t *>(init_centroids);
        l.H = p->n_heads; l.K = p->n_clusters; l.B = p->group_size; l.T = p->n_stages; l.S = S; l.iters = I;
        l.cent_out = static_cast<bf16_t *>(centroids_out); l.cent_out_stride = cent_out_stride_head;
        l.ids = ids_out; l.codes = codes_out; l.scales = scales_out;
        l.codes_stride = out_stride_head_tokens * p->n_stages * (kHeadDim * p->bits / 8);
        l.out_stride = out_stride_head_tokens; l.id_wide = id_wide(p);
        l.fmt = fmt; l.fused = lloyd_fuses(fmt, p->group_size, p->n_stages);
        l.init_norms = reinterpret_cast<const uint2 *>(ws + w.init_norms);
        l.meet = reinterpret_cast<uint32_t *>(ws + w.cent[1]);           // 256 bytes per unit; a table has at least one row
        l.ids_x = reinterpret_cast<uint16_t *>(ws + w.perm);
        l.table = reinterpret_cast<bf16_t *>(ws + w.cent[0]); l.norms = reinterpret_cast<uint2 *>(ws + w.norms);
        for (int i = 0; i < 2; ++i) l.resid[i] = reinterpret_cast<bf16_t *>(ws + w.resid[i]);
        l.n_blocks = (int)((n_tokens + 255) / 256); l.groups = groups;
        l.wanted = wanted > 0 ? wanted : groups;
        if (launch_lloyd(l, s) != hipSuccess) return QVG_ERR_LAUNCH;
        if (l.fused) return QVG_OK;
        QuantArgs q{};
        q.x = l.x; q.stride_head = stride_head; q.stride_token = stride_token;
        if (S > 1) { q.x = l.resid[S & 1]; q.stride_head = n_tokens * kHeadDim; q.stride_token = kHeadDim; }   // stage S - 2 left it
        q.n_tokens = n_tokens; q.cent = static_cast<const bf16_t *>(centroids_out) + (S - 1) * table; q.cent_stride = cent_out_stride_head;
        q.ids = ids_out; q.ids_step = S; q.ids_off = S - 1; q.codes = codes_out; q.scales = scales_out;
        q.out_stride = out_stride_head_tokens; q.H = p->n_heads; q.K = p->n_clusters; q.B = p->group_size;
        q.T = p->n_stages; q.fmt = fmt; q.id_wide = id_wide(p);
        return launch_quantize(q, s) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
    }
    // every stage's start table is known: one launch takes all their norms (none for a small call)
    uint2 *init_norms = assign_takes_norms(p->n_heads, p->n_clusters, n_tokens, I == 0 && S == 1 && fmt == 0) ? nullptr : reinterpret_cast<uint2 *>(ws + w.init_norms);
    if (init_norms && launch_half_norms(static_cast<const bf16_t *>(init_centroids), S * table, p->n_heads, S, p->n_clusters, init_norms, s) != hipSuccess)
        return QVG_ERR_LAUNCH;
    // input of the current smoothing stage: the caller's view first, then dense residual tensors
    const bf16_t *xin = static_cast<const bf16_t *>(x);
    int64_t sh = stride_head, stt = stride_token;
    for (int stage = 0; stage < S; ++stage) {
        AssignArgs a{};
        a.x = xin; a.stride_head = sh; a.stride_token = stt;
        a.n_tokens = n_tokens; a.H = p->n_heads; a.K = p->n_clusters; a.B = p->group_size;
        a.T = p->n_stages; a.ids = ids_out; a.out_stride = out_stride_head_tokens; a.fused = 0;
        a.ids_step = S; a.ids_off = stage; a.id_wide = id_wide(p);
        // the caller's start tables are [H][S][K][d], the Lloyd loop's are dense
        a.cent = static_cast<const bf16_t *>(init_centroids) + stage * table; a.cent_stride = S * table;
        if (init_norms) { a.nh3 = init_norms + stage * kpad; a.nh3_stride = S * kpad; }
        bf16_t *buf[2] = {reinterpret_cast<bf16_t *>(ws + w.cent[0]), reinterpret_cast<bf16_t *>(ws + w.cent[1])};
        if (I > 0) {
            UpdateArgs u{};
            u.x = a.x; u.stride_head = sh; u.stride_token = stt; u.n_tokens = n_tokens;
            u.counts_out = nullptr; u.H = p->n_heads; u.K = p->n_clusters;
            u.lists = member_lists(p, n_tokens, ws, w); u.stage = stage;
            u.nh3 = reinterpret_cast<uint2 *>(ws + w.norms);
            for (int it = 0; it < I; ++it) {
                a.lists = u.lists;
                if (launch_assign(a, s) != hipSuccess) return QVG_ERR_LAUNCH;
                u.cent_prev = a.cent; u.prev_stride = a.cent_stride; u.cent_out = buf[it & 1];
                if (launch_update(u, s) != hipSuccess) return QVG_ERR_LAUNCH;
                a.cent = u.cent_out; a.cent_stride = table;
                a.nh3 = u.nh3; a.nh3_stride = kpad;
            }
            a.lists = MemberLists{};
        }
        // this stage's table goes out as H rows of K*d bf16 with the caller's pitch: the stage's
        // last assignment writes them while it stages the table (no copy of its own)
        bf16_t *cdst = static_cast<bf16_t *>(centroids_out) + stage * table;
        if (!(a.cent == cdst && a.cent_stride == cent_out_stride_head)) {
            a.cent_copy = cdst; a.cent_copy_stride = cent_out_stride_head;
        }
        if (stage + 1 < S) {
            // final assignment of this stage; the bf16 residual it leaves is the next stage's input
            a.resid = reinterpret_cast<bf16_t *>(ws + w.resid[stage & 1]);
            if (launch_assign(a, s) != hipSuccess) return QVG_ERR_LAUNCH;
            xin = a.resid; sh = n_tokens * kHeadDim; stt = kHeadDim;
        } else if (fmt == 0) {
            a.codes = codes_out; a.scales = static_cast<f16_t *>(scales_out); a.fused = 1;
            if (launch_assign(a, s) != hipSuccess) return QVG_ERR_LAUNCH;
        } else {
            // the other stored formats: assignment, then the quantization kernel
            if (launch_assign(a, s) != hipSuccess) return QVG_ERR_LAUNCH;
            QuantArgs q{};
            q.x = xin; q.stride_head = sh; q.stride_token = stt; q.n_tokens = n_tokens;
            q.cent = a.cent; q.cent_stride = a.cent_stride;
            q.ids = ids_out; q.ids_step = S; q.ids_off = stage; q.codes = codes_out; q.scales = scales_out;
            q.out_stride = out_stride_head_tokens; q.H = p->n_heads; q.K = p->n_clusters; q.B = p->group_size;
            q.T = p->n_stages; q.fmt = fmt; q.id_wide = id_wide(p);
            if (launch_quantize(q, s) != hipSuccess) return QVG_ERR_LAUNCH;
        }
    }
    return QVG_OK;
}

}  // namespace

extern "C" {

int qvg_version(void) { return 100; }

const char *qvg_status_string(int status) {
    switch (status) {
        case QVG_OK: return "ok";
        case QVG_ERR_NULL: return "a required pointer is NULL";
        case QVG_ERR_BAD_PARAM: return "a size or parameter is out of range";
        case QVG_ERR_UNSUPPORTED: return "parameter combination not built (head_dim 128, up to 4 smoothing stages, group 16/32/64/128)";
        case QVG_ERR_WORKSPACE: return "workspace missing or too small";
        case QVG_ERR_ALIGN: return "pointer not 16-byte aligned or stride not a multiple of 8 elements";
        case QVG_ERR_LAUNCH: return "HIP runtime error while enqueuing";
        case QVG_ERR_SCRATCH_LIMIT: return "the call needs more scratch memory than the library's static buffer holds";
        default: return "unknown status";
    }
}

int qvg_workspace_bytes(const qvg_params *p, int which_entry, int64_t n_tokens, int64_t n_q,
                        size_t *out) {
    if (!out) return QVG_ERR_NULL;
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (n_tokens < 0 || n_q < 0) return QVG_ERR_BAD_PARAM;
    switch (which_entry) {
        case QVG_ENTRY_ENCODE:
            *out = n_tokens == 0 ? 0 : encode_ws(p, n_tokens, true, p->kmeans_iters > 0,
                                                 p->kmeans_iters > 0).total;   // same call as qvg_encode_chunk
            return QVG_OK;
        case QVG_ENTRY_KMEANS_UPDATE:
            *out = encode_ws(p, n_tokens, false, false).total;
            return QVG_OK;
        case QVG_ENTRY_KMEANS_ASSIGN:
            *out = n_tokens == 0 ? 0 : encode_ws(p, n_tokens, true, false, false).total;
            return QVG_OK;
        case QVG_ENTRY_DECODE:
            *out = 0;
            return QVG_OK;
        case QVG_ENTRY_ATTN:
            // optional: the queries' running state + the decoded tiles of n_tokens tokens (whole
            // chunks, each counted as a multiple of 64 tokens)
            *out = attn_slab_state_bytes(p->n_heads, n_q) + attn_slab_chunk_bytes(p->n_heads, n_tokens);
            return QVG_OK;
        default:
            return QVG_ERR_BAD_PARAM;
    }
}

int64_t qvg_compressed_bytes(const qvg_params *p, int64_t n_tokens) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (n_tokens < 0) return QVG_ERR_BAD_PARAM;
    const int64_t d = p->head_dim, T = p->n_stages;
    const int64_t S = p->n_smooth_stages;
    const int64_t scale_bytes = p->scale_format == QVG_SCALE_E4M3 ? 1 : 2;
    const int64_t per_token = T * (d * p->bits / 8 + scale_bytes * (d / p->group_size)) + S * (id_wide(p) ? 2 : 1);
    return (int64_t)p->n_heads * (n_tokens * per_token + S * (int64_t)p->n_clusters * d * 2);
}

int qvg_kmeans_assign(const qvg_params *p, int64_t n_tokens, const void *x, int64_t stride_head,
                      int64_t stride_token, const void *centroids, uint8_t *ids_out, void *workspace,
                      size_t workspace_bytes, void *stream) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (n_tokens < 0 || n_tokens > kMaxTokensPerChunk) return QVG_ERR_BAD_PARAM;
    if (n_tokens == 0) return QVG_OK;
    if (!x || !centroids || !ids_out) return QVG_ERR_NULL;
    if ((st = check_view(x, stride_head, stride_token, n_tokens)) != QVG_OK) return st;
    if (!aligned16(centroids) || !ids_aligned(p, ids_out)) return QVG_ERR_ALIGN;
    const EncodeWs w = encode_ws(p, n_tokens, true, false, false);
    if (!workspace || workspace_bytes < w.total) return QVG_ERR_WORKSPACE;
    if (!aligned16(workspace)) return QVG_ERR_ALIGN;
    AssignArgs a{};
    const int64_t table = (int64_t)p->n_clusters * kHeadDim;
    uint2 *nh3 = assign_takes_norms(p->n_heads, p->n_clusters, n_tokens, false) ? nullptr
                     : reinterpret_cast<uint2 *>(static_cast<unsigned char *>(workspace) + w.init_norms);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (nh3 && launch_half_norms(static_cast<const bf16_t *>(centroids), table, p->n_heads, 1, p->n_clusters, nh3, s) != hipSuccess)
        return QVG_ERR_LAUNCH;
    a.nh3 = nh3; a.nh3_stride = k_padded(p->n_clusters);
    a.x = static_cast<const bf16_t *>(x); a.stride_head = stride_head; a.stride_token = stride_token;
    a.n_tokens = n_tokens; a.cent = static_cast<const bf16_t *>(centroids); a.cent_stride = table;
    a.H = p->n_heads; a.K = p->n_clusters; a.B = p->group_size; a.T = p->n_stages;
    a.ids = ids_out; a.codes = nullptr; a.scales = nullptr; a.out_stride = n_tokens; a.fused = 0;
    a.ids_step = 1; a.ids_off = 0; a.id_wide = id_wide(p);
    return launch_assign(a, s) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_kmeans_update(const qvg_params *p, int64_t n_tokens, const void *x, int64_t stride_head,
                      int64_t stride_token, const uint8_t *ids, const void *cent_prev,
                      void *cent_out, int32_t *counts_out, void *workspace, size_t workspace_bytes,
                      void *stream) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (n_tokens < 0 || n_tokens > kMaxTokensPerChunk) return QVG_ERR_BAD_PARAM;
    if (!cent_prev || !cent_out) return QVG_ERR_NULL;
    if (n_tokens > 0 && (!x || !ids)) return QVG_ERR_NULL;
    if (n_tokens > 0 && (st = check_view(x, stride_head, stride_token, n_tokens)) != QVG_OK) return st;
    if (!aligned16(cent_prev) || !aligned16(cent_out) || !ids_aligned(p, ids)) return QVG_ERR_ALIGN;
    const EncodeWs w = encode_ws(p, n_tokens, false, false);
    if (!workspace || workspace_bytes < w.total) return QVG_ERR_WORKSPACE;
    if (!aligned16(workspace)) return QVG_ERR_ALIGN;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    UpdateArgs u{};
    u.x = static_cast<const bf16_t *>(x); u.stride_head = stride_head; u.stride_token = stride_token;
    u.n_tokens = n_tokens; u.lists = member_lists(p, n_tokens, ws, w);
    u.cent_prev = static_cast<const bf16_t *>(cent_prev); u.prev_stride = (int64_t)p->n_clusters * kHeadDim;
    u.cent_out = static_cast<bf16_t *>(cent_out); u.counts_out = counts_out;
    u.H = p->n_heads; u.K = p->n_clusters;
    if (launch_member_lists(ids, n_tokens, n_tokens, p->n_heads, p->n_clusters, id_wide(p), u.lists, s) != hipSuccess)
        return QVG_ERR_LAUNCH;
    return launch_update(u, s) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_encode_chunk(const qvg_params *p, int64_t n_tokens, const void *x, int64_t stride_head,
                     int64_t stride_token, const void *init_centroids, void *centroids_out,
                     int64_t cent_out_stride_head, uint8_t *ids_out, uint8_t *codes_out,
                     void *scales_out, int64_t out_stride_head_tokens, void *workspace,
                     size_t workspace_bytes, void *stream) {
    return encode_call(p, n_tokens, x, stride_head, stride_token, init_centroids, centroids_out, cent_out_stride_head, ids_out,
                       codes_out, scales_out, out_stride_head_tokens, workspace, workspace_bytes, 0, stream);
}

// qvg_encode_chunk with another number of workgroups that the one-launch encoder's units wait for, so that a test reaches
// the teams of a busy chip: up to a unit's workgroups, those that come first do the unit (0: one alone); beyond them, the wait for
// more ends by the clock.  Not part of the interface.
int qvg_encode_chunk_wait(const qvg_params *p, int64_t n_tokens, const void *x, int64_t stride_head,
                          int64_t stride_token, const void *init_centroids, void *centroids_out,
                          int64_t cent_out_stride_head, uint8_t *ids_out, uint8_t *codes_out,
                          void *scales_out, int64_t out_stride_head_tokens, void *workspace,
                          size_t workspace_bytes, void *stream, uint32_t wanted) {
    return encode_call(p, n_tokens, x, stride_head, stride_token, init_centroids, centroids_out, cent_out_stride_head, ids_out,
                       codes_out, scales_out, out_stride_head_tokens, workspace, workspace_bytes, wanted > 0 ? (int)wanted : 1, stream);
}

}  // extern "C"

// ---- scratch memory owned by the library, for qvg_encode_chunk_static -------------------------
// One array per GPU the library's code object is loaded on (each device has its own copy at its
// own address), alive until the process ends.  The name below is only a handle on the host: the
// device address comes from hipGetSymbolAddress, once per device, and only that address is ever
// passed to a kernel or a copy.
constexpr size_t kStaticArrayBytes = (size_t)48 << 20;
static __device__ __align__(256) unsigned char scratch[kStaticArrayBytes];

namespace {
// The bytes that QVG_STATIC_SCRATCH_BYTES limits (see the header): what a call is accepted by stays
// the same when the workspace's layout changes.  The layout in use takes more per token (the member lists) and per
// stage (the norms): at most 43 MB over the sizes that the rule accepts.
size_t static_rule_bytes(const qvg_params *p, int64_t N) {
    const size_t H = (size_t)p->n_heads, K = (size_t)p->n_clusters, n = (size_t)(N > 0 ? N : 1);
    size_t o = round256(H * k_padded(p->n_clusters) * 8) + round256(H * 4);
    if (p->kmeans_iters > 0 || p->n_smooth_stages > 1) o += 2 * round256(H * K * kHeadDim * 2);
    if (p->kmeans_iters > 0) o += round256(H * n * 4) + round256(H * (K + 1) * 4);
    const int resid = p->n_smooth_stages > 2 ? 2 : p->n_smooth_stages - 1;
    return o + resid * round256(H * n * kHeadDim * 2);
}
constexpr int kMaxDevices = 64;
// device address of `scratch` on the current device (looked up on the first call on that device)
int static_scratch_address(void **out) {
    static std::mutex mu;
    static void *address[kMaxDevices] = {};
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return QVG_ERR_LAUNCH;
    if (dev < 0 || dev >= kMaxDevices) return QVG_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lock(mu);
    if (!address[dev]) {
        void *ptr = nullptr;
        if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)) != hipSuccess || !ptr) return QVG_ERR_LAUNCH;
        address[dev] = ptr;
    }
    *out = address[dev];
    return QVG_OK;
}
}  // namespace

extern "C" {

int qvg_encode_chunk_static(const qvg_params *p, int64_t n_tokens, const void *x, int64_t stride_head,
                            int64_t stride_token, const void *init_centroids, void *centroids_out,
                            int64_t cent_out_stride_head, uint8_t *ids_out, uint8_t *codes_out,
                            void *scales_out, int64_t out_stride_head_tokens, void *stream) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (n_tokens < 0 || n_tokens > kMaxTokensPerChunk) return QVG_ERR_BAD_PARAM;
    // the same workspace layout as qvg_encode_chunk, placed in the static array
    const size_t need = n_tokens == 0 ? 0 : encode_ws(p, n_tokens, true, p->kmeans_iters > 0,
                                                      p->kmeans_iters > 0).total;
    if (need > 0 && static_rule_bytes(p, n_tokens) > (size_t)QVG_STATIC_SCRATCH_BYTES) return QVG_ERR_SCRATCH_LIMIT;
    if (need > kStaticArrayBytes) return QVG_ERR_SCRATCH_LIMIT;
    void *ws = nullptr;
    if (need > 0 && (st = static_scratch_address(&ws)) != QVG_OK) return st;
    // nothing in the workspace has to start at zero: every kernel writes what it later reads
    return qvg_encode_chunk(p, n_tokens, x, stride_head, stride_token, init_centroids, centroids_out,
                            cent_out_stride_head, ids_out, codes_out, scales_out, out_stride_head_tokens,
                            need > 0 ? ws : nullptr, need, stream);
}

int qvg_decode(const qvg_params *p, int64_t n_tokens, int64_t chunk_len, const void *centroids,
               const uint8_t *ids, const uint8_t *codes, const void *scales, void *x_out,
               int64_t stride_head, int64_t stride_token, void *stream) {
    return qvg_decode_ex(p, n_tokens, chunk_len, 0, 0, centroids, ids, codes, scales, x_out, stride_head,
                         stride_token, stream);
}

int qvg_decode_ex(const qvg_params *p, int64_t n_tokens, int64_t chunk_len, int64_t kv_capacity_tokens,
                  int64_t first_token, const void *centroids, const uint8_t *ids, const uint8_t *codes,
                  const void *scales, void *x_out, int64_t stride_head, int64_t stride_token,
                  void *stream) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (n_tokens < 0 || n_tokens > 0x7fffffff || chunk_len < 1) return QVG_ERR_BAD_PARAM;
    if (first_token < 0 || first_token % chunk_len != 0) return QVG_ERR_BAD_PARAM;
    if (kv_capacity_tokens == 0) kv_capacity_tokens = first_token + n_tokens;
    if (kv_capacity_tokens < first_token + n_tokens) return QVG_ERR_BAD_PARAM;
    const int64_t cap_chunks = chunk_count(kv_capacity_tokens, chunk_len);
    if (cap_chunks > 0x7fffffff) return QVG_ERR_BAD_PARAM;
    if (n_tokens == 0) return QVG_OK;
    if (!centroids || !ids || !codes || !scales || !x_out) return QVG_ERR_NULL;
    if ((st = check_view(x_out, stride_head, stride_token, n_tokens)) != QVG_OK) return st;
    if (!aligned16(centroids) || !aligned16(codes) || !scales_aligned(p, scales) || !ids_aligned(p, ids)) return QVG_ERR_ALIGN;
    const int64_t n_chunks = chunk_count(n_tokens, chunk_len);
    if (n_chunks > 0x7fffffff) return QVG_ERR_BAD_PARAM;
    DecodeArgs a{};
    // the range starts on a chunk boundary: move the unit-0 pointers to it, keep the unit strides
    const int64_t S_ = p->n_smooth_stages, T_ = p->n_stages, G_ = p->head_dim / p->group_size;
    a.cent = static_cast<const bf16_t *>(centroids) + (first_token / chunk_len) * S_ * p->n_clusters * kHeadDim;
    a.ids = ids + first_token * S_ * (id_wide(p) ? 2 : 1);
    a.id_wide = id_wide(p);
    a.codes = codes + first_token * T_ * (kHeadDim * p->bits / 8);
    a.scales = reinterpret_cast<const f16_t *>(static_cast<const uint8_t *>(scales) +
                                               first_token * T_ * G_ * (p->scale_format == QVG_SCALE_E4M3 ? 1 : 2));
    a.out = static_cast<bf16_t *>(x_out);
    a.kv_stride = kv_capacity_tokens; a.chunk_stride = (int)cap_chunks;
    a.n_tokens = n_tokens; a.chunk_len = bounded_chunk_len(chunk_len); a.n_chunks = (int)n_chunks;
    a.H = p->n_heads; a.K = p->n_clusters; a.B = p->group_size; a.T = p->n_stages;
    a.stride_head = stride_head; a.stride_token = stride_token; a.S = p->n_smooth_stages; a.fmt = format_of(p);
    return launch_decode(a, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_attn_decode(const qvg_params *p, int64_t n_q, const void *q, int64_t n_kv_tokens,
                    int64_t chunk_len, const void *k_centroids, const uint8_t *k_ids,
                    const uint8_t *k_codes, const void *k_scales, const void *v_centroids,
                    const uint8_t *v_ids, const uint8_t *v_codes, const void *v_scales,
                    float softmax_scale, void *out, float *lse_out, void *workspace,
                    size_t workspace_bytes, void *stream) {
    return qvg_attn_decode_ex(p, n_q, q, n_kv_tokens, chunk_len, 0, k_centroids, k_ids, k_codes, k_scales,
                              v_centroids, v_ids, v_codes, v_scales, nullptr, softmax_scale, out, lse_out,
                              workspace, workspace_bytes, stream);
}

int qvg_attn_merge(int64_t n_rows, int32_t head_dim, const void *out_a, const float *lse_a,
                   const void *out_b, const float *lse_b, void *out, float *lse_out, void *stream) {
    if (n_rows < 0) return QVG_ERR_BAD_PARAM;
    if (head_dim != kHeadDim) return QVG_ERR_UNSUPPORTED;
    if (n_rows == 0) return QVG_OK;
    if (!out_a || !lse_a || !out_b || !lse_b || !out) return QVG_ERR_NULL;
    if (!aligned16(out_a) || !aligned16(out_b) || !aligned16(out)) return QVG_ERR_ALIGN;
    MergeArgs m{};
    m.oa = static_cast<const bf16_t *>(out_a); m.lsea = lse_a; m.ob = static_cast<const bf16_t *>(out_b);
    m.lseb = lse_b; m.out = static_cast<bf16_t *>(out); m.lse = lse_out; m.rows = n_rows;
    return launch_attn_merge(m, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_attn_decode_ex(const qvg_params *p, int64_t n_q, const void *q, int64_t n_kv_tokens,
                       int64_t chunk_len, int64_t kv_capacity_tokens, const void *k_centroids,
                       const uint8_t *k_ids, const uint8_t *k_codes, const void *k_scales,
                       const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                       const void *v_scales, const void *k_rope, float softmax_scale, void *out,
                       float *lse_out, void *workspace, size_t workspace_bytes, void *stream) {
    return qvg_attn_decode_causal(p, n_q, q, n_kv_tokens, chunk_len, kv_capacity_tokens, k_centroids, k_ids, k_codes,
                                  k_scales, v_centroids, v_ids, v_codes, v_scales, k_rope, nullptr, softmax_scale, out,
                                  lse_out, workspace, workspace_bytes, stream);
}

}  // extern "C"

namespace {
// the one implementation behind every attention entry point; exactly one of out / out_f32 is set
int attn_call(const qvg_params *p, int64_t n_q, const void *q, int64_t n_kv_tokens,
              int64_t chunk_len, int64_t kv_capacity_tokens, const void *k_centroids,
              const uint8_t *k_ids, const uint8_t *k_codes, const void *k_scales,
              const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
              const void *v_scales, const void *k_rope, const int32_t *q_kv_len,
              float softmax_scale, void *out, float *out_f32, float *lse_out, void *workspace,
              size_t workspace_bytes, void *scratch, size_t scratch_bytes, void *stream) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (n_q < 0 || n_kv_tokens < 1 || n_kv_tokens > 0x7fffffff || chunk_len < 1) return QVG_ERR_BAD_PARAM;
    if (!(softmax_scale > 0.0f) || softmax_scale - softmax_scale != 0.0f) return QVG_ERR_BAD_PARAM;   // positive, finite
    if (n_q == 0) return QVG_OK;
    if (!q || (!out && !out_f32) || !k_centroids || !k_ids || !k_codes || !k_scales || !v_centroids || !v_ids ||
        !v_codes || !v_scales)
        return QVG_ERR_NULL;
    if (!aligned16(q) || !aligned16(out) || !aligned16(out_f32) || !aligned16(k_centroids) || !aligned16(v_centroids) ||
        !aligned16(k_codes) || !aligned16(v_codes) || !scales_aligned(p, k_scales) || !scales_aligned(p, v_scales))
        return QVG_ERR_ALIGN;
    const int64_t n_chunks = chunk_count(n_kv_tokens, chunk_len);
    if (n_chunks > 0x7fffffff) return QVG_ERR_BAD_PARAM;
    if ((n_q + 127) / 128 > 0x7fffffff) return QVG_ERR_BAD_PARAM;
    if (kv_capacity_tokens == 0) kv_capacity_tokens = n_kv_tokens;
    if (kv_capacity_tokens < n_kv_tokens) return QVG_ERR_BAD_PARAM;
    const int64_t cap_chunks = chunk_count(kv_capacity_tokens, chunk_len);
    if (cap_chunks > 0x7fffffff) return QVG_ERR_BAD_PARAM;
    if (k_rope && !aligned16(k_rope)) return QVG_ERR_ALIGN;
    AttnArgs a{};
    a.q = static_cast<const bf16_t *>(q); a.out = static_cast<bf16_t *>(out); a.out_f32 = out_f32; a.lse = lse_out;
    a.n_q = n_q; a.n_kv = n_kv_tokens; a.chunk_len = bounded_chunk_len(chunk_len); a.n_chunks = (int)n_chunks;
    a.H = p->n_heads; a.K = p->n_clusters; a.B = p->group_size; a.T = p->n_stages;
    a.scale = softmax_scale;
    a.k_cent = static_cast<const bf16_t *>(k_centroids); a.k_ids = k_ids; a.k_codes = k_codes;
    a.k_scales = static_cast<const f16_t *>(k_scales);
    a.v_cent = static_cast<const bf16_t *>(v_centroids); a.v_ids = v_ids; a.v_codes = v_codes;
    a.v_scales = static_cast<const f16_t *>(v_scales);
    a.S = p->n_smooth_stages; a.fmt = format_of(p);
    a.kv_stride = kv_capacity_tokens; a.chunk_stride = (int)cap_chunks;
    a.rope = static_cast<const f16_t *>(k_rope);
    a.id_wide = id_wide(p);
    if (!ids_aligned(p, k_ids) || !ids_aligned(p, v_ids)) return QVG_ERR_ALIGN;
    if (q_kv_len && (reinterpret_cast<uintptr_t>(q_kv_len) & 3u)) return QVG_ERR_ALIGN;
    a.q_len = q_kv_len;
    // (without room for parts every workgroup walks the whole cache)
    const bool unaligned = !aligned16(scratch);
    const AttnParts parts = attn_parts(a.H, n_q, n_kv_tokens, a.chunk_len, q_kv_len != nullptr, scratch && !unaligned ? scratch_bytes : 0);
    if (unaligned && parts.aligned && scratch_bytes >= attn_state_bytes(a.H, n_q, AttnParts{parts.aligned, 0, 0, 0})) return QVG_ERR_ALIGN;
    a.parts = parts.parts; a.part_tiles = parts.part_tiles; a.whole = parts.whole;
    if (a.parts > 1) a.part_state = static_cast<float *>(scratch);
    hipStream_t s = static_cast<hipStream_t>(stream);
    // a workspace that holds at least one chunk's decoded tiles switches to the shared-tile path
    if (workspace && attn_slab_applicable(a, workspace, workspace_bytes)) {
        if (!aligned16(workspace)) return QVG_ERR_ALIGN;
        if (launch_attn_slab(a, workspace, workspace_bytes, s) != hipSuccess) return QVG_ERR_LAUNCH;
    } else if (launch_attn(a, s) != hipSuccess) {
        return QVG_ERR_LAUNCH;
    }
    if (a.parts > 1 && launch_attn_join(a, s) != hipSuccess) return QVG_ERR_LAUNCH;
    return QVG_OK;
}
}  // namespace

extern "C" {

int qvg_attn_decode_causal(const qvg_params *p, int64_t n_q, const void *q, int64_t n_kv_tokens,
                           int64_t chunk_len, int64_t kv_capacity_tokens, const void *k_centroids,
                           const uint8_t *k_ids, const uint8_t *k_codes, const void *k_scales,
                           const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                           const void *v_scales, const void *k_rope, const int32_t *q_kv_len,
                           float softmax_scale, void *out, float *lse_out, void *workspace,
                           size_t workspace_bytes, void *stream) {
    return attn_call(p, n_q, q, n_kv_tokens, chunk_len, kv_capacity_tokens, k_centroids, k_ids, k_codes, k_scales,
                     v_centroids, v_ids, v_codes, v_scales, k_rope, q_kv_len, softmax_scale, out, nullptr, lse_out,
                     workspace, workspace_bytes, nullptr, 0, stream);
}

int qvg_attn_scratch_bytes(const qvg_params *p, int64_t n_q, int64_t n_kv_tokens, int64_t chunk_len, size_t *out) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (!out) return QVG_ERR_NULL;
    if (n_q < 0 || n_kv_tokens < 1 || n_kv_tokens > 0x7fffffff || chunk_len < 1) return QVG_ERR_BAD_PARAM;
    *out = attn_state_bytes(p->n_heads, n_q, attn_parts(p->n_heads, n_q, n_kv_tokens, bounded_chunk_len(chunk_len), false));
    return QVG_OK;
}

int qvg_attn_scratch_bytes_causal(const qvg_params *p, int64_t n_q, int64_t n_kv_tokens, int64_t chunk_len, size_t *out) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (!out) return QVG_ERR_NULL;
    if (n_q < 0 || n_kv_tokens < 1 || n_kv_tokens > 0x7fffffff || chunk_len < 1) return QVG_ERR_BAD_PARAM;
    *out = attn_state_bytes(p->n_heads, n_q, attn_parts(p->n_heads, n_q, n_kv_tokens, bounded_chunk_len(chunk_len), true));
    return QVG_OK;
}

int qvg_attn_decode_parts(const qvg_params *p, int64_t n_q, const void *q, int64_t n_kv_tokens,
                          int64_t chunk_len, int64_t kv_capacity_tokens, const void *k_centroids,
                          const uint8_t *k_ids, const uint8_t *k_codes, const void *k_scales,
                          const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                          const void *v_scales, const void *k_rope, const int32_t *q_kv_len,
                          float softmax_scale, void *out_bf16, float *out_f32, float *lse_out, void *workspace,
                          size_t workspace_bytes, void *scratch, size_t scratch_bytes, void *stream) {
    if (out_bf16 && out_f32) return QVG_ERR_BAD_PARAM;
    return attn_call(p, n_q, q, n_kv_tokens, chunk_len, kv_capacity_tokens, k_centroids, k_ids, k_codes, k_scales,
                     v_centroids, v_ids, v_codes, v_scales, k_rope, q_kv_len, softmax_scale, out_bf16, out_f32, lse_out,
                     workspace, workspace_bytes, scratch, scratch_bytes, stream);
}

int qvg_attn_decode_f32(const qvg_params *p, int64_t n_q, const void *q, int64_t n_kv_tokens,
                        int64_t chunk_len, int64_t kv_capacity_tokens, const void *k_centroids,
                        const uint8_t *k_ids, const uint8_t *k_codes, const void *k_scales,
                        const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                        const void *v_scales, const void *k_rope, const int32_t *q_kv_len,
                        float softmax_scale, float *out_f32, float *lse_out, void *stream) {
    return attn_call(p, n_q, q, n_kv_tokens, chunk_len, kv_capacity_tokens, k_centroids, k_ids, k_codes, k_scales,
                     v_centroids, v_ids, v_codes, v_scales, k_rope, q_kv_len, softmax_scale, nullptr, out_f32, lse_out,
                     nullptr, 0, nullptr, 0, stream);
}

}  // extern "C"

// ---- paged caches -----------------------------------------------------------------------------
namespace {

// a bf16 view of rows of 128 elements whose strides (in elements) keep every row 16-byte aligned
bool rows_aligned(const void *base, int64_t seq, int64_t head, int64_t row) {
    return aligned16(base) && ((seq | head | row) & 7) == 0;
}
constexpr int64_t kMaxInt = 0x7fffffff;

// the sizes of a step (not its pointers)
int check_step_sizes(const qvg_params *p, const qvg_tree_step *t) {
    if (!t) return QVG_ERR_NULL;
    if (t->n_seqs < 0 || t->n_seqs > 65535 || t->group < 1 || t->n_nodes < 0 || t->table_pages < 0 || t->tail_capacity < 0 || t->reserved != 0)
        return QVG_ERR_BAD_PARAM;
    if ((int64_t)t->group * t->n_nodes > (1 << 20)) return QVG_ERR_BAD_PARAM;
    if (t->page_len < 1 || t->page_len > kMaxInt || t->pool_pages < 1 || t->pool_pages > kMaxInt) return QVG_ERR_BAD_PARAM;
    if (t->table_pages > 0 && t->page_len > kMaxInt / t->table_pages) return QVG_ERR_BAD_PARAM;
    // (tiles of 32 tokens, and blocks of query rows, are counted in 32 bits)
    if ((int64_t)t->table_pages * tree_tiles((int)t->page_len) + tree_tiles(t->tail_capacity) + tree_tiles(t->n_nodes) > kMaxInt - 1024)
        return QVG_ERR_BAD_PARAM;
    const int64_t rows = (int64_t)t->group * t->n_nodes, br = tree_block_rows(rows, false, false);
    if ((int64_t)t->n_seqs * p->n_heads * ((rows + br - 1) / br) > (1 << 30)) return QVG_ERR_BAD_PARAM;
    return QVG_OK;
}

}  // namespace

extern "C" {

int qvg_attn_tree_scratch_bytes(const qvg_params *p, const qvg_tree_step *t, size_t *out) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (!out) return QVG_ERR_NULL;
    if ((st = check_step_sizes(p, t)) != QVG_OK) return st;
    // (with a rotation or without)
    const size_t plain = tree_plan(*p, *t, false).state_bytes, rotated = tree_plan(*p, *t, true).state_bytes;
    *out = plain > rotated ? plain : rotated;
    return QVG_OK;
}

int qvg_attn_tree(const qvg_params *p, const qvg_tree_step *t, const void *k_centroids, const uint8_t *k_ids,
                  const uint8_t *k_codes, const void *k_scales, const void *v_centroids, const uint8_t *v_ids,
                  const uint8_t *v_codes, const void *v_scales, float softmax_scale, void *scratch, size_t scratch_bytes,
                  void *stream) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if ((st = check_step_sizes(p, t)) != QVG_OK) return st;
    if (!(softmax_scale > 0.0f) || softmax_scale - softmax_scale != 0.0f) return QVG_ERR_BAD_PARAM;   // positive, finite
    if (t->k_rope_f16 && t->table_pages > 0 && t->rope_tokens < 1) return QVG_ERR_BAD_PARAM;
    if (t->n_seqs == 0 || t->n_nodes == 0) return QVG_OK;
    if (!t->q || !t->out || !t->k_new || !t->v_new) return QVG_ERR_NULL;
    if (t->table_pages > 0 && (!t->page_table || !t->kv_len || !k_centroids || !k_ids || !k_codes || !k_scales || !v_centroids ||
                               !v_ids || !v_codes || !v_scales))
        return QVG_ERR_NULL;
    if (t->tail_capacity > 0 && (!t->k_tail || !t->v_tail || !t->tail_len)) return QVG_ERR_NULL;
    if (!rows_aligned(t->q, t->q_stride_seq, t->q_stride_head, t->q_stride_node) ||
        !rows_aligned(t->out, t->out_stride_seq, t->out_stride_head, t->out_stride_node) ||
        !rows_aligned(t->k_new, t->new_stride_seq, t->new_stride_head, t->new_stride_node) || !aligned16(t->v_new))
        return QVG_ERR_ALIGN;
    if (t->tail_capacity > 0 && (!rows_aligned(t->k_tail, t->tail_stride_seq, t->tail_stride_head, t->tail_stride_token) || !aligned16(t->v_tail)))
        return QVG_ERR_ALIGN;
    if (t->table_pages > 0 && (!aligned16(k_centroids) || !aligned16(v_centroids) || !aligned16(k_codes) || !aligned16(v_codes) ||
                               !scales_aligned(p, k_scales) || !scales_aligned(p, v_scales) || !ids_aligned(p, k_ids) || !ids_aligned(p, v_ids)))
        return QVG_ERR_ALIGN;
    if (!aligned16(t->k_rope_f16) || !aligned16(scratch)) return QVG_ERR_ALIGN;
    const uintptr_t words = reinterpret_cast<uintptr_t>(t->page_table) | reinterpret_cast<uintptr_t>(t->kv_len) | reinterpret_cast<uintptr_t>(t->tail_len) |
                            reinterpret_cast<uintptr_t>(t->nodes) | reinterpret_cast<uintptr_t>(t->mask) | reinterpret_cast<uintptr_t>(t->lse);
    if (words & 3u) return QVG_ERR_ALIGN;
    TreeArgs a{};
    a.k = PoolSide{static_cast<const bf16_t *>(k_centroids), k_ids, k_codes, static_cast<const uint8_t *>(k_scales)};
    a.v = PoolSide{static_cast<const bf16_t *>(v_centroids), v_ids, v_codes, static_cast<const uint8_t *>(v_scales)};
    a.H = p->n_heads; a.K = p->n_clusters; a.B = p->group_size; a.T = p->n_stages; a.S = p->n_smooth_stages;
    a.fmt = format_of(p); a.id_wide = id_wide(p); a.t = *t; a.scale = softmax_scale;
    const TreePlan plan = tree_plan(*p, *t, t->k_rope_f16 != nullptr);
    a.row_blocks = plan.row_blocks;
    a.rows = plan.rows;
    a.slots = scratch && scratch_bytes >= plan.state_bytes ? plan.slots : 0;
    a.share = plan.share;
    a.state = static_cast<float *>(scratch);
    if (a.slots) a.places = reinterpret_cast<int2 *>(static_cast<char *>(scratch) + plan.state_bytes - (size_t)t->n_seqs * sizeof(int2));
    return launch_attn_tree(a, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_tree_mask(int64_t n_seqs, int64_t n_nodes, const int32_t *parents, const int32_t *nodes, uint32_t *mask_out,
                  int32_t *depth_out, void *stream) {
    if (n_seqs < 0 || n_seqs > kMaxInt || n_nodes < 0 || n_nodes > 1024) return QVG_ERR_BAD_PARAM;
    if (n_seqs == 0 || n_nodes == 0) return QVG_OK;
    if (!parents || !mask_out) return QVG_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(parents) | reinterpret_cast<uintptr_t>(nodes) | reinterpret_cast<uintptr_t>(mask_out) |
         reinterpret_cast<uintptr_t>(depth_out)) & 3u)
        return QVG_ERR_ALIGN;
    return launch_tree_mask((int)n_seqs, (int)n_nodes, parents, nodes, mask_out, depth_out, static_cast<hipStream_t>(stream)) == hipSuccess
               ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_keep_nodes(int32_t n_heads, int32_t head_dim, int64_t n_seqs, int64_t n_nodes, const void *k_new, const void *v_new,
                   int64_t new_stride_seq, int64_t new_stride_head, int64_t new_stride_node, const int32_t *path, int64_t n_path,
                   const int32_t *n_keep, void *k_tail, void *v_tail, int64_t tail_stride_seq, int64_t tail_stride_head,
                   int64_t tail_stride_token, int64_t tail_capacity, const int32_t *tail_len, int32_t *tail_len_out, void *stream) {
    if (n_heads < 1 || n_heads > 65535 || n_seqs < 0 || n_seqs > 65535 || n_nodes < 0 || n_nodes > (1 << 20) || n_path < 0 ||
        n_path > (1 << 20) || tail_capacity < 0 || tail_capacity > kMaxInt)
        return QVG_ERR_BAD_PARAM;
    if (head_dim != kHeadDim) return QVG_ERR_UNSUPPORTED;
    const int64_t blocks = (n_path + 15) / 16;
    if (n_seqs * 2 * n_heads * blocks > kMaxInt) return QVG_ERR_BAD_PARAM;
    if (n_seqs == 0) return QVG_OK;
    if (!n_keep || !tail_len) return QVG_ERR_NULL;
    const bool rows = n_path > 0 && n_nodes > 0 && tail_capacity > 0;
    if (rows && (!k_new || !v_new || !path || !k_tail || !v_tail)) return QVG_ERR_NULL;
    if (rows && (!rows_aligned(k_new, new_stride_seq, new_stride_head, new_stride_node) || !aligned16(v_new) ||
                 !rows_aligned(k_tail, tail_stride_seq, tail_stride_head, tail_stride_token) || !aligned16(v_tail)))
        return QVG_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(path) | reinterpret_cast<uintptr_t>(n_keep) | reinterpret_cast<uintptr_t>(tail_len) |
         reinterpret_cast<uintptr_t>(tail_len_out)) & 3u)
        return QVG_ERR_ALIGN;
    KeepArgs a{};
    a.k_new = static_cast<const bf16_t *>(k_new); a.v_new = static_cast<const bf16_t *>(v_new);
    a.new_seq = new_stride_seq; a.new_head = new_stride_head; a.new_node = new_stride_node;
    a.k_tail = static_cast<bf16_t *>(k_tail); a.v_tail = static_cast<bf16_t *>(v_tail);
    a.tail_seq = tail_stride_seq; a.tail_head = tail_stride_head; a.tail_token = tail_stride_token;
    a.path = path; a.keep = n_keep; a.tail_len = tail_len; a.tail_len_out = tail_len_out;
    a.H = n_heads; a.n_seqs = (int)n_seqs; a.n_nodes = (int)n_nodes; a.n_path = (int)n_path; a.capacity = (int)tail_capacity;
    a.blocks = rows ? (int)blocks : 0;
    const uintptr_t was = reinterpret_cast<uintptr_t>(tail_len), now = reinterpret_cast<uintptr_t>(tail_len_out), size = (uintptr_t)n_seqs * sizeof(int32_t);
    a.lengths_here = rows && tail_len_out && (now >= was + size || was >= now + size);
    return launch_keep_nodes(a, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_copy_pages(const qvg_params *p, int64_t page_len, int64_t n_pairs, const int32_t *src, const int32_t *dst,
                   int64_t src_pool_pages, const void *src_centroids, const uint8_t *src_ids, const uint8_t *src_codes,
                   const void *src_scales, int64_t dst_pool_pages, void *dst_centroids, uint8_t *dst_ids, uint8_t *dst_codes,
                   void *dst_scales, void *stream) {
    int st = check_params(p);
    if (st != QVG_OK) return st;
    if (page_len < 1 || page_len > kMaxInt || n_pairs < 0 || src_pool_pages < 0 || src_pool_pages > kMaxInt || dst_pool_pages < 0 ||
        dst_pool_pages > kMaxInt)
        return QVG_ERR_BAD_PARAM;
    if (n_pairs == 0) return QVG_OK;
    if (n_pairs > dst_pool_pages) return QVG_ERR_BAD_PARAM;              // some destination is named twice
    if (!src || !dst || !src_centroids || !src_ids || !src_codes || !src_scales || !dst_centroids || !dst_ids || !dst_codes || !dst_scales)
        return QVG_ERR_NULL;
    if (!aligned16(src_centroids) || !aligned16(dst_centroids) || !aligned16(src_codes) || !aligned16(dst_codes) ||
        !scales_aligned(p, src_scales) || !scales_aligned(p, dst_scales) || !ids_aligned(p, src_ids) || !ids_aligned(p, dst_ids))
        return QVG_ERR_ALIGN;
    {
        const bool same = src_codes == dst_codes;
        uint8_t *named = new (std::nothrow) uint8_t[(size_t)dst_pool_pages]();      // pages that are written
        if (!named) return QVG_ERR_WORKSPACE;
        bool ok = true;
        for (int64_t i = 0; i < n_pairs && ok; ++i) {
            ok = src[i] >= 0 && src[i] < src_pool_pages && dst[i] >= 0 && dst[i] < dst_pool_pages && !named[dst[i]];
            if (ok) named[dst[i]] = 1;
        }
        for (int64_t i = 0; i < n_pairs && ok && same; ++i) ok = src[i] >= dst_pool_pages || !named[src[i]];
        delete[] named;
        if (!ok) return QVG_ERR_BAD_PARAM;
    }
    const int64_t table = (int64_t)p->n_smooth_stages * p->n_clusters * kHeadDim * (int64_t)sizeof(bf16_t);
    const int64_t per_token[3] = {(int64_t)p->n_smooth_stages * (id_wide(p) ? 2 : 1), (int64_t)p->n_stages * (kHeadDim * p->bits / 8),
                                  (int64_t)p->n_stages * (kHeadDim / p->group_size) * (p->scale_format == QVG_SCALE_E4M3 ? 1 : 2)};
    const uint8_t *from[4] = {static_cast<const uint8_t *>(src_centroids), src_ids, src_codes, static_cast<const uint8_t *>(src_scales)};
    uint8_t *to[4] = {static_cast<uint8_t *>(dst_centroids), dst_ids, dst_codes, static_cast<uint8_t *>(dst_scales)};
    PageArray arrays[4];
    for (int k = 0; k < 4; ++k) {
        const int64_t bytes = k == 0 ? table : per_token[k - 1] * page_len;
        arrays[k] = PageArray{from[k], to[k], bytes, bytes * src_pool_pages, bytes * dst_pool_pages};
    }
    return launch_copy_pages(arrays, p->n_heads, n_pairs, src, dst, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

}  // extern "C"

// ---- rotary positions, caches of 16-bit pages -----------------------------------------------------
namespace {

inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// rows of elements of `size` bytes, strides in elements: every row starts at a multiple of 16 bytes
bool rows_aligned(const void *base, int size, int64_t seq, int64_t head, int64_t row) {
    return aligned16(base) && ((seq | head | row) & (16 / size - 1)) == 0;
}
constexpr int kMaxRow = 512;                       // channels of a row that is turned or put into pages
constexpr int64_t kMaxTokens = (int64_t)1 << 30;   // of a sequence's table of 16-bit pages

int check_rotary(const qvg_rotary *r, int head_dim) {
    if (r->type != QVG_F16 && r->type != QVG_F32) return QVG_ERR_BAD_PARAM;
    if (r->n_pairs < 1 || r->n_pairs > head_dim / 2 || r->n_rows < 1 || r->n_rows > kMaxInt || (r->half != 0 && r->half != 1) || r->reserved != 0)
        return QVG_ERR_BAD_PARAM;
    return QVG_OK;
}
int check_rotary_pointers(const qvg_rotary *r) {
    if (!r->table) return QVG_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(r->table) & (r->type == QVG_F32 ? 7u : 3u)) != 0 || !aligned4(r->positions)) return QVG_ERR_ALIGN;
    return QVG_OK;
}

// the sizes of a cache of 16-bit pages (not its pointers)
int check_cache(const qvg_page_cache *c) {
    if (!c) return QVG_ERR_NULL;
    if (c->type != QVG_BF16 && c->type != QVG_F16) return QVG_ERR_BAD_PARAM;
    if (c->n_seqs < 0 || c->n_seqs > 65535 || c->n_heads < 1 || c->n_heads > 65535 || c->head_dim < 1 || c->table_pages < 0 || c->reserved != 0)
        return QVG_ERR_BAD_PARAM;
    if (c->page_len < 1 || c->page_len > kMaxInt || c->pool_pages < 1 || c->pool_pages > kMaxInt) return QVG_ERR_BAD_PARAM;
    if (c->table_pages > 0 && c->page_len > kMaxTokens / c->table_pages) return QVG_ERR_BAD_PARAM;
    if (c->stride_token < 0 || c->stride_token > (1 << 24)) return QVG_ERR_BAD_PARAM;
    return QVG_OK;
}
int check_cache_pointers(const qvg_page_cache *c) {
    if (!c->kv_len || (c->table_pages > 0 && (!c->page_table || !c->k_pages || !c->v_pages))) return QVG_ERR_NULL;
    if (c->table_pages > 0 && (!rows_aligned(c->k_pages, 2, c->stride_head, c->stride_page, c->stride_token) || !aligned16(c->v_pages)))
        return QVG_ERR_ALIGN;
    return aligned4(c->page_table) && aligned4(c->kv_len) ? QVG_OK : QVG_ERR_ALIGN;
}
int check_page_step(const qvg_page_cache *c, const qvg_page_step *t) {
    int st = check_cache(c);
    if (st != QVG_OK) return st;
    if (!t) return QVG_ERR_NULL;
    if (t->group < 1 || t->n_new < 0 || (int64_t)t->group * t->n_new > (1 << 20) || (t->causal != 0 && t->causal != 1) || t->window < 0 ||
        t->sink < 0 || t->reserved != 0)
        return QVG_ERR_BAD_PARAM;
    if (!page_attn_dim(c->head_dim)) return QVG_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)t->group * t->n_new;
    if ((int64_t)c->n_seqs * c->n_heads * ((rows + 31) / 32) > (1 << 23)) return QVG_ERR_BAD_PARAM;
    return QVG_OK;
}

}  // namespace

extern "C" {

int qvg_rope_table(int64_t n_rows, int32_t n_pairs, const double *frequencies, int64_t first, const int32_t *positions, int32_t n_axes,
                   const int32_t *axis, float amplitude, int32_t type, void *out, void *stream) {
    if (n_rows < 0 || n_rows > kMaxInt || n_pairs < 1 || n_pairs > 256 || n_axes < 1 || n_axes > 8) return QVG_ERR_BAD_PARAM;
    if ((type != QVG_F16 && type != QVG_F32) || amplitude - amplitude != 0.0f) return QVG_ERR_BAD_PARAM;
    if (!positions && (n_axes != 1 || first < 0 || first > kMaxInt || first + n_rows > kMaxInt + 1)) return QVG_ERR_BAD_PARAM;
    for (int p = 0; axis && p < n_pairs; ++p)
        if (axis[p] < 0 || axis[p] >= n_axes) return QVG_ERR_BAD_PARAM;
    if (n_rows == 0) return QVG_OK;
    if (!frequencies || !out) return QVG_ERR_NULL;
    if (!aligned16(out) || (reinterpret_cast<uintptr_t>(frequencies) & 7u) || !aligned4(positions)) return QVG_ERR_ALIGN;
    RopeTableArgs a{n_rows, n_pairs, n_axes, first, frequencies, positions, amplitude, out, {}, 0};
    for (int p = 0; axis && p < n_pairs; ++p) a.axis[p] = (uint8_t)axis[p];
    return launch_rope_table(a, type == QVG_F32, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_rope(const qvg_rotary *r, int32_t type, int64_t n_seqs, int32_t n_heads, int64_t n_tokens, int32_t head_dim, const void *x,
             int64_t x_stride_seq, int64_t x_stride_head, int64_t x_stride_token, const int32_t *first, int32_t backward, void *out,
             int64_t out_stride_seq, int64_t out_stride_head, int64_t out_stride_token, void *stream) {
    if (!r) return QVG_ERR_NULL;
    if (type != QVG_BF16 && type != QVG_F16 && type != QVG_F32) return QVG_ERR_BAD_PARAM;
    if (n_seqs < 0 || n_heads < 1 || n_heads > 65535 || n_tokens < 0 || n_seqs > kMaxInt || n_tokens > kMaxInt || n_seqs * n_tokens > kMaxInt)
        return QVG_ERR_BAD_PARAM;
    if (head_dim < 8 || head_dim > kMaxRow || head_dim % 8 || (backward != 0 && backward != 1)) return QVG_ERR_BAD_PARAM;
    int st = check_rotary(r, head_dim);
    if (st != QVG_OK) return st;
    if (n_seqs == 0 || n_tokens == 0) return QVG_OK;
    if (!x || !out) return QVG_ERR_NULL;
    if ((st = check_rotary_pointers(r)) != QVG_OK) return st;
    const int size = type == QVG_F32 ? 4 : 2;
    if (!rows_aligned(x, size, x_stride_seq, x_stride_head, x_stride_token) ||
        !rows_aligned(out, size, out_stride_seq, out_stride_head, out_stride_token) || !aligned4(first))
        return QVG_ERR_ALIGN;
    if (x == out && (x_stride_seq != out_stride_seq || x_stride_head != out_stride_head || x_stride_token != out_stride_token))
        return QVG_ERR_BAD_PARAM;
    TurnArgs a{};
    a.x = x; a.out = out;
    a.x_seq = x_stride_seq; a.x_head = x_stride_head; a.x_tok = x_stride_token;
    a.o_seq = out_stride_seq; a.o_head = out_stride_head; a.o_tok = out_stride_token;
    a.r = *r; a.first = first; a.backward = backward;
    a.H = n_heads; a.d = head_dim; a.n_tokens = (int)n_tokens; a.tokens = n_seqs * n_tokens;
    return launch_rope(a, type, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_append_pages(const qvg_page_cache *c, int64_t n_new, const void *k_new, const void *v_new, int64_t new_stride_seq,
                     int64_t new_stride_head, int64_t new_stride_token, const int32_t *n_live, const qvg_rotary *r, int32_t *len_out,
                     void *stream) {
    int st = check_cache(c);
    if (st != QVG_OK) return st;
    if (n_new < 0 || n_new > kMaxTokens || c->n_seqs * n_new > kMaxInt) return QVG_ERR_BAD_PARAM;
    if (c->head_dim % 8 || c->head_dim > kMaxRow) return QVG_ERR_BAD_PARAM;
    if (r && (st = check_rotary(r, c->head_dim)) != QVG_OK) return st;
    if (c->n_seqs == 0) return QVG_OK;
    if ((st = check_cache_pointers(c)) != QVG_OK) return st;
    const bool rows = n_new > 0 && c->table_pages > 0;
    if (rows && (!k_new || !v_new)) return QVG_ERR_NULL;
    if (rows && r && (st = check_rotary_pointers(r)) != QVG_OK) return st;
    if (rows && (!rows_aligned(k_new, 2, new_stride_seq, new_stride_head, new_stride_token) || !aligned16(v_new))) return QVG_ERR_ALIGN;
    if (!aligned4(n_live) || !aligned4(len_out)) return QVG_ERR_ALIGN;
    TurnArgs a{};
    a.x = k_new; a.v = v_new;
    a.x_seq = new_stride_seq; a.x_head = new_stride_head; a.x_tok = new_stride_token;
    if (r) a.r = *r;
    a.H = c->n_heads; a.d = c->head_dim; a.n_tokens = (int)n_new; a.tokens = rows ? c->n_seqs * n_new : 0;
    a.k_pages = c->k_pages; a.v_pages = c->v_pages; a.head = c->stride_head; a.page = c->stride_page; a.tok = c->stride_token;
    a.table = c->page_table; a.kv_len = c->kv_len; a.live = n_live; a.len_out = len_out;
    a.table_pages = c->table_pages; a.capacity = (int)(c->table_pages * c->page_len); a.pool_pages = (uint32_t)c->pool_pages;
    a.by_page = fast_div((uint32_t)c->page_len);
    const uintptr_t was = reinterpret_cast<uintptr_t>(c->kv_len), live = reinterpret_cast<uintptr_t>(n_live), now = reinterpret_cast<uintptr_t>(len_out),
                    size = (uintptr_t)c->n_seqs * sizeof(int32_t);
    auto apart = [&](uintptr_t x) { return now >= x + size || x >= now + size; };
    a.lengths_here = rows && len_out && apart(was) && (!n_live || apart(live));
    return launch_append(a, c->n_seqs, c->type, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

int qvg_attn_pages_scratch_bytes(const qvg_page_cache *c, const qvg_page_step *t, size_t *out) {
    const int st = check_page_step(c, t);
    if (st != QVG_OK) return st;
    if (!out) return QVG_ERR_NULL;
    *out = page_plan(*c, *t).state_bytes;
    return QVG_OK;
}

int qvg_attn_pages(const qvg_page_cache *c, const qvg_page_step *t, float softmax_scale, void *scratch, size_t scratch_bytes, void *stream) {
    int st = check_page_step(c, t);
    if (st != QVG_OK) return st;
    const float scale = softmax_scale * 1.4426950408889634f;
    if (!(softmax_scale > 0.0f) || scale - scale != 0.0f) return QVG_ERR_BAD_PARAM;       // positive, finite, also to base 2
    if (c->n_seqs == 0 || t->n_new == 0) return QVG_OK;
    if ((st = check_cache_pointers(c)) != QVG_OK) return st;
    if (!t->q || !t->out) return QVG_ERR_NULL;
    if (!rows_aligned(t->q, 2, t->q_stride_seq, t->q_stride_head, t->q_stride_token) ||
        !rows_aligned(t->out, 2, t->out_stride_seq, t->out_stride_head, t->out_stride_token) || !aligned4(t->n_live) || !aligned4(t->lse) ||
        !aligned16(scratch))
        return QVG_ERR_ALIGN;
    // (a workgroup reads its own rows of q before it writes them, and no others)
    if (t->q == t->out && ((c->n_seqs > 1 && t->q_stride_seq != t->out_stride_seq) || ((c->n_heads > 1 || t->group > 1) && t->q_stride_head != t->out_stride_head) ||
                           (t->n_new > 1 && t->q_stride_token != t->out_stride_token)))
        return QVG_ERR_BAD_PARAM;
    const PagePlan plan = page_plan(*c, *t);
    PageAttnArgs a{};
    a.c = *c; a.t = *t; a.scale = scale;
    a.paged = plan.paged; a.rows = plan.rows; a.row_blocks = plan.row_blocks;
    a.by_page = fast_div((uint32_t)c->page_len);
    a.by_tiles = fast_div((uint32_t)page_tiles((int)c->page_len));
    a.by_units = fast_div((uint32_t)(c->n_heads * plan.row_blocks)); a.by_blocks = fast_div((uint32_t)plan.row_blocks); a.by_new = fast_div((uint32_t)t->n_new);
    a.slots = scratch && scratch_bytes >= plan.state_bytes ? plan.slots : 0;
    a.extra = plan.extra; a.kept = plan.kept;
    a.state = static_cast<float *>(scratch);
    if (a.slots) a.places = reinterpret_cast<int2 *>(static_cast<char *>(scratch) + plan.state_bytes - (size_t)c->n_seqs * sizeof(int2));
    return launch_attn_pages(a, static_cast<hipStream_t>(stream)) == hipSuccess ? QVG_OK : QVG_ERR_LAUNCH;
}

}  // extern "C"
