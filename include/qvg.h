/*
 * qvg.h - C ABI of the MI355X (gfx950) KV-cache codec of Quant VideoGen.
 *
 * The codec compresses the K or V tensor of one chunk of video tokens of one
 * attention head (paper Sec. 4.1: X in R^{N x d}) in two steps:
 *   1. semantic-aware smoothing: k-means groups the N tokens into K groups and
 *      the group centroid is subtracted from each token (Sec. 4.1, Eq. 5-6);
 *   2. progressive residual quantization: the residual is quantized to 2 bits
 *      per element in groups of B channels, and what that leaves is quantized
 *      again, n_stages times (Sec. 3.2 Eq. 1-2 applied to the residual of
 *      Sec. 4.2; each stage stores its own codes and per-group scales).
 * Decoding replays the stages (Sec. 4.2 Eq. 7); the fused entry point decodes
 * tile by tile inside an attention kernel, so the bf16 cache never exists.
 *
 * General conventions
 *   - Every data pointer is a DEVICE pointer, 16-byte aligned, owned by the
 *     caller; the library allocates no device memory and keeps no state (the one exception is
 *     the static scratch array of qvg_encode_chunk_static, described there).
 *     `const qvg_params*`, `size_t*` are HOST pointers.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).  Calls
 *     only enqueue work on it and never synchronise.
 *   - "bf16" is the upper 16 bits of an IEEE binary32; "f16" is IEEE binary16.
 *   - Return value: QVG_OK (0) or a negative qvg_status; on error nothing was
 *     enqueued unless the status is QVG_ERR_LAUNCH (outputs then undefined).
 *   - Inputs must be finite; non-finite values are not detected.
 *
 * Stored format of one chunk of one unit (n_heads counts independent units;
 * K and V of all heads and layers may be stacked into it):
 *   centroids [K][d]            bf16
 *   ids       [N]               uint8   index of the token's centroid
 *   codes     [N][T][d/4]       uint8   channel 4i+j in bits 2j..2j+1 of byte i, holding the
 *                                       level q in {-1,0,1} (Eq. 2, b = 2) as 2-bit two's
 *                                       complement: 0b00 = 0, 0b01 = +1, 0b11 = -1 (0b10 unused)
 *   scales    [N][T][d/B]       f16     per group of B consecutive channels
 * Format variants (Sec. 5 "Implementation"): with bits = 4 (INT4) the levels are -7..7 as 4-bit
 * two's complement, codes [N][T][d/2], channel 2i+j in bits 4j..4j+3 of byte i; with
 * scale_format = QVG_SCALE_E4M3 a scale is one byte in the OCP FP8 E4M3 layout (1 sign, 4
 * exponent bits with bias 7, 3 mantissa bits; largest finite value 448, no infinity, subnormals
 * m/8 * 2^-6), scales [N][T][d/B] uint8; the encoder never writes the NaN code 0x7F, and a
 * decoder that meets it reads 480.  E4M3 scale arrays need no alignment.
 * With more than 256 centroids (the codebook-size study of Sec. 5, Table 5, goes to K = 512) an id
 * is a 16-bit word: every "uint8_t *ids" argument then points at uint16 data, 2-byte aligned
 * (with S smoothing stages: S consecutive words per token).
 * The encoder writes ids below K only; a decoder (qvg_decode*, qvg_attn_decode*) that meets a
 * larger one, in a cache it did not write, reads the table's last row for it instead of memory
 * beyond the table.
 * A cache of several chunks concatenates ids/codes/scales along N and keeps one
 * centroid table per chunk: centroids [n_chunks][K][d].
 * Alignment inside a cache: qvg_encode_chunk wants every output pointer 16-byte aligned, so a chunk
 * can be encoded in place at token offset c * chunk_len only if chunk_len * T * (d/B) * 2 bytes of
 * binary16 scales (and chunk_len * T * d*b/8 bytes of codes) are multiples of 16: a chunk_len that
 * is a multiple of 8 tokens always is (E4M3 scale bytes need no alignment).  The attention entry
 * points read any chunk length and capacity; their fastest kernel needs the same property of
 * chunk_len and, with several units, of the capacity, and the others are read by a general kernel.
 *
 * With S = n_smooth_stages > 1 (the paper's progressive residual quantization, Sec. 4.2: the
 * residual of one k-means round is clustered again, S times, before it is quantized) a chunk
 * keeps S tables, centroids [n_chunks][S][K][d], and a token S ids, ids [N][S]; the residual
 * handed from one round to the next is rounded to bf16.  Everywhere below "[K][d]" then reads
 * "[S][K][d]" and "ids [N]" reads "ids [N][S]".
 */
#ifndef QVG_H
#define QVG_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum qvg_status {
    QVG_OK = 0,
    QVG_ERR_NULL = -1,         /* a required pointer is NULL                      */
    QVG_ERR_BAD_PARAM = -2,    /* a size or parameter is out of its stated range  */
    QVG_ERR_UNSUPPORTED = -3,  /* valid in the paper, not built here              */
    QVG_ERR_WORKSPACE = -4,    /* workspace missing or too small                  */
    QVG_ERR_ALIGN = -5,        /* pointer or stride breaks the alignment rule     */
    QVG_ERR_LAUNCH = -6,       /* the HIP runtime refused a launch or a copy      */
    QVG_ERR_SCRATCH_LIMIT = -7 /* qvg_encode_chunk_static: the sizes need more scratch memory than
                                  QVG_STATIC_SCRATCH_BYTES                         */
} qvg_status;

/* Codec parameters, in the paper's symbols (Sec. 4, Sec. 5 "Implementation"). */
typedef struct qvg_params {
    int32_t n_heads;         /* H >= 1: independent units handled by one call           */
    int32_t head_dim;        /* d: 128                                                  */
    int32_t n_clusters;      /* K: 1..512; ids are uint8 up to 256 (Sec. 5: K = 256), uint16 beyond */
    int32_t group_size;      /* B: 16, 32, 64 or 128 consecutive channels of one token  */
    int32_t n_stages;        /* T: 1..8 rounds of b-bit quantization of the residual    */
    int32_t bits;            /* b: 2 or 4 bits per level (Sec. 5: INT2 / INT4)          */
    int32_t n_smooth_stages; /* S: 1..4 k-means smoothing rounds (QVG: 1, QVG-Pro: 4)        */
    int32_t kmeans_iters;    /* I >= 0 Lloyd iterations before the final assignment     */
    int32_t scale_format;    /* QVG_SCALE_F16 or QVG_SCALE_E4M3 (Sec. 5 "Implementation") */
} qvg_params;

#define QVG_SCALE_F16  0
#define QVG_SCALE_E4M3 1

/* which_entry values for qvg_workspace_bytes */
#define QVG_ENTRY_ENCODE 0
#define QVG_ENTRY_DECODE 1
#define QVG_ENTRY_ATTN   2
#define QVG_ENTRY_KMEANS_UPDATE 3
#define QVG_ENTRY_KMEANS_ASSIGN 4

/*
 * Encode one chunk (Sec. 4.1 and 4.2): I Lloyd iterations from init_centroids
 * (Sec. 4.3: the previous chunk's centroids, or any start the caller picks),
 * a final assignment, centroid subtraction (Eq. 5), then T rounds of 2-bit
 * group quantization of the residual (Eq. 1-2) with bit packing.
 *   x              [H][N][d] bf16 view: element (h,n,c) at x[h*stride_head + n*stride_token + c],
 *                  strides in elements, multiples of 8
 *   init_centroids [H][K][d] bf16 ([H][S][K][d]: one start table per smoothing round)
 *   centroids_out  [H][K][d] bf16, unit h at centroids_out + h*cent_out_stride_head elements
 *                  (0 = dense K*d; a multiple of 8; may equal init_centroids when I == 0 and dense)
 *   ids_out        [H][N]           codes_out [H][N][T][d/4]   scales_out [H][N][T][d/B] f16,
 *                  unit h starting out_stride_head_tokens tokens after unit h-1 (0 = dense N;
 *                  >= N).  The two strides let a chunk be written straight into a cache that
 *                  holds several chunks per unit: point the outputs at the chunk's first token
 *                  and table, and pass the cache's tokens and table elements per unit.
 *   workspace      qvg_workspace_bytes(p, QVG_ENTRY_ENCODE, N, 0) bytes (a few KB per unit when I == 0)
 * A call that the free chip holds at once (up to 6144 tokens per unit, 512 workgroups of 256 tokens) runs all its iterations in one launch, whose
 * workgroups wait for each other.  Where another stream's kernel holds part of the chip, a unit is done by those of its
 * workgroups that have a place: same results, 1.1 to 2 times the time that one launch per step takes beside the same kernel.
 * n_tokens in 0 .. 2^20.  n_tokens == 0 only copies the centroids.
 * Rounding rules that fix the stored integers: a group's scale is max|r| / qmax (one fp32
 * division; qmax = 2^(b-1) - 1, so 1 for b = 2), saturated at the scale format's largest finite
 * value (65504 or 448) and rounded to nearest even; q = round-half-even(r * (1/scale))
 * with 1/scale one correctly rounded fp32 division, clamped to [-qmax, qmax]; a zero scale gives
 * q = 0; the next round sees fma(-scale, q, r).  Assignment: smallest squared Euclidean
 * distance, the lowest index among exactly equal ones; a centroid is the mean of its
 * members summed in token order in fp64, rounded to fp32 then to bf16; an empty group
 * keeps its centroid.
 */
int qvg_encode_chunk(const qvg_params *p, int64_t n_tokens,
                     const void *x_bf16, int64_t stride_head, int64_t stride_token,
                     const void *init_centroids_bf16, void *centroids_bf16_out,
                     int64_t cent_out_stride_head,
                     uint8_t *ids_out, uint8_t *codes_out, void *scales_f16_out,
                     int64_t out_stride_head_tokens,
                     void *workspace, size_t workspace_bytes, void *stream);

/*
 * qvg_encode_chunk for callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same call without the workspace
 * arguments.  The workspace lives in a static device array inside the library,
 * 48 MiB per GPU the library runs on, held until the process ends; the call
 * allocates and frees nothing.  Arguments, results and errors are those of qvg_encode_chunk, plus
 *   QVG_ERR_SCRATCH_LIMIT  when the sum of 8 bytes per centroid (K rounded up to a multiple of
 *                          64) and 4 per unit, of two bf16 tables (kmeans_iters > 0 or several
 *                          stages), of 4 bytes per token and 4 (K + 1) per unit (kmeans_iters > 0), and of
 *                          one (two stages) or two (more) bf16 copies of the chunk, each rounded up
 *                          to 256 bytes, exceeds QVG_STATIC_SCRATCH_BYTES
 *                          (nothing was enqueued).  One layer's chunk of
 *                          every configuration this library is measured on fits (24 units x 4680
 *                          tokens, K = 256: 3.7 MB; 80 units x 10800 tokens, K = 128: 9 MB);
 *                          several smoothing stages need two bf16 copies of the chunk and fit only
 *                          for small chunks.
 * All calls on one GPU share that GPU's array: two calls whose kernels may overlap in time (on
 * different streams, or from different threads on the same stream without ordering) race.  Calls
 * on one stream are ordered and safe.  The array keeps the previous call's contents; nothing in it
 * needs to start at zero.
 */
#define QVG_STATIC_SCRATCH_BYTES (16u << 20)
int qvg_encode_chunk_static(const qvg_params *p, int64_t n_tokens,
                            const void *x_bf16, int64_t stride_head, int64_t stride_token,
                            const void *init_centroids_bf16, void *centroids_bf16_out,
                            int64_t cent_out_stride_head,
                            uint8_t *ids_out, uint8_t *codes_out, void *scales_f16_out,
                            int64_t out_stride_head_tokens, void *stream);

/*
 * Decode (Sec. 4.2 "dequantization process", Eq. 7; Sec. 4.3 "Dequantization
 * kernel": all stages in one kernel, the running value kept in registers):
 * x_hat = centroid[id] + sum_t scale_t * q_t, fp32 fma in stage order, one
 * rounding to bf16 (S > 1: the S centroid rows are added first, in round order, in fp32).
 *   n_tokens (0 .. 2^31-1) tokens per unit in chunks of chunk_len (the last may be shorter;
 *   chunk_len >= n_tokens means one chunk); centroids [H][n_chunks][K][d].
 *   x_bf16_out: same view convention as the encoder's x.
 */
int qvg_decode(const qvg_params *p, int64_t n_tokens, int64_t chunk_len,
               const void *centroids_bf16, const uint8_t *ids, const uint8_t *codes,
               const void *scales_f16, void *x_bf16_out, int64_t stride_head,
               int64_t stride_token, void *stream);

/*
 * qvg_decode of a token range of caches that are allocated for more tokens than are decoded:
 * tokens first_token .. first_token + n_tokens - 1 of every unit, first_token a multiple of
 * chunk_len; unit h starts kv_capacity_tokens tokens (ids, codes, scales) and
 * ceil(kv_capacity_tokens / chunk_len) tables after unit h-1 (0 = first_token + n_tokens).
 * The array pointers are those of the whole cache (token 0 of unit 0); x_bf16_out receives
 * the range only, [H][n_tokens][d] in the view convention of qvg_decode.
 */
int qvg_decode_ex(const qvg_params *p, int64_t n_tokens, int64_t chunk_len,
                  int64_t kv_capacity_tokens, int64_t first_token,
                  const void *centroids_bf16, const uint8_t *ids, const uint8_t *codes,
                  const void *scales, void *x_bf16_out, int64_t stride_head,
                  int64_t stride_token, void *stream);

/*
 * Attention over the compressed cache: O = softmax(softmax_scale * Q K_hat^T) V_hat
 * per unit, no mask, where K_hat and V_hat are what qvg_decode would return (bf16),
 * produced tile by tile in LDS and never written to memory (or, with a workspace, written one
 * slab of chunks at a time into it: see `workspace`).
 *   q_bf16   [H][n_q][d] contiguous       out_bf16 [H][n_q][d] contiguous
 *   K and V caches: n_kv_tokens tokens in chunks of chunk_len, each with the
 *   layout qvg_decode reads; both use the parameters in *p.
 *   lse_out  [H][n_q] fp32 natural-log sum of exp of the scaled scores, or NULL
 *   workspace: optional device memory, 16-byte aligned.  Without it (NULL, 0) every block of 256
 *              queries decodes the cache for itself inside one kernel.  With it every 64-token tile
 *              is decoded ONCE per unit into the workspace (K_hat as bf16, V_hat as binary16, 512
 *              bytes per token and unit) and read from there by all query blocks: a slab of as many
 *              whole chunks as fit at a time, two launches per slab, the queries' running soft-max
 *              state (528 bytes per query and unit) carried in the workspace from slab to slab.
 *              The full-precision cache is never held beyond one slab.  Useful from 512 queries
 *              per unit upward (the dequantization is what bounds the one-kernel form).
 *              qvg_workspace_bytes(p, QVG_ENTRY_ATTN, tokens, n_q) gives the bytes that hold
 *              `tokens` tokens of decoded tiles plus the state, where tokens = number of chunks in
 *              a slab x chunk_len rounded up to a multiple of 64.  A workspace that cannot hold one
 *              chunk (plus the state, when the cache has more chunks than fit) is ignored, and so is
 *              any workspace when n_q <= 256.  Contents are
 *              scratch: nothing has to be initialised and nothing survives the call.  The result
 *              equals the one-kernel form's bit for bit (same operands, same order of operations).
 * n_kv_tokens >= 1; n_q == 0 is a no-op; softmax_scale must be positive and finite.
 */
int qvg_attn_decode(const qvg_params *p, int64_t n_q, const void *q_bf16,
                    int64_t n_kv_tokens, int64_t chunk_len,
                    const void *k_centroids, const uint8_t *k_ids, const uint8_t *k_codes,
                    const void *k_scales,
                    const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                    const void *v_scales,
                    float softmax_scale, void *out_bf16, float *lse_out,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * qvg_attn_decode with what a generation step needs around it (Sec. 3.1: a chunk attends to the
 * cached chunks and to itself; Sec. 5 "Implementation": keys are cached BEFORE the rotary
 * position embedding):
 *   kv_capacity_tokens  the caches may be allocated for more tokens than they hold: unit h starts
 *                       kv_capacity_tokens tokens (ids, codes, scales) and
 *                       ceil(kv_capacity_tokens / chunk_len) tables (centroids) after unit h-1;
 *                       only the first n_kv_tokens tokens are read.  0 = n_kv_tokens.  Attention
 *                       of an earlier chunk's queries over a prefix of the cache (chunk-causal
 *                       order) is a call with a smaller n_kv_tokens.
 *   k_rope_f16          NULL, or [n_kv_tokens][d/2][2] f16 = (cos, sin) of the rotation angle of
 *                       token n and channel pair i, shared by all units: every decoded key,
 *                       rounded to bf16 as qvg_decode returns it, is rotated on interleaved pairs,
 *                       y[2i] = x[2i] cos - x[2i+1] sin, y[2i+1] = x[2i] sin + x[2i+1] cos (one
 *                       fp32 product and one fma each, then bf16), before the scores are taken.
 *                       The queries arrive already rotated.  V is not rotated.
 * Everything else as in qvg_attn_decode.
 */
int qvg_attn_decode_ex(const qvg_params *p, int64_t n_q, const void *q_bf16,
                       int64_t n_kv_tokens, int64_t chunk_len, int64_t kv_capacity_tokens,
                       const void *k_centroids, const uint8_t *k_ids, const uint8_t *k_codes,
                       const void *k_scales,
                       const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                       const void *v_scales,
                       const void *k_rope_f16,
                       float softmax_scale, void *out_bf16, float *lse_out,
                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * qvg_attn_decode_ex with a prefix length per query: query i (of every unit) sees the cached
 * tokens 0 .. q_kv_len[i]-1 only.  With lengths that are multiples of chunk_len this is the
 * chunk-causal order of Sec. 3.1 for the queries of SEVERAL chunks in one call (each chunk
 * attends to the chunks before it; its own keys are not in the compressed cache: see
 * qvg_attn_merge).
 *   q_kv_len   [n_q] int32, device; values are clamped to 0 .. n_kv_tokens.  NULL = every query
 *              sees all n_kv_tokens tokens (the call is then qvg_attn_decode_ex).  A query with
 *              length 0 (the first chunk of a chunk-causal batch: nothing is cached before it)
 *              gets a zero output row and lse = -infinity, which qvg_attn_merge treats as a
 *              partial result without weight.
 * A workgroup stops at the longest prefix among its 256 queries, so queries sorted by length
 * cost what their prefixes cost (with a workspace every tile of the cache is still decoded once;
 * the query blocks stop reading at their longest prefix).
 */
int qvg_attn_decode_causal(const qvg_params *p, int64_t n_q, const void *q_bf16,
                           int64_t n_kv_tokens, int64_t chunk_len, int64_t kv_capacity_tokens,
                           const void *k_centroids, const uint8_t *k_ids, const uint8_t *k_codes,
                           const void *k_scales,
                           const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                           const void *v_scales,
                           const void *k_rope_f16, const int32_t *q_kv_len,
                           float softmax_scale, void *out_bf16, float *lse_out,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * qvg_attn_decode_causal with the result left in fp32, [H][n_q][d] float, before the final rounding
 * to bf16 (no workspace arguments).  For checking the kernel's own arithmetic against a reference:
 * with a bf16 result, half an ulp of the output (2^-9 of its magnitude) hides what the kernel adds.
 * What the kernel adds: the scores are bf16 x bf16 products accumulated in fp32; the probabilities
 * enter the second contraction as binary16 rounded to nearest (the normaliser is the sum of the
 * rounded values), the decoded values as binary16 (exact: they are bf16 numbers; magnitudes beyond
 * 65504 are not supported).  The output error is therefore about 2^-12 of the magnitude of the
 * values a query attends to: below 2e-3 in absolute terms for |V| up to about 8, and it grows in
 * proportion beyond that (keys of any magnitude only sharpen the soft-max).
 */
int qvg_attn_decode_f32(const qvg_params *p, int64_t n_q, const void *q_bf16,
                        int64_t n_kv_tokens, int64_t chunk_len, int64_t kv_capacity_tokens,
                        const void *k_centroids, const uint8_t *k_ids, const uint8_t *k_codes,
                        const void *k_scales,
                        const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                        const void *v_scales,
                        const void *k_rope_f16, const int32_t *q_kv_len,
                        float softmax_scale, float *out_f32, float *lse_out, void *stream);

/*
 * qvg_attn_decode_causal (out_bf16) or qvg_attn_decode_f32 (out_f32; exactly one of the two is given)
 * with scratch memory for calls of few query blocks, of prefixes of different lengths, or with a few blocks beyond a
 * multiple of 256.  Such a call fills, or ends with, a fraction of the chip while
 * every workgroup walks the whole cache; with scratch of at least qvg_attn_scratch_bytes bytes, or with q_kv_len
 * qvg_attn_scratch_bytes_causal bytes (16-byte aligned), the cache's tiles are dealt to several workgroups per query block, and one
 * more launch joins their partial results (fp32).  How many depends on n_heads, n_q, n_kv_tokens, chunk_len
 * and the prefix lengths only, so equal calls give equal bits, with and without `workspace`.  They differ from the undivided
 * result by the order of fp32 sums and by the maxima that the binary16 probabilities are taken
 * against.  Without scratch (NULL, 0) or with less, this is the undivided call; except that of up to 256 blocks of 256 queries the
 * number of parts may fall as the cache grows, and scratch for a longer cache (n_kv_tokens larger, all else equal) divides a
 * shorter one into as many parts as it holds.
 * Prefix lengths may come in any order.  Calls of more than 128 blocks of 256 queries over 192 tiles or more read off
 * the first and the last query's what the others are like: where these two see about as much no block is divided, else the
 * blocks at the end that sees more run first.  Any other order gets the same results, not the best time.
 */
int qvg_attn_decode_parts(const qvg_params *p, int64_t n_q, const void *q_bf16,
                          int64_t n_kv_tokens, int64_t chunk_len, int64_t kv_capacity_tokens,
                          const void *k_centroids, const uint8_t *k_ids, const uint8_t *k_codes,
                          const void *k_scales,
                          const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes,
                          const void *v_scales,
                          const void *k_rope_f16, const int32_t *q_kv_len,
                          float softmax_scale, void *out_bf16, float *out_f32, float *lse_out,
                          void *workspace, size_t workspace_bytes,
                          void *scratch, size_t scratch_bytes, void *stream);

/* Bytes of scratch that let qvg_attn_decode_parts divide this call without q_kv_len; 0 when it would not be divided. */
int qvg_attn_scratch_bytes(const qvg_params *p, int64_t n_q, int64_t n_kv_tokens, int64_t chunk_len, size_t *out);
/* The same for a call with a prefix length per query: calls of up to 256 blocks of 256 queries are divided too, since
 * their blocks' shares of the cache differ. */
int qvg_attn_scratch_bytes_causal(const qvg_params *p, int64_t n_q, int64_t n_kv_tokens, int64_t chunk_len, size_t *out);

/*
 * Merge two attention results over DISJOINT key sets (the compressed cache, from
 * qvg_attn_decode with lse_out, and the current chunk's own bf16 keys, from the model's
 * attention kernel) into the attention over their union (Sec. 3.1):
 *   lse = log(exp(lse_a) + exp(lse_b)),  out = exp(lse_a - lse) out_a + exp(lse_b - lse) out_b.
 *   out_a, out_b, out  [n_rows][head_dim] bf16 contiguous (out may be out_a or out_b)
 *   lse_a, lse_b       [n_rows] fp32 natural-log sum of exp of the scaled scores; at least one
 *                      of the two must be finite in every row
 *   lse_out            [n_rows] fp32 or NULL
 */
int qvg_attn_merge(int64_t n_rows, int32_t head_dim, const void *out_a_bf16, const float *lse_a,
                   const void *out_b_bf16, const float *lse_b, void *out_bf16, float *lse_out,
                   void *stream);

/*
 * Paged caches.  A cache of several chunks per unit (chunk_len = page_len tokens each) also serves as a POOL of pages for
 * many sequences: page i of a unit is its tokens i * page_len .. (i + 1) * page_len - 1 and its table(s) i, written by
 * qvg_encode_chunk like chunk i of a cache.  A sequence is a list of pages, the same ones in every unit; the pages hold its
 * oldest tokens, all of them full but perhaps the last, and a bf16 TAIL holds the newest ones until they fill a page.
 */

/* What a step of a batch of sequences attends with and to (a HOST structure; its pointers are device pointers). */
typedef struct qvg_tree_step {
    int32_t n_seqs;            /* sequences, 0 .. 65535                                                          */
    int32_t group;             /* query heads per KV head, >= 1: query head h reads KV head h / group            */
    int32_t n_nodes;           /* new tokens per sequence, >= 0 (rows of q, k_new and v_new); group * n_nodes <= 2^20 */
    int32_t table_pages;       /* entries of page_table per sequence, >= 0                                       */
    int64_t page_len;          /* tokens of a page, >= 1; table_pages * page_len below 2^31                      */
    int64_t pool_pages;        /* pages of a unit in the pool, 1 .. 2^31 - 1                                     */
    const int32_t *page_table; /* [n_seqs][table_pages]: the sequence's pages in order; entries behind its last page are not
                                  read; one outside 0 .. pool_pages - 1 reads the nearest page of the pool       */
    const int32_t *kv_len;     /* [n_seqs] compressed tokens, clamped to 0 .. table_pages * page_len; NULL with table_pages == 0 */
    const void *q;             /* bf16 [n_seqs][n_heads * group][n_nodes][d]: strides in elements, multiples of 8 */
    int64_t q_stride_seq, q_stride_head, q_stride_node;
    const void *k_new, *v_new; /* bf16 [n_seqs][n_heads][n_nodes][d]: K (already rotated) and V of the new tokens */
    int64_t new_stride_seq, new_stride_head, new_stride_node;
    const void *k_tail, *v_tail;  /* bf16 [n_seqs][n_heads][tail_capacity][d] (K already rotated); NULL with tail_capacity == 0 */
    int64_t tail_stride_seq, tail_stride_head, tail_stride_token;
    const int32_t *tail_len;   /* [n_seqs], clamped to 0 .. tail_capacity; NULL with tail_capacity == 0           */
    int32_t tail_capacity;
    int32_t reserved;          /* 0 */
    const int32_t *nodes;      /* [n_seqs] new tokens that are there, clamped to 0 .. n_nodes; NULL: n_nodes      */
    const uint32_t *mask;      /* [n_seqs][n_nodes][ceil(n_nodes / 32)]: bit j of row i (bit j % 32 of word j / 32): new token i
                                  sees new token j; NULL: it sees the new tokens 0 .. i                          */
    const void *k_rope_f16;    /* NULL, or [rope_tokens][d/2][2] f16 (cos, sin), as in qvg_attn_decode_ex: compressed keys are
                                  rotated by their place in the sequence (0 .. kv_len - 1; beyond the table: its last row) */
    int64_t rope_tokens;
    void *out;                 /* bf16 [n_seqs][n_heads * group][n_nodes][d], strides like q's                    */
    int64_t out_stride_seq, out_stride_head, out_stride_node;
    float *lse;                /* [n_seqs][n_heads * group][n_nodes] fp32 natural-log sum of exp, or NULL         */
} qvg_tree_step;

/*
 * Attention of the few new tokens of a step (one per sequence, or a tree of drafted tokens) over everything their sequence
 * holds: O = softmax(softmax_scale * Q K^T) V per query head, where the keys of new token i of sequence b are
 *   - the kv_len[b] compressed tokens in the sequence's pages: K_hat and V_hat of Eq. 7, not rounded in between,
 *   - the tail_len[b] tokens of its tail,
 *   - the new tokens j < nodes[b] that the mask's row i names.
 * Rows i >= nodes[b] and rows that see no token at all get a zero output row and lse = -infinity.
 * A new token that no row sees may hold anything (also what is no number), and so may what lies behind a sequence's new tokens
 * or tail; every other value must be finite, and so must the scaled scores be.  Keys (also the rotated ones), values and the sums
 * of any of the parts of decoded ones are of magnitude up to 65504.
 *   k_*, v_*  the K and the V pool, [n_heads] units each, layout of a cache of pool_pages * page_len tokens per unit
 *   out       may be q with q's strides; it overlaps no other input
 *   scratch   optional, 16-byte aligned: with qvg_attn_tree_scratch_bytes bytes the sequences' tokens are dealt to several
 *             workgroups per KV head, by the sequences' lengths, and one more launch joins their partial results.  NULL or
 *             less: one workgroup per sequence, KV head and block of query rows, whose result differs by the order of fp32
 *             sums.  Equal calls give equal bits; among others a sequence's result may differ by that order too.
 *             Contents are scratch: nothing has to be initialised and nothing survives the call.
 * What is rounded: queries, keys, values and probabilities enter the two contractions with 11 bits or more, as binary16
 * (queries scaled by a power of two per row, probabilities by one per row and workgroup; keys and values as they are, with
 * binary16's step of 2^-24 below 2^-14), or where centroid rows and new tokens enter as stored in bf16 with probabilities of
 * 16 bits.  Sums of Eq. 7's rounds are formed in binary16 (one rounding a round, after the first) or fp32.  Scores,
 * normaliser and output are accumulated in fp32.
 * What is fast: one smoothing stage of one to four rounds of 2-bit levels with binary16 scales (B = 64; 32 from two rounds on), or of
 * one round with E4M3 scales (2-bit levels: B = 64 or 16, 4-bit: 64); four stages of one round with E4M3 scales (either levels, B = 16).
 * Every other format that the encoder writes takes a general kernel, five to ten times as long.
 */
int qvg_attn_tree(const qvg_params *p, const qvg_tree_step *t,
                  const void *k_centroids, const uint8_t *k_ids, const uint8_t *k_codes, const void *k_scales,
                  const void *v_centroids, const uint8_t *v_ids, const uint8_t *v_codes, const void *v_scales,
                  float softmax_scale, void *scratch, size_t scratch_bytes, void *stream);

/* Bytes of scratch that let qvg_attn_tree divide a call of these sizes (from n_seqs, group, n_nodes, table_pages, page_len and
 * tail_capacity; the pointers are not looked at); 0 when it would not be divided. */
int qvg_attn_tree_scratch_bytes(const qvg_params *p, const qvg_tree_step *t, size_t *out);

/*
 * Masks of draft trees from their parents, as qvg_attn_tree reads them, and the nodes' depths.
 *   parents    [n_seqs][n_nodes] int32: the parent of node i, below i; -1: the node follows the sequence's last token.
 *              Any other value, or i >= nodes[b], makes the node a hole: no node sees it, it sees no node, and neither does
 *              any node below it.
 *   nodes      [n_seqs] int32 or NULL
 *   mask_out   [n_seqs][n_nodes][ceil(n_nodes / 32)]: node i sees itself and its ancestors
 *   depth_out  [n_seqs][n_nodes] int32 or NULL: number of ancestors (the token's place is the sequence's length + depth);
 *              -1 for a hole
 * n_nodes in 0 .. 1024.
 */
int qvg_tree_mask(int64_t n_seqs, int64_t n_nodes, const int32_t *parents, const int32_t *nodes, uint32_t *mask_out,
                  int32_t *depth_out, void *stream);

/*
 * Append the K and V of the new tokens that are kept (the accepted path of a draft tree) to the tails:
 *   tail[b][.][tail_len[b] + i] = new[b][.][path[b][i]],  i < n_keep[b],   tail_len_out[b] = tail_len[b] + n_keep[b].
 *   path [n_seqs][n_path] int32, n_keep [n_seqs] (clamped to 0 .. n_path) int32, device.  A path entry outside
 *   0 .. n_nodes - 1 leaves its row of the tail as it was, and so does a row beyond tail_capacity; tail_len_out (may be
 *   tail_len, or NULL) is clamped to tail_capacity.  Views as in qvg_tree_step; the tails must not overlap k_new or v_new.
 */
int qvg_keep_nodes(int32_t n_heads, int32_t head_dim, int64_t n_seqs, int64_t n_nodes, const void *k_new, const void *v_new,
                   int64_t new_stride_seq, int64_t new_stride_head, int64_t new_stride_node,
                   const int32_t *path, int64_t n_path, const int32_t *n_keep,
                   void *k_tail, void *v_tail, int64_t tail_stride_seq, int64_t tail_stride_head, int64_t tail_stride_token,
                   int64_t tail_capacity, const int32_t *tail_len, int32_t *tail_len_out, void *stream);

/*
 * Copy whole pages, all arrays of all n_heads units: page src[i] of one pool becomes page dst[i] of another of the same
 * parameters and page_len, or of the same one (compaction of a pool; gathering a sequence's pages into consecutive ones,
 * which qvg_decode and qvg_attn_decode read).  src and dst are HOST arrays, read before the call returns.  QVG_ERR_BAD_PARAM
 * for a page outside its pool, a destination named twice, and, within one pool (the same codes pointer), a destination that
 * is also a source: the pairs are copied in no particular order.  Different pools must not overlap.
 */
int qvg_copy_pages(const qvg_params *p, int64_t page_len, int64_t n_pairs, const int32_t *src, const int32_t *dst,
                   int64_t src_pool_pages, const void *src_centroids, const uint8_t *src_ids, const uint8_t *src_codes,
                   const void *src_scales,
                   int64_t dst_pool_pages, void *dst_centroids, uint8_t *dst_ids, uint8_t *dst_codes, void *dst_scales,
                   void *stream);

/*
 * Rotary positions.  A table holds (cos, sin) of an angle for every place and pair of channels; a row of a head's channels is turned
 * pair by pair by the table's row of its place.
 */
enum {                     /* element types */
    QVG_BF16 = 0, QVG_F16 = 1, QVG_F32 = 2
};

/* How rows are turned (a HOST structure; its pointers are device pointers). */
typedef struct qvg_rotary {
    const void *table;         /* [n_rows][n_pairs][2] (cos, sin); aligned to a pair (4 or 8 bytes), faster from 16 on            */
    int32_t type;              /* QVG_F16 or QVG_F32                                                                              */
    int32_t n_pairs;           /* 1 .. head_dim / 2: channels 0 .. 2 n_pairs - 1 of a row are turned, the others stay as they are  */
    int64_t n_rows;            /* 1 .. 2^31 - 1; a place outside 0 .. n_rows - 1 takes the nearest row                             */
    int32_t half;              /* 0: pair p is channels (2p, 2p + 1), as in qvg_attn_decode_ex; 1: channels (p, p + n_pairs)       */
    int32_t reserved;          /* 0 */
    const int32_t *positions;  /* [n_seqs][n_tokens] the tokens' places, or NULL: see the entry point                             */
} qvg_rotary;

/*
 * The table of n_rows places:  out[i][p] = amplitude * (cos, sin)(place(i, axis[p]) * frequencies[p]).
 *   frequencies  [n_pairs] double, device: radians per place, finite; the product with the place is taken in 64 bits and reduced there
 *                to less than a turn, so a far place loses 2^-51 of its angle and no more
 *   positions    [n_rows][n_axes] int32, device, or NULL (n_axes 1): place i is first + i
 *   axis         [n_pairs] int32, HOST, read before the call returns: values in 0 .. n_axes - 1; or NULL: all 0
 *   amplitude    finite (long contexts; 1 else)
 *   out          [n_rows][n_pairs][2] of `type`, QVG_F16 or QVG_F32, 16-byte aligned
 * n_pairs 1 .. 256, n_axes 1 .. 8, n_rows 0 .. 2^31 - 1; first 0 .. 2^31 - 1 and first + n_rows at most 2^31.
 */
int qvg_rope_table(int64_t n_rows, int32_t n_pairs, const double *frequencies, int64_t first, const int32_t *positions, int32_t n_axes,
                   const int32_t *axis, float amplitude, int32_t type, void *out, void *stream);

/*
 * Rows turned:  (y0, y1) = (cos x0 - sin x1, sin x0 + cos x1) for every pair, one product and one fma in fp32 each, rounded to the type;
 * backward: the gradient with respect to x of a gradient x with respect to y, (cos x0 + sin x1, cos x1 - sin x0).
 *   type         QVG_BF16, QVG_F16 or QVG_F32, of x and out
 *   x, out       [n_seqs][n_heads][n_tokens][head_dim], strides in elements; every row is 16-byte aligned and contiguous.  out may
 *                be x with x's strides, and overlaps it in no other way
 *   r            token i of sequence b stands at r->positions[b][i]; without positions at first[b] + i; without first at i
 *   first        [n_seqs] int32, device, or NULL
 * head_dim a multiple of 8 up to 512; n_seqs * n_tokens below 2^31.  Slower, three times and more: half with n_pairs no multiple of 8.
 */
int qvg_rope(const qvg_rotary *r, int32_t type, int64_t n_seqs, int32_t n_heads, int64_t n_tokens, int32_t head_dim,
             const void *x, int64_t x_stride_seq, int64_t x_stride_head, int64_t x_stride_token, const int32_t *first, int32_t backward,
             void *out, int64_t out_stride_seq, int64_t out_stride_head, int64_t out_stride_token, void *stream);

/*
 * Caches of 16-bit pages: what is not compressed, or not yet.  A pool holds pages of page_len tokens of every KV head; a sequence is a
 * list of pages, the same ones for all heads, of which it fills the first kv_len tokens.
 */
typedef struct qvg_page_cache {    /* a HOST structure; its pointers are device pointers */
    int32_t type;              /* QVG_BF16 or QVG_F16                                                                             */
    int32_t n_seqs;            /* 0 .. 65535                                                                                      */
    int32_t n_heads;           /* KV heads, 1 .. 65535                                                                            */
    int32_t head_dim;
    int32_t table_pages;       /* entries of page_table per sequence, >= 0                                                        */
    int32_t reserved;          /* 0 */
    int64_t page_len;          /* tokens of a page, >= 1; table_pages * page_len at most 2^30                                     */
    int64_t pool_pages;        /* pages of the pool, 1 .. 2^31 - 1                                                                */
    const int32_t *page_table; /* [n_seqs][table_pages]: the sequence's pages in order; those behind its last are not looked at   */
    const int32_t *kv_len;     /* [n_seqs] tokens, clamped to 0 .. table_pages * page_len                                         */
    void *k_pages, *v_pages;   /* token t of page p of KV head h at h * stride_head + p * stride_page + t * stride_token elements;
                                  rows of head_dim contiguous elements, 16-byte aligned                                           */
    int64_t stride_head, stride_page;
    int64_t stride_token;      /* 0 .. 2^24 */
} qvg_page_cache;

/*
 * The new tokens' keys and values go behind the sequences:  token i of sequence b, i < n_live[b], to place kv_len[b] + i, its key turned
 * on the way if r is given (without r->positions by the row of that place), its value as it is.
 *   k_new, v_new  [n_seqs][n_heads][n_new][head_dim] of c->type, strides in elements, rows 16-byte aligned
 *   n_live        [n_seqs] int32, device, clamped to 0 .. n_new; NULL: n_new
 *   len_out       [n_seqs] int32 or NULL: kv_len[b] + n_live[b], at most table_pages * page_len; may be kv_len
 * A token beyond the table, or whose page is outside 0 .. pool_pages - 1, is not written; nothing else of the pool is touched.
 * No two tokens may go to the same place (of a page that sequences share, or that a table names twice), and the pool must not overlap
 * k_new or v_new.  head_dim a multiple of 8 up to 512 (qvg_attn_pages reads 64, 96, 128, 192 and 256); n_seqs * n_new below 2^31.
 */
int qvg_append_pages(const qvg_page_cache *c, int64_t n_new, const void *k_new, const void *v_new, int64_t new_stride_seq,
                     int64_t new_stride_head, int64_t new_stride_token, const int32_t *n_live, const qvg_rotary *r, int32_t *len_out,
                     void *stream);

/* What attends to a cache of 16-bit pages (a HOST structure; its pointers are device pointers). */
typedef struct qvg_page_step {
    int32_t group;             /* query heads per KV head, >= 1: query head h reads KV head h / group                             */
    int32_t n_new;             /* query rows per sequence and head, >= 0; group * n_new <= 2^20                                   */
    const int32_t *n_live;     /* [n_seqs], clamped to 0 .. n_new: rows that are there; NULL: n_new                               */
    const void *q;             /* [n_seqs][n_heads * group][n_new][head_dim] of the cache's type, turned already; strides in
                                  elements, rows 16-byte aligned                                                                  */
    int64_t q_stride_seq, q_stride_head, q_stride_token;
    int32_t causal;            /* 1: row i, at place kv_len - n_live + i, sees the tokens up to its place; 0: all kv_len           */
    int32_t window;            /* > 0: of these only those from place - window + 1 on, and the first `sink`; 0: all                */
    int32_t sink;              /* >= 0 */
    int32_t reserved;          /* 0 */
    void *out;                 /* like q, strides of its own                                                                      */
    int64_t out_stride_seq, out_stride_head, out_stride_token;
    float *lse;                /* [n_seqs][n_heads * group][n_new] fp32 natural-log sum of exp, or NULL                            */
} qvg_page_step;

/*
 * Attention of a step's tokens over their sequences' pages, themselves among them (qvg_append_pages has put them there; kv_len counts
 * them):  O = softmax(softmax_scale * Q K^T) V per query head.
 * Rows i >= n_live[b], and rows that see no token, get a zero row and lse = -infinity.  What no row of a sequence sees may hold anything (also
 * what is no number): tokens behind kv_len, tokens between the first `sink` and the first row's window, whose pages may be
 * gone.  A page of a token that is seen, outside 0 .. pool_pages - 1, reads the nearest page of the pool.  All else must be
 * finite, and so must the scores, before and after they are scaled: the lse of a row with a score that is no number, or
 * infinite, is no number, and neither is the row if none of its scores is one or one is infinite (-infinity: a weight of 0).
 *   head_dim 64, 96, 128, 192 or 256; n_seqs times n_heads times blocks of 32 of a KV head's query rows at most 2^23
 *   out      may be q with q's strides; it overlaps no other input
 *   scratch  optional, 16-byte aligned: with qvg_attn_pages_scratch_bytes bytes the sequences' tokens are dealt to several workgroups
 *            per KV head, by the sequences' lengths, and one more launch joins their partial results.  NULL or less: undivided, which
 *            differs by the order of fp32 sums.  Equal calls give equal bits; among others a sequence's result may differ by
 *            that order too.  Contents are scratch: nothing has to be initialised and nothing survives the call.
 * What is rounded: queries, keys and values enter the two contractions as they are, weights as two numbers of the type, off by at
 * most 2^-16 of themselves (bf16), or the larger of 2^-22 of themselves and 2^-24 of the largest of their 32 tokens' (binary16);
 * scores, sums and output are fp32 until the output is rounded.
 */
int qvg_attn_pages(const qvg_page_cache *c, const qvg_page_step *t, float softmax_scale, void *scratch, size_t scratch_bytes, void *stream);

/* Bytes of scratch that let qvg_attn_pages divide a call of these sizes (the pointers are not looked at); 0 when it would not be. */
int qvg_attn_pages_scratch_bytes(const qvg_page_cache *c, const qvg_page_step *t, size_t *out);

/*
 * The two k-means steps on their own (Sec. 4.1), as the encoder runs them.
 * assign: ids_out[h][n] = index of the nearest centroid of unit h; workspace
 *         qvg_workspace_bytes(p, QVG_ENTRY_KMEANS_ASSIGN, N, 0) bytes.
 * update: centroid = mean of its members (see qvg_encode_chunk for the rounding);
 *         counts_out [H][K] int32 may be NULL; workspace
 *         qvg_workspace_bytes(p, QVG_ENTRY_KMEANS_UPDATE, N, 0) bytes.
 */
int qvg_kmeans_assign(const qvg_params *p, int64_t n_tokens,
                      const void *x_bf16, int64_t stride_head, int64_t stride_token,
                      const void *centroids_bf16, uint8_t *ids_out,
                      void *workspace, size_t workspace_bytes, void *stream);
int qvg_kmeans_update(const qvg_params *p, int64_t n_tokens,
                      const void *x_bf16, int64_t stride_head, int64_t stride_token,
                      const uint8_t *ids, const void *centroids_prev_bf16,
                      void *centroids_bf16_out, int32_t *counts_out,
                      void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace an entry point needs for these sizes (host call, no GPU). */
int qvg_workspace_bytes(const qvg_params *p, int which_entry, int64_t n_tokens,
                        int64_t n_q, size_t *out);

/* Stored bytes of one chunk of n_tokens tokens for all H units: codes, scales,
 * ids and one centroid table per unit (Sec. 5 "Memory usage breakdown").
 * Negative qvg_status on bad parameters. */
int64_t qvg_compressed_bytes(const qvg_params *p, int64_t n_tokens);

/* Static, NUL-terminated description of a status code. */
const char *qvg_status_string(int status);

/* Library version: major*10000 + minor*100 + patch. */
int qvg_version(void);

#ifdef __cplusplus
}
#endif
#endif /* QVG_H */
