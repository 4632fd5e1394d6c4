/*
 * attn.h -- C-ABI of the MI355X (gfx950) DBRX-style self-attention block, the
 * other half of a decoder layer beside the MoE FFN of moe.h (Chen et al.,
 * RACS'24: Sec. 2.1 and its decoder-layer figure -- self-attention then the
 * MoE FFN; Table tab:vars -- D_embed 6144, D_qkv_hidden 8192, and note (b):
 * a D_qkv_hidden x D_embed fused query/key/value projection plus a
 * D_embed x D_embed output projection per layer; Sec. 4.3 -- the block is
 * replicated on every node, so one device computes it whole).
 *
 * For T new tokens at positions pos0 .. pos0+T-1 of one sequence, per layer:
 *   h      = bf16( (x - mean) / sqrt(var + eps) * gamma )        layer norm
 *   q|k|v  = h Wqkv   (n_heads, n_kv_heads, n_kv_heads heads of head_dim)
 *   q, k   rotated by position (rotary encoding, pairs i and i + head_dim/2,
 *          angle pos * theta^(-2i/head_dim)), then q, k, v rounded to bf16;
 *          k and v are appended to the layer's cache
 *   a_j    = bf16( softmax_p(q_j . k_p / sqrt(head_dim)) v_p ), p over
 *          positions 0 .. pos of the token; query head j uses key/value head
 *          j / (n_heads / n_kv_heads)
 *   o      = a Wo (fp32)           y = bf16(x + o)
 * The paper fixes the widths; the head split, the norm, the rotary encoding
 * and the rounding points are this library's readings.
 *
 * Conventions are those of moe.h: bf16 as uint16_t bits, device pointers
 * owned by the caller and 16-byte aligned, work enqueued on `stream`, every
 * argument checked on the host before any launch, a moe_status returned and
 * a message kept for attn_last_error.  A context is used by one host thread
 * and one stream at a time.
 */
#ifndef ATTN_H
#define ATTN_H

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct attn_ctx attn_ctx;

/* Block configuration.
 *   d_model    : D_embed, a multiple of 256, at most 8192.
 *   n_heads, n_kv_heads, head_dim : query heads, key/value heads (dividing
 *                n_heads) and their width, 64 or 128; (n_heads + 2
 *                n_kv_heads) head_dim is D_qkv_hidden, a multiple of 16, and
 *                n_heads head_dim a multiple of 256.
 *   n_layers   : layers held in the weight arena and the cache (>= 1).
 *   max_seq    : cache positions per layer (>= 1).
 *   max_tokens : largest T of a call, 1 .. 32768.  Up to 16 tokens a call
 *                takes the decode path (weight-streaming GEMVs, attention
 *                over position chunks or ranges); above, the prefill path (matrix-core
 *                GEMMs for the projections, causal attention on the matrix
 *                cores), which needs (n_heads + 2 n_kv_heads) head_dim to be
 *                a multiple of 256 when max_tokens > 16.
 *   rope_theta : base of the rotary frequencies (> 1).
 *   norm_eps   : layer-norm epsilon (>= 0).
 *   flags      : must be 0. */
typedef struct {
    int32_t d_model, n_heads, n_kv_heads, head_dim;
    int32_t n_layers, max_seq, max_tokens;
    float rope_theta, norm_eps;
    int32_t flags;
} attn_config;

/* Bytes of the caller-allocated weight arena (per layer: gamma fp32 [d]
 * padded to 256 B, the rotary frequencies fp64 [head_dim/2] padded to 256 B,
 * the post-attention norm's gamma2 fp32 [d] padded to 256 B,
 * then Wqkv and Wo repacked into the fragment-tiled layout
 * of moe.h's experts, the query and key rows of Wqkv reordered within each
 * head so that the two members of every rotation pair share a 16-row tile),
 * of the key/value cache, and of the workspace; 0 if cfg is invalid.  Cache layout, per layer l: K then V, each bf16
 * [n_kv_heads][max_seq][head_dim] (head-major, positions contiguous), so K of
 * layer l head g position p starts at element
 * ((l * 2 + 0) * n_kv_heads + g) * max_seq * head_dim + p * head_dim.  A
 * caller may write earlier positions' keys and values there directly. */
MOE_API size_t attn_weight_bytes(const attn_config *cfg);
MOE_API size_t attn_cache_bytes(const attn_config *cfg);
MOE_API size_t attn_workspace_bytes(const attn_config *cfg);

/* Sec. 4.1's persistent buffers, applied to the block: validates cfg and
 * records the three caller-allocated device buffers (256-byte aligned, kept
 * until attn_destroy).  Allocates only the host-side context.  Errors as
 * moe_init; the message is readable through attn_last_error(NULL). */
MOE_API moe_status attn_init(const attn_config *cfg, void *weight_arena, void *kv_cache,
                             void *workspace, attn_ctx **out);

/* Table tab:vars note (b): loads one layer's weights, repacking them once
 * into the arena.  gamma fp32 [d]; wqkv bf16 [d][(n_heads + 2 n_kv_heads)
 * head_dim] row-major (h wqkv gives q | k | v, heads in order); wo bf16
 * [n_heads head_dim][d] row-major (a wo gives o).  src_on_device as in
 * moe_load_expert (1: device pointers, kernels enqueued on stream; 0: host
 * pointers, repacked on the host and copied before returning). */
MOE_API moe_status attn_load_layer(attn_ctx *ctx, int32_t layer, const float *gamma,
                                   const uint16_t *wqkv, const uint16_t *wo,
                                   int32_t src_on_device, moe_stream_t stream);

/* Sec. 2.1 / Sec. 4.3: the block on T tokens x (bf16 [T, d]) at positions
 * pos0 .. pos0+T-1 of layer `layer`'s cache, which must already hold
 * positions 0 .. pos0-1; writes the tokens' keys and values at their
 * positions and y = bf16(x + o) (bf16 [T, d]; y may be x).  Requires
 * 1 <= T <= max_tokens (T == 0: no-op), pos0 >= 0, pos0 + T <= max_seq
 * (MOE_E_CAPACITY otherwise) and the layer loaded (MOE_E_STATE). */
MOE_API moe_status attn_forward(attn_ctx *ctx, int32_t layer, const uint16_t *x, uint16_t *y,
                                int32_t T, int32_t pos0, moe_stream_t stream);

/* The post-attention norm of a DBRX decoder layer (its attention part is
 * norm, attention, norm; Sec. 2.1's decoder layer feeds the MoE FFN the
 * block's output): loads gamma2 fp32 [d] of layer `layer` (src_on_device as
 * attn_load_layer). */
MOE_API moe_status attn_load_post_norm(attn_ctx *ctx, int32_t layer, const float *gamma2,
                                       int32_t src_on_device, moe_stream_t stream);

/* attn_forward, then z = bf16((y - mean) / sqrt(var + eps) * gamma2) (bf16
 * [T, d]), the normalised input of the layer's MoE FFN; z may be y.
 * Requires attn_load_post_norm of the layer (MOE_E_STATE). */
MOE_API moe_status attn_forward_norm(attn_ctx *ctx, int32_t layer, const uint16_t *x, uint16_t *y,
                                     uint16_t *z, int32_t T, int32_t pos0, moe_stream_t stream);

/* Introspection for tests: device pointers into the workspace with the last
 * forward's intermediates, valid until the next forward: h bf16 [T, d],
 * qkv fp32 [T, (n_heads + 2 n_kv_heads) head_dim] (before rotation), q bf16
 * [T, n_heads head_dim] (rotated), a bf16 [T, n_heads head_dim] (attention
 * output), o fp32 [T, d].  Any pointer may be NULL. */
MOE_API moe_status attn_intermediates(const attn_ctx *ctx, const uint16_t **h, const float **qkv,
                                      const uint16_t **q, const uint16_t **a, const float **o);

/* Per-kernel timing, as moe_profile_enable / moe_profile_read, with the
 * kinds of attn_kernel_kind. */
typedef enum {
    ATTN_K_NORM = 0,       /* layer norm */
    ATTN_K_QKV = 1,        /* fused projection (+ rotary + cache append, unless split) */
    ATTN_K_SCORE = 2,      /* causal attention (over position chunks or ranges) */
    ATTN_K_COMBINE = 3,    /* merge of the chunks or ranges (not with one range) */
    ATTN_K_OUT = 4,        /* output projection (+ residual, unless split) */
    ATTN_K_PACK = 5,       /* weight repacking */
    ATTN_K_ROPE = 6,       /* rotary + cache append (prefill, split projection) */
    ATTN_K_RESIDUAL = 7,   /* y = bf16(x + o) (prefill, split projection) */
    ATTN_K_POST_NORM = 8,  /* z = norm(y) (attn_forward_norm) */
    ATTN_K_COUNT = 9
} attn_kernel_kind;
MOE_API moe_status attn_profile_enable(attn_ctx *ctx, int32_t max_launches);
MOE_API moe_status attn_profile_read(attn_ctx *ctx, double *total_ms, int64_t *launches,
                                     int64_t *dropped);

/* Frees the host-side context (never the caller's buffers). */
MOE_API void attn_destroy(attn_ctx *ctx);

/* Message of the last failing call on ctx; with ctx == NULL, of the last
 * failing attn_init on this thread. */
MOE_API const char *attn_last_error(const attn_ctx *ctx);

/* ------------------------------------------------------------ paged cache --
 * The cache of many sequences at once, handed out in pages, for a server that
 * generates for a batch of them (the single-sequence cache above is one run of
 * positions).  A sequence's position p lies in page table[p / page_size] at
 * slot p % page_size; which pages are whose is the caller's business.  Two
 * operators work on it, each on the batch that attn_paged_set_batch set:
 *
 *   attn_paged_append  rotates the new tokens' queries and keys by their
 *                      positions (as attn_forward: pairs i and i + head_dim/2,
 *                      angle pos * theta^(-2i/head_dim)), writes the queries
 *                      out as bf16 and the keys and values to their pages;
 *   attn_paged_attend  o_j = bf16( softmax_p(q_j . k_p / sqrt(head_dim)) v_p ),
 *                      p over the token's sequence's positions up to its own;
 *                      query head j uses key/value head j / (n_heads /
 *                      n_kv_heads).
 *
 * attn_forward_paged is the attention block on top of them.
 *
 * Pages hold bf16, or with ATTN_PAGED_E4M3 one byte per element: e4m3 (1 sign,
 * 4 exponent, 3 mantissa bits, bias 7, largest value 448, no infinities) times
 * a scale per page and key/value head, keys and values apart.  A scale is a
 * power of two, so a stored value is code * scale exactly and exactly a bf16.
 * Append sets it to 2^e, e the least integer from -100 on such that 448 * 2^e is
 * no less than any finite new value of the page (at most 119: values past 448 *
 * 2^119 are stored as that).  Where the page already
 * holds earlier tokens of the sequence (the first new slot is not slot 0), the
 * scale never falls, and where it grows the earlier codes are rounded again to
 * the new one (which changes only values below 2^-6 of the new scale).  Codes
 * are rounded to nearest, ties to even, once, from the fp32 value.
 *
 * Values that are not finite: bf16 pages keep them; e4m3 pages store them as
 * NaN.  A row that sees such a value is not finite in its dimension, whatever
 * its weight; a key counts by its score q . k: NaN or +inf, and the row is not
 * finite in any dimension; -inf, and the position weighs nothing (a row all of
 * whose scores are -inf gives zeros, as one that sees no position).  Rows that
 * do not see it are untouched by it, and so are all rows by what slots behind a
 * sequence's last token hold.
 *
 * Numbers: scores are sums in fp32 (where the sum of |q_i k_i| passes its range
 * they may be infinite or NaN, and count as such), the weights' maximum and sum
 * are fp32, each weight enters its product with v as two bf16 terms (16 bits),
 * these sums are fp32, and the result is rounded to bf16 once.  The order of the
 * sums, and with it the last bits, depends on how a batch's positions are
 * divided. */

typedef struct attn_paged_ctx attn_paged_ctx;

#define ATTN_PAGED_E4M3 0x1 /* pages of e4m3 with a scale per page and key/value head */

/*   n_heads, n_kv_heads, head_dim : as attn_config, with at most 16 query
 *                heads per key/value head and n_heads * head_dim at most 65536.
 *   page_size  : positions per page, 16, 32, 64, 128 or 256.
 *   n_pages    : pages in each layer's pool, at most 2^24 (a page number means
 *                the same page of every layer).
 *   n_layers   : layers in the cache, 1 .. 1024.
 *   max_seqs   : most sequences of a batch, 1 .. 4096.
 *   max_tokens : most new tokens of a batch, all sequences together, 1 .. 32768.
 *   max_blocks : most pages of one sequence, 1 .. 65536 (max_blocks *
 *                page_size positions at most 2^24); max_seqs * max_blocks at
 *                most 2^26.
 *   rope_theta : base of the rotary frequencies (> 1).
 *   flags      : 0 or ATTN_PAGED_E4M3. */
typedef struct {
    int32_t n_heads, n_kv_heads, head_dim, page_size;
    int32_t n_pages, n_layers, max_seqs, max_tokens, max_blocks;
    float rope_theta;
    int32_t flags;
} attn_paged_config;

/* Bytes of the caller-allocated cache and workspace; 0 if cfg is invalid.
 * Cache layout, per layer: K, then V, each [n_pages][n_kv_heads][page_size]
 * [head_dim] of bf16 or e4m3 codes, then with ATTN_PAGED_E4M3 the scales of K
 * and of V, each fp32 [n_pages][n_kv_heads] padded to 256 B.  A caller may
 * write pages there directly (scales: powers of two from 2^-100 to 2^119). */
MOE_API size_t attn_paged_cache_bytes(const attn_paged_config *cfg);
MOE_API size_t attn_paged_workspace_bytes(const attn_paged_config *cfg);

/* Validates cfg and records the two caller-allocated device buffers (256-byte
 * aligned, kept until attn_paged_destroy).  Allocates only the host-side
 * context.  Errors as attn_init; the message is readable through
 * attn_paged_last_error(NULL). */
MOE_API moe_status attn_paged_init(const attn_paged_config *cfg, void *cache, void *workspace,
                                   attn_paged_ctx **out);

/* Sets the batch that the calls after it work on (one per generation step,
 * for all layers).  All arrays are host memory, read before the call returns:
 * n_new and pos0 int32 [n_seqs], sequence s having n_new[s] >= 0 new tokens
 * behind pos0[s] >= 0 cached ones; table int32 [n_seqs][ld], its row s the
 * sequence's pages (ceil((pos0 + n_new) / page_size) entries are read).  The
 * batch's tokens are the sequences' new tokens in order, T = sum of n_new.
 * A table entry of -1 is no page: its positions are left out of the
 * attention (a row that sees no position gives zeros); append refuses a batch
 * whose new tokens do not all have pages.
 * Enqueues one small kernel on stream that hands the batch to the device (not
 * where neither it nor the batch before has a token);
 * allocates no device memory (the first calls allocate pinned host memory).
 * Errors, the previous batch then staying set: MOE_E_ARG (a NULL array,
 * negative counts, ld too small, an entry outside -1 .. n_pages - 1, a page
 * that two sequences or two blocks of one would write), MOE_E_CAPACITY (n_seqs,
 * T or a sequence's length beyond the config's), MOE_E_STATE (stream is
 * capturing a graph); after MOE_E_HIP no batch is set.
 * The calls on a context share its workspace: they go to one stream, or the
 * caller orders them.
 * A graph captured over append and attend calls replays on the batch that is
 * set when it is replayed, which must have as many sequences and the same
 * n_new as the one set at its capture (positions and pages may differ);
 * on a batch with another number of tokens it does nothing. */
MOE_API moe_status attn_paged_set_batch(attn_paged_ctx *ctx, int32_t n_seqs, const int32_t *n_new,
                                        const int32_t *pos0, const int32_t *table, int32_t ld,
                                        moe_stream_t stream);

/* Types of attn_paged_append's q | k | v. */
typedef enum { ATTN_QKV_F32 = 0, ATTN_QKV_BF16 = 1 } attn_qkv_type;

/* q | k | v of the batch's T tokens (rows of (n_heads + 2 n_kv_heads) head_dim
 * elements, ld elements apart, rows 16-byte aligned) in; q out bf16 [T][n_heads
 * head_dim]; keys and values to the pages of layer `layer`; slots of other
 * positions keep their values (see above for scales that grow).  q may not
 * overlap what lies between qkv's first element and its last (MOE_E_ARG).
 * Requires a batch whose new tokens all have pages (MOE_E_STATE); T == 0 is a
 * no-op. */
MOE_API moe_status attn_paged_append(attn_paged_ctx *ctx, int32_t layer, const void *qkv, int64_t ld,
                                     int32_t type, uint16_t *q, moe_stream_t stream);

/* Attention of the batch's T tokens, q bf16 [T][n_heads head_dim] (rotated),
 * over their sequences' positions up to their own in layer `layer`'s pages,
 * which must hold them; out bf16 [T][n_heads head_dim] may not overlap q
 * (MOE_E_ARG). */
MOE_API moe_status attn_paged_attend(attn_paged_ctx *ctx, int32_t layer, const uint16_t *q, uint16_t *out,
                                     moe_stream_t stream);

/* Frees the host-side context and its pinned memory (never the caller's
 * buffers); waits for a batch still on its way to the device. */
MOE_API void attn_paged_destroy(attn_paged_ctx *ctx);

/* Message of the last failing call on ctx; with ctx == NULL, of the last
 * failing attn_paged_init on this thread. */
MOE_API const char *attn_paged_last_error(const attn_paged_ctx *ctx);

/* attn_forward on a paged cache: the block on the T tokens of the batch set on
 * `cache`, x and y bf16 [T, d] (y may be x), layer `layer` of both contexts;
 * with z not NULL also z = norm2(y), as attn_forward_norm.  The contexts must
 * agree in n_heads, n_kv_heads, head_dim and rope_theta (MOE_E_SHAPE) and
 * share one device; T <= max_tokens of ctx, whose own cache is not used.
 * (attn_intermediates then finds no q | k | v in the order it names; and a graph
 * replayed on a batch with another number of tokens leaves the pages alone, but
 * y and z without meaning.)  Errors
 * as attn_forward and attn_forward_norm; MOE_E_STATE without a batch that
 * append takes. */
MOE_API moe_status attn_forward_paged(attn_ctx *ctx, int32_t layer, attn_paged_ctx *cache, const uint16_t *x,
                                      uint16_t *y, uint16_t *z, moe_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTN_H */
