/*
 * taper_latent -- attention over a paged cache that holds one latent vector a token (MI355X / gfx950).
 *
 * The same batches as taper_attn.h (serial requests, and branches that share their request's prefix pages), on
 * models that keep, instead of keys and values per head, one latent vector c_t of latent_dim values and one rotated
 * key part r_t of rope_dim values for all heads.  Head h's key of token t is (W_k[h] c_t, r_t), its value
 * W_v[h] c_t.  A query is (q_n, q_r), head_dim values and rope_dim values:
 *     out[s,h,:] = sum_t softmax_t(scale * (q_n . W_k[h] c_t  +  q_r . r_t)) W_v[h] c_t
 *
 * Two forms of one operation.  The decode step is computed absorbed: (W_k[h]^T q_n, q_r) meets the cache as it is
 * stored, and W_v[h] is applied to the weighted sum of latents, so that a step reads each cached token once for all
 * heads.  Prompts are computed expanded: every head's keys and values are made once per token and then met by many
 * queries.
 *
 * Entry points, statuses and taper_last_error() follow taper_attn.h: plain C, 0 or a negative taper_status, nothing
 * throws or aborts, every call enqueues on the caller's stream and (creation and plans apart) allocates nothing and
 * does not synchronise.  "host" / "device" after a pointer says where the memory must live.
 *
 * ---------------------------------------------------------------- data layout
 * pages (the pool), device: bf16 [n_pool_pages][(latent_dim + rope_dim) / 8][page_size][8]: value d of a token (its
 *     latent vector, then its rotated key part) is at (d / 8) * (page_size * 8) + tok * 8 + d % 8 of its page.
 *     Slots past a length and unreferenced pages may hold any bit pattern; results do not depend on them.
 * w_up  : bf16 [n_heads][2 * head_dim][latent_dim]: W_k[h] and below it W_v[h], device.
 * q     : bf16 [rows][n_heads][head_dim + rope_dim];  out: bf16 [rows][n_heads][head_dim];
 * lse   : f32 [rows][n_heads], may be NULL: natural-log normaliser.  Rows of a decode step are its sequences.
 * All device pointers must be multiples of 16 bytes (lse: 4), else TAPER_EINVAL.
 */
#ifndef TAPER_LATENT_H
#define TAPER_LATENT_H

#include "taper_attn.h"

#define TAPER_LATENT_API TAPER_API

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int n_heads;    /* 1 to 256                                                            */
    int latent_dim; /* 256 or 512                                                          */
    int rope_dim;   /* 64                                                                  */
    int head_dim;   /* 64 or 128: a head's key part without rotation, and its values       */
    int page_size;  /* 16                                                                  */
    float scale;    /* softmax scale, normally 1/sqrt(head_dim + rope_dim)                 */
    int device;     /* HIP device ordinal; -1 = host-only context (see taper_attn_config)  */
} taper_latent_config;

typedef struct taper_latent_ctx taper_latent_ctx;
typedef struct taper_latent_plan taper_latent_plan;

TAPER_LATENT_API int taper_latent_create(const taper_latent_config *cfg /* host */, taper_latent_ctx **out_ctx);
TAPER_LATENT_API void taper_latent_destroy(taper_latent_ctx *ctx); /* synchronises the device: not while a stream is being recorded */

/* One unit of a decode step's work: n_tokens tokens from block-table entry page0 of row seq0 on, against n_rows query rows
 * (row = sequence * n_heads + head) from row0 on; its partial rows start at part_row.  n_rows 0: nothing (filler). */
typedef struct {
    int32_t seq0, page0, n_tokens, row0, n_rows, part_row;
} taper_latent_item;

/* Read-only view of a decode plan's integers (valid until taper_latent_plan_free). */
typedef struct {
    int32_t n_seqs, n_groups, n_items;
    const taper_latent_item *items;
    const int32_t *piece_start; /* [n_seqs + 1] CSR over piece_row                                              */
    const int32_t *piece_row;   /* the partial row of head 0 of each piece of the sequence; head h's is h below */
    int64_t n_partial_rows, tokens_unique, tokens_logical, device_bytes;
} taper_latent_view;

/*
 * Index resolution for one decode step; the batch arrays are those of taper_plan_build_segments, and so are the
 * checks and their statuses (seg_start may be NULL: one private segment per sequence).  One plan serves every layer
 * of the step.  A plan owns the partial rows and rewritten queries of its calls, so two plans never share a
 * workspace; the calls of one plan must be ordered on one stream, or by events.  target_workgroups 0: as many as the
 * device has compute units (256 on a host-only context).  TAPER_EINVAL on a stream that is being recorded into a graph.
 * Memory of a freed plan is used again by later plans of the
 * context, whose calls must be ordered behind its own.  Not safe to call concurrently on one ctx.  Plans are freed
 * before their context is destroyed.
 */
TAPER_LATENT_API int taper_latent_plan_build(taper_latent_ctx *ctx, int n_seqs, const int32_t *block_table /* host */, int bt_row_stride,
                                      const int32_t *branch_group /* host */, const int32_t *prefix_len /* host */,
                                      const int32_t *seg_start /* host, may be NULL */, const int32_t *seg_len /* host */,
                                      int64_t n_pool_pages, int target_workgroups, void *hip_stream, taper_latent_plan **out_plan);
/*
 * Index resolution for the prompt tokens of a batch: sequence s sees prefix_len[s] shared tokens and suffix_len[s] private
 * ones, all of them in the cache already, and its last new_len[s] (0 to suffix_len[s]) private tokens are the query rows.
 * Query i of n sees all tokens of its sequence but the last n - 1 - i.  Rows of q, out and lse are packed: sequence
 * s's begin at new_len[0] + .. + new_len[s - 1].  TAPER_ELEN for a new_len outside its range, or when no sequence has a
 * new token.  A shared prefix is expanded once for all branches of its request.
 */
TAPER_LATENT_API int taper_latent_prompt_plan_build(taper_latent_ctx *ctx, int n_seqs, const int32_t *block_table /* host */,
                                             int bt_row_stride, const int32_t *branch_group /* host */,
                                             const int32_t *prefix_len /* host */, const int32_t *suffix_len /* host */,
                                             const int32_t *new_len /* host */, int64_t n_pool_pages, void *hip_stream,
                                             taper_latent_plan **out_plan);
TAPER_LATENT_API void taper_latent_plan_free(taper_latent_plan *plan);
/* TAPER_EINVAL for a prompt plan. */
TAPER_LATENT_API int taper_latent_plan_export(const taper_latent_plan *plan, taper_latent_view *out_view /* host */);

/* The decode step's attention, one query row per sequence.  The call may be recorded into a HIP graph and replayed
 * while the plan lives. */
TAPER_LATENT_API int taper_latent_decode_step_attention(taper_latent_ctx *ctx, const taper_latent_plan *plan, const void *q /* device */,
                                                 const void *w_up /* device */, const void *pages /* device */, void *out /* device */,
                                                 float *lse /* device, may be NULL */, void *hip_stream);
/* Causal attention of the plan's new tokens.  Values of a sequence's tokens must be finite: one that is not may reach
 * the rows of earlier queries too.  May be recorded and replayed as above. */
TAPER_LATENT_API int taper_latent_prompt_attention(taper_latent_ctx *ctx, const taper_latent_plan *plan, const void *q /* device */,
                                            const void *w_up /* device */, const void *pages /* device */, void *out /* device */,
                                            float *lse /* device, may be NULL */, void *hip_stream);

/*
 * Append: token i's latent vector and rotated key part become slot slots[i] (page * page_size + token, as
 * taper_append_slots gives them) of the pool.  Rows of `latent` and `rope` are latent_stride and rope_stride elements
 * apart (multiples of 8, at least latent_dim and rope_dim), so that both may be parts of one wider tensor.  A slot
 * outside the pool, a negative one say, leaves the token out (padded batches).  Slots must be distinct.
 */
TAPER_LATENT_API int taper_latent_append(taper_latent_ctx *ctx, int64_t n_tokens, const void *latent /* device */, int64_t latent_stride,
                                  const void *rope /* device */, int64_t rope_stride, const int64_t *slots /* device */,
                                  void *pages /* device, written */, int64_t n_pool_pages, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TAPER_LATENT_H */
