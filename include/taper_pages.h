/*
 * taper_pages -- copying, forking, joining, compacting and freeing pages of a paged cache (MI355X / gfx950).
 *
 * A page pool counts who uses each page (host integers); a mover moves pages or tokens on the device, through all
 * layers of a model in one call, for the KV pool of taper_attn.h and for the latent pool of taper_latent.h.
 *   fork     a branch that starts in the middle of a page shares the full pages and gets a copy of the last one
 *            (taper_page_pool_fork, taper_pages_copy);
 *   join     branches that have ended become one contiguous run of pages with the prefix, which can then be the shared
 *            prefix of the request's next parallel phase (taper_pages_pack);
 *   compact  live pages move to the front of the pool, so that its end can be given back (taper_page_pool_compact,
 *            taper_pages_copy, taper_pages_remap);
 *   free     a page whose last user is gone is free again (taper_page_pool_release).
 *
 * Statuses and taper_last_error() as in taper_attn.h; nothing throws or aborts.
 */
#ifndef TAPER_PAGES_H
#define TAPER_PAGES_H

#include "taper_attn.h"

#define TAPER_PAGES_API TAPER_API

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- who uses a page (host only) */
typedef struct taper_page_pool taper_page_pool; /* not safe to use from several threads at once */

TAPER_PAGES_API int taper_page_pool_create(int64_t n_pages, taper_page_pool **out_pool);
TAPER_PAGES_API void taper_page_pool_destroy(taper_page_pool *pool);
TAPER_PAGES_API int64_t taper_page_pool_free_pages(const taper_page_pool *pool); /* -1 for NULL */
/* Users of a page: 0 if it is free, -1 if it is outside the pool. */
TAPER_PAGES_API int32_t taper_page_pool_users(const taper_page_pool *pool, int32_t page);
/* n free pages, lowest numbers first, one user each.  TAPER_ENOMEM (and nothing taken) when fewer are free. */
TAPER_PAGES_API int taper_page_pool_alloc(taper_page_pool *pool, int64_t n, int32_t *pages /* out */);
/* One user more, or one less, for each entry (an entry may occur twice).  TAPER_EBLOCK, with nothing changed, when a page
 * is outside the pool, free, or released more often than it has users.  n_freed (may be NULL): pages that became free. */
TAPER_PAGES_API int taper_page_pool_share(taper_page_pool *pool, int64_t n, const int32_t *pages);
TAPER_PAGES_API int taper_page_pool_release(taper_page_pool *pool, int64_t n, const int32_t *pages, int64_t *n_freed);
/*
 * A child of a run of pages that holds n_tokens tokens: child_row gets ceil(n_tokens / page_size) entries, the full pages
 * shared with the parent (one user more), and, when the last one is not full, a page of its own: then *copy_src and
 * *copy_dst name the copy that taper_pages_copy has to make (-1 both when there is none).
 */
TAPER_PAGES_API int taper_page_pool_fork(taper_page_pool *pool, const int32_t *parent_row, int64_t n_tokens, int page_size,
                                  int32_t *child_row /* out */, int32_t *copy_src, int32_t *copy_dst);
/*
 * Moves that bring the live pages to the front: the highest live page to the lowest free one while that is lower, at most
 * max_moves (room in src and dst).  No page is source and destination.  The pool counts the pages at their new places at
 * once; the caller makes the copies and rewrites its block tables before it uses or frees any of them.
 */
TAPER_PAGES_API int taper_page_pool_compact(taper_page_pool *pool, int64_t max_moves, int32_t *src /* out */, int32_t *dst /* out */,
                                     int64_t *n_moves);
/* Entries of block tables that name a moved page name its new place. */
TAPER_PAGES_API int taper_pages_remap(int64_t n_entries, int32_t *entries, int64_t n_moves, const int32_t *src, const int32_t *dst);

/* ---------------------------------------------------------------- moving what pages hold */
typedef enum {
    TAPER_PAGES_KV = 0,    /* the pool of taper_attn.h: n_heads KV heads, dim = head_dim (64 or 128)            */
    TAPER_PAGES_LATENT = 1 /* the pool of taper_latent.h: n_heads 1, dim = latent_dim + rope_dim (320 or 576)    */
} taper_page_kind;

typedef struct {
    int kind;      /* taper_page_kind */
    int n_heads;
    int dim;
    int page_size; /* 16 */
    int device;    /* HIP device ordinal; -1 = host-only: arguments are checked, then TAPER_EHIP */
} taper_page_format;

typedef struct taper_mover taper_mover; /* holds the lists of calls in flight */

TAPER_PAGES_API int taper_mover_create(const taper_page_format *format /* host */, taper_mover **out_mover);
TAPER_PAGES_API void taper_mover_destroy(taper_mover *mover); /* synchronises the device: not while a stream is being recorded */
/*
 * Page dst[i] becomes a copy of page src[i], in each of the n_layers pools (one launch for all of them; each of
 * n_pool_pages pages, 16-byte aligned).  A source may be copied several times.  TAPER_EBLOCK for a page outside the pool,
 * TAPER_EINVAL when a destination occurs twice or is a source too.  Host arrays are read during the call, which enqueues
 * and returns; it allocates when a list is longer than any before it.  May be recorded into a HIP graph.  Calls on one mover
 * may come from several threads and on several streams.
 */
TAPER_PAGES_API int taper_pages_copy(taper_mover *mover, int n_layers, void *const *pools /* host array of device ptrs */, int64_t n_moves,
                              const int32_t *src /* host */, const int32_t *dst /* host */, int64_t n_pool_pages, void *hip_stream);
/*
 * Join: sequence s holds prefix_len[s] tokens and then the segments seg_len[seg_start[s] .. seg_start[s+1]), each on pages of
 * its own (arrays and checks as in taper_plan_build_segments).  Its tokens from first_token[s] on (a multiple of
 * page_size; NULL: all) are written one after the other to the pages dst_table[s][0 ..].  The rest of the last page
 * stays as it is.  A sequence may have nothing to move.  TAPER_EINVAL when a destination occurs twice or is a page that is
 * read.  Otherwise as taper_pages_copy, but a call on a capturing stream is refused (TAPER_EINVAL).
 */
TAPER_PAGES_API int taper_pages_pack(taper_mover *mover, int n_layers, void *const *pools /* host array of device ptrs */, int n_seqs,
                              const int32_t *block_table /* host */, int bt_row_stride, const int32_t *prefix_len /* host */,
                              const int32_t *seg_start /* host */, const int32_t *seg_len /* host */,
                              const int32_t *first_token /* host, may be NULL */, const int32_t *dst_table /* host */,
                              int dst_row_stride, int64_t n_pool_pages, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TAPER_PAGES_H */
