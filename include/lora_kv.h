/*
 * lora_kv.h -- C ABI of the paged key-value cache and the attention that reads it (gfx950).
 *
 * What stands between the adapters of a layer's q, k, v projections and those of its o projection.  The batch is the
 * one lora_apply works on: T packed tokens cut into segments, one segment per request (one token of a decode request,
 * the next tokens -- or all -- of a prompt).  A request here is a sequence of the cache: the tokens it has cached so
 * far and the pages they lie in.  With c cached tokens before the batch, token i of the segment stands at position
 * p = c + i, and
 *
 *   lora_kv_append   K[p] = turn(k_i, p), V[p] = v_i, q'_i = turn(q_i, p)       (turn: rotary positions, see there)
 *   lora_kv_attend   out_i[h] = sum_{s <= p} w_s V[s][h / g],  w = softmax_{s <= p}(scale * q_i[h] . K[s][h / g])
 *
 * with g = n_heads / n_kv_heads query heads to a key-value head.
 *
 * The cache lies in otherwise idle GPU memory beside the adapters and shrinks and grows with them (paper section 4.2:
 * the adapter cache takes what the requests' keys and values leave): pages are moved together with lora_kv_compact
 * and lora_kv_set_limit keeps the ones above a limit out of use.
 *
 * Layout.  One caller-owned buffer [n_pages][n_layers][2][n_kv_heads][page_tokens * head_dim], so that a page's
 * bytes are contiguous over all layers.  In chunks of u values (16 bytes: u = 8 for LORA_BF16, 4 for LORA_F32) the
 * keys of a page and head lie [head_dim / u][page_tokens][u values of head_dim], its values
 * [page_tokens / u][head_dim][u tokens]: both as the matrix instructions take them, a chunk to a lane.  What lies
 * beyond a sequence's last token is never used, whatever its bits are.
 *
 * Conventions are those of lora_cache.h: every function returns LORA_OK or a negative lora_status, nothing aborts or
 * throws; device memory is the caller's; streams are hipStream_t as void* (NULL = the default stream); calls only
 * enqueue work.  A cache belongs to the device that is current when it is created: its buffers, tensors and streams are that
 * device's (calls make it current for themselves).  One lora_kv_t is driven by one host thread at a time.  Calls that enqueue work wait, on the device,
 * for the latest earlier call's stream if theirs is another one (that stream has to exist still; while it is being captured
 * calls on others return LORA_E_STATE; an ordering between captured calls and others is the caller's).  Lists of sequences
 * are checked before anything changes: a call that returns an error has changed nothing, except LORA_E_HIP.
 */
#ifndef LORA_KV_H
#define LORA_KV_H

#include <stddef.h>
#include <stdint.h>

#include "lora_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lora_kv lora_kv_t;             /* opaque */
typedef struct lora_kv_batch lora_kv_batch_t; /* opaque: device-resident lists of one batch; a handle never comes back, that of a destroyed batch is refused */

enum { LORA_KV_HOST_ONLY = 1 }; /* flags: sequences and pages only, no device work */

#define LORA_KV_MAX_TOKENS (1 << 28) /* of one sequence */

typedef struct {
    int32_t n_layers;
    int32_t n_heads, n_kv_heads; /* n_heads a multiple of n_kv_heads */
    int32_t head_dim;            /* 64, 128 or 256 */
    int32_t page_tokens;         /* 32, 64, 128 or 256 */
    int32_t n_pages;
    int32_t max_seqs;            /* sequences alive at once */
    int32_t max_batch_seqs;      /* segments of a batch */
    int32_t max_batch_tokens;    /* tokens of a batch; times n_heads / n_kv_heads at most LORA_KV_MAX_TOKENS */
    int32_t max_batch_pages;     /* pages of all sequences of a batch together (a shared page counts for each) */
    int32_t n_batches;           /* batches alive at once */
    int32_t dtype;               /* LORA_F32 | LORA_BF16: q, k, v, out and the pages */
    int32_t flags;
} lora_kv_config_t;

/* ---- sizes (pure host arithmetic; 0 on a bad config: a page, all layers, is less than 4 GB) ---- */
size_t lora_kv_page_bytes(const lora_kv_config_t *cfg);  /* one page, all layers */
size_t lora_kv_pages_bytes(const lora_kv_config_t *cfg); /* the pages' buffer */
/* The other buffer: lists of n_batches batches, and 64 MB in which attention over parts of a cache keeps what is joined afterwards. */
size_t lora_kv_work_bytes(const lora_kv_config_t *cfg);

/* ---- life cycle ------------------------------------------------------------------------ */

/* Both buffers are device memory, 256-byte aligned, and have to outlive the cache.  With LORA_KV_HOST_ONLY both may be NULL and
 * only the calls on sequences work (pages are handed out, shared and moved in the books alone). */
int lora_kv_create(const lora_kv_config_t *cfg, void *dev_pages, size_t pages_bytes, void *dev_work, size_t work_bytes,
                   lora_kv_t **out);
int lora_kv_destroy(lora_kv_t *kv); /* the caller has synchronised the streams that use it */

/* ---- sequences -------------------------------------------------------------------------- */

/* n new sequences without tokens.  LORA_E_STATE if an id is there already or named twice, LORA_E_NOMEM beyond max_seqs. */
int lora_kv_seq_add(lora_kv_t *kv, int32_t n, const int64_t *ids);

/* n new sequences that begin with the first n_tokens tokens of `parent` (-1: all of them): they share its pages, and a
 * shared page is copied only when one of its holders is about to write into it.  Fork after the appends of the
 * parent's batch are enqueued.  Errors as lora_kv_seq_add; LORA_E_NOTFOUND, LORA_E_INVAL if the parent has fewer tokens. */
int lora_kv_seq_fork(lora_kv_t *kv, int64_t parent, int32_t n, const int64_t *ids, int32_t n_tokens);

/* Add n_tokens[i] tokens to sequence ids[i] whose keys and values the caller puts into the pages himself (restored from
 * elsewhere, say) by work on `stream`, which waits for the cache's earlier work on other streams: takes pages -- the free ones with the lowest
 * numbers --, copies a shared page that the tokens begin in.
 * Batches with a sequence whose page was copied can't be used any more.  LORA_E_NOMEM if there are too few pages, LORA_E_NOTFOUND,
 * LORA_E_INVAL (a sequence named twice, a negative count), LORA_E_STATE on a stream that is captured. */
int lora_kv_seq_extend(lora_kv_t *kv, int32_t n, const int64_t *ids, const int32_t *n_tokens, void *stream);

/* Keep the first n_tokens[i] tokens (rejected drafts, a repeated iteration); pages that hold none of them are given
 * back.  Batches with one of the sequences can't be used any more. */
int lora_kv_seq_truncate(lora_kv_t *kv, int32_t n, const int64_t *ids, const int32_t *n_tokens);

/* The sequences end; pages that no other sequence shares are free. */
int lora_kv_seq_free(lora_kv_t *kv, int32_t n, const int64_t *ids);

typedef struct {
    int32_t n_tokens, n_pages, n_shared; /* n_shared: pages that other sequences hold too */
} lora_kv_seq_info_t;
int lora_kv_seq_info(const lora_kv_t *kv, int64_t id, lora_kv_seq_info_t *out);

/* The sequence's pages in order; *n receives how many there are, `pages` (may be NULL) up to cap of them. */
int lora_kv_seq_pages(const lora_kv_t *kv, int64_t id, int32_t *pages, int32_t cap, int32_t *n);

/* ---- pages ------------------------------------------------------------------------------- */

/* Move pages so that the ones in use are the lowest numbers (the highest ones are copied, all layers, into the holes).  *moved
 * receives how many.  All batches that are alive can't be used any more if any page moved.  Work on `stream` after the call comes after all
 * earlier work on the pages, also if none moved: it may put those that are free behind a limit to another use.  LORA_E_STATE on a stream that is captured. */
int lora_kv_compact(lora_kv_t *kv, void *stream, int32_t *moved);

/* Pages with numbers from `limit` on are not handed out (limit up to n_pages; the memory behind them is the caller's to use).
 * LORA_E_STATE if one of them is in use: compact first. */
int lora_kv_set_limit(lora_kv_t *kv, int32_t limit);

typedef struct {
    int32_t limit, pages_used, pages_free, pages_shared, pages_end, seqs; /* pages_end: one past the highest in use */
    int64_t pages_copied;                                                 /* since the cache was created: on writes, and moved */
} lora_kv_stats_t;
int lora_kv_stats(const lora_kv_t *kv, lora_kv_stats_t *out);

/* ---- batches ------------------------------------------------------------------------------ */

/* The next iteration: segment i is tokens [seg_offsets[i], seg_offsets[i + 1]) of the packed batch and the next tokens of sequence
 * seg_seq[i]; seg_offsets[0] = 0; a segment may be empty.  The sequences get these tokens (pages as lora_kv_seq_extend takes them),
 * and the batch's lists -- pages, what is appended where, how the attention is cut up -- are uploaded.  One batch serves every layer.
 * (The host waits here only if the lists' memory is still on its way up for a batch that was destroyed: two more than n_batches are kept.)
 * LORA_E_INVAL (malformed offsets, a sequence named twice), LORA_E_NOTFOUND, LORA_E_NOMEM (pages, the config's maxima, batches
 * alive), LORA_E_STATE on a stream that is captured. */
int lora_kv_batch_create(lora_kv_t *kv, int32_t n_seg, const int64_t *seg_seq, const int32_t *seg_offsets, void *stream,
                         lora_kv_batch_t **out);
int lora_kv_batch_destroy(lora_kv_t *kv, lora_kv_batch_t *batch);

/* How the attention works on tiles of rows: four wavefronts to a tile; the same, three tiles on a compute unit; two groups of four wavefronts to a
 * tile; tiles of twice as many rows, two groups in turns. */
enum { LORA_KV_TILES_PLAIN = 0, LORA_KV_TILES_MANY = 1, LORA_KV_TILES_PAIRS = 2, LORA_KV_TILES_TURNS = 3 };

/* What the batch was cut into, for tests and tools. */
typedef struct {
    int32_t n_tokens, n_segments, n_pages; /* n_pages: entries of the page lists */
    int32_t n_groups;                      /* pieces of the append */
    int32_t n_row_items, n_tile_items;     /* attention, per key-value head: pieces with up to 16 rows, tiles of rows */
    int32_t n_joins;                       /* row blocks whose pieces are joined afterwards */
    int32_t n_short_items;                 /* of the row items: those that a wavefront has to itself */
    int32_t tiles_way;                     /* LORA_KV_TILES_* */
} lora_kv_batch_info_t;
int lora_kv_batch_info(const lora_kv_batch_t *batch, lora_kv_batch_info_t *out);

enum { LORA_ROPE_HALVES = 0, LORA_ROPE_NEIGHBOURS = 1 };

typedef struct {
    const void *k, *v;                   /* device [T][n_kv_heads][head_dim]: heads one after the other, tokens k_stride / v_stride values apart */
    int64_t k_stride, v_stride;
    const void *q;                       /* device [T][n_heads][head_dim], or NULL: keys and values only */
    void *q_out;                         /* where turned queries go; may be q itself with the same stride */
    int64_t q_stride, q_out_stride;
    const float *rope;                   /* device [rope_positions][rope_dim]: rope_dim / 2 cosines, then as many sines, 16-byte aligned; or NULL: nothing turns */
    int32_t rope_positions, rope_dim;    /* rope_dim: a multiple of 16 up to head_dim; values beyond it are not turned */
    int32_t rope_pairs;                  /* LORA_ROPE_HALVES: values (j, j + rope_dim / 2) turn together; LORA_ROPE_NEIGHBOURS: (2j, 2j + 1) */
} lora_kv_append_t;

/* Put the batch's keys and values of one layer into the pages.  Each pair (a, b) of a key or query at position p becomes
 * (a cos - b sin, b cos + a sin) with entry j of the table's row p, in fp32, rounded once.  Pointers and strides 16-byte aligned.
 * LORA_E_INVAL on bad arguments (a position of the batch beyond rope_positions among them), LORA_E_STATE if the batch can't be
 * used any more. */
int lora_kv_append(lora_kv_t *kv, lora_kv_batch_t *batch, int32_t layer, const lora_kv_append_t *a, void *stream);

/* Attention of the batch's tokens over their sequences' pages in one layer, causal: q and out device [T][n_heads][head_dim], tokens
 * q_stride / out_stride values apart, 16-byte aligned; out may be q itself with the same stride; scale > 0.  Scores, sums and outputs are held in fp32 and outputs
 * rounded once; with LORA_BF16 the weights exp(score - max) are rounded to bf16 for the product with the values (of segments with up to 16
 * rows -- tokens times n_heads / n_kv_heads -- to 16 significant bits, which costs nothing there).  A key or value
 * beyond a token's position has no influence on its output, whatever it is.  Sums are kept in range: an output is finite where the scores and
 * values that its token sees are, and infinite where one of the values is (if its weight is not 0).  The batch's parts are summed in an order
 * that depends on the batch alone: the same call gives the same bits. */
int lora_kv_attend(lora_kv_t *kv, lora_kv_batch_t *batch, int32_t layer, const void *q, int64_t q_stride, void *out,
                   int64_t out_stride, float scale, void *stream);

#ifdef __cplusplus
}
#endif
#endif
