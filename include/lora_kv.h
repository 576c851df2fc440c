/*
 * lora_kv.h - Paged key-value cache and the attention that reads it, on
 * MI355X (gfx950).
 *
 * A step of continuous batching (Section 2.2 of the paper) runs, in every
 * layer, the adapted q, k and v projections (lora.h), then what this header
 * declares: the new keys and values go into the request's cache
 * (lora_kv_append), attention reads the cache (lora_attn_decode for requests
 * that decode one token, lora_attn_prompt for prompt segments), and its output
 * is the input of the adapted o projection.  Requests start, branch and end
 * between steps: their pages are handed out, shared, released and moved by the
 * lora_kv_grow, _grow_step, _fork, _fork_step, _free, _trim, _copy and _compact calls.
 *
 * Cache.  A page holds page_rows consecutive tokens of one sequence, for every
 * layer and every key-value head.  Element d of head h of row r of page p in
 * layer i is at
 *
 *     i * layer_stride + p * page_stride + h * head_stride + r * row_stride + d
 *
 * from k (and from v), in elements; strides may come in any order of size.
 * Token j of sequence s is row j % page_rows of page tables[s][j / page_rows].
 *
 * Attention.  For a query row at position p (0-based) of a sequence of len
 * tokens, with q head h reading key-value head h / (n_heads / n_kv_heads):
 *
 *     visible(j) = 0 <= j <= p  and  (window == 0 or j > p - window or j < n_sinks)
 *     out[d] = sum_j w_j V[j][d] / sum_j w_j,   w_j = exp(scale * q . K[j])
 *
 * over the visible tokens j < len.  A visible token whose page is outside
 * [0, n_pages) is left out.  A row for which nothing is left, or whose
 * weights are all zero, gets zeros.  Keys and values of tokens that a row does
 * not see have no effect on it, whatever they hold (NaN included); table
 * entries of pages in which no token is visible are not used.  Scores, the softmax's maximum and
 * sum and the output's sums are float32; a weight is rounded to the storage
 * type for the product with V, and the sum of weights is that of the rounded
 * ones; the output is rounded once.  (Against 64 bits that is a relative error of 0.0019 to
 * 0.0023 in bfloat16 and 0.00022 to 0.00026 in binary16, where the output's rounding
 * alone is 0.0017 and 0.0002.)  Binary16 weights below 2^-32 of the largest are zero.
 * The output's sums are divided at the end: bfloat16 values of 2^119 and more, or of 2^127
 * over the number of tokens, may pass float32's range in them.
 *
 * Tables, lengths and reference counts are in DEVICE memory and are read when
 * a launch runs: a decode step recorded in a HIP graph is replayed for the
 * next token, while lora_kv_grow_step, recorded with it, moves the lengths and
 * hands out pages.  What the device holds cannot be checked by the call;
 * every kernel checks it where it is used: a length is read as at most
 * max_len and at least 0, an entry outside [0, n_pages) as no page, segment
 * offsets as at most n_rows and at least 0.  No value in these arrays makes a
 * launch read or write outside the buffers described.
 *
 * Requirements, checked on the host before anything is enqueued (negative
 * code, lora_last_error() set, nothing enqueued):
 *   - dtype LORA_F16 or LORA_BF16; head_dim a multiple of 8 in [8, 256];
 *     n_heads a positive multiple of n_kv_heads;
 *   - page_rows a power of two in [16, 65536];
 *   - k, v, q, out 16-byte aligned, their strides and leading dimensions
 *     multiples of 8 elements (no cache stride below head_dim, leading
 *     dimensions at least n_heads or n_kv_heads times head_dim);
 *   - one page's rows of one head span less than 2 GiB;
 *   - max_len <= ld_table * page_rows and <= 2^30, scale positive and finite, window and
 *     n_sinks not negative;
 *   - q and out do not overlap;
 *   - a launch's tiles can be counted in 32 bits (n_seqs * n_heads *
 *     max_len / 128 is the order of their number): LORA_E_SHAPE if not.
 *
 * Asynchrony, errors and thread safety are lora.h's: calls are enqueued on the
 * caller's stream, allocate nothing (lora_attn_create does), copy nothing to
 * the host and never wait.  All may be recorded in a HIP graph; what is passed in host
 * arrays is fixed in the record.  The same inputs give the same bits.
 */
#ifndef LORA_KV_H
#define LORA_KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* The cache of every layer (HOST structure; k and v are DEVICE pointers). */
typedef struct {
    void* k;
    void* v;
    int64_t layer_stride, page_stride, head_stride, row_stride; /* elements */
    int32_t dtype;              /* LORA_F16 or LORA_BF16              */
    int32_t n_layers, n_pages, n_kv_heads;
    int32_t page_rows;          /* tokens per page                    */
    int32_t head_dim;
} lora_kv_cache_t;

/* The sequences of a step (HOST structure of DEVICE pointers). */
typedef struct {
    const int32_t* tables;      /* [n_seqs, ld_table]: page ids        */
    const int32_t* lens;        /* [n_seqs]: tokens, this step's included (lora_kv_grow_step's step_lens) */
    int32_t n_seqs, ld_table;
    int32_t max_len;            /* no length above this is read: sizes the launch
                                   (and bounds lora_kv_grow_step, or is ld_table * page_rows) */
} lora_kv_seqs_t;

/* Who holds which page (HOST structure of DEVICE pointers).  refs[p] counts
 * the sequences that hold page p; 0 is a free page.  A sequence holds the
 * pages of its first ceil(len / page_rows) table entries (entries outside
 * [0, n_pages) hold none); further entries have no meaning. */
typedef struct {
    int32_t* tables;            /* [n_seqs, ld_table], below 2^31 in all */
    int32_t* lens;              /* [n_seqs]                            */
    int32_t* refs;              /* [n_pages]                           */
    int32_t n_seqs, ld_table, n_pages;   /* n_pages <= 2^30            */
    int32_t page_rows;
} lora_kv_book_t;

/*
 * The rows' keys and values into the cache.  Rows seg_offset[s] ..
 * seg_offset[s + 1] of k_new and v_new [n_rows, ld] (heads one after the
 * other, head_dim elements each) are the last tokens of sequence s: row i of
 * a segment of n rows goes to token lens[s] - n + i.  seg_offset is a DEVICE
 * array [n_seqs + 1], nondecreasing from 0, or NULL for one row per sequence
 * (n_rows == n_seqs).  Rows at negative positions, past the table or on no
 * page are not stored.  k_new and v_new must not overlap the cache.
 */
int lora_kv_append(const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s, const int32_t* seg_offset,
                   int32_t n_rows, const void* k_new, int64_t ldk, const void* v_new, int64_t ldv, void* stream);

/*
 * What attention launches share: counters and float32 partial results of
 * key ranges that several workgroups read (about 70 MB of device memory, the
 * same for every call).  Creation allocates, and waits for `stream`; it
 * refuses a capturing stream.  Launches that share one handle must be ordered
 * on one stream.  Destroying it frees the memory: no launch may still use it.
 */
typedef struct lora_attn_s* lora_attn_t;
int lora_attn_create(lora_attn_t* out, int device, void* stream);
int lora_attn_destroy(lora_attn_t a);

/*
 * Attention of one new token per sequence: q [n_seqs, ldq] and out
 * [n_seqs, ldo], heads one after the other; row s is at position lens[s] - 1
 * (its key and value are in the cache).  The visible tokens are divided evenly
 * over the chip whatever the lengths; a sequence's head that several
 * workgroups read is joined by the last of them.
 */
int lora_attn_decode(lora_attn_t a, const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s,
                     int32_t n_heads, const void* q, int64_t ldq, void* out, int64_t ldo, float scale,
                     int32_t window, int32_t n_sinks, void* stream);

/*
 * Attention of prompt segments: rows seg_offset[s] .. seg_offset[s + 1] of q
 * and out [n_rows, ld] are the last tokens of sequence s (row i of n at
 * position lens[s] - n + i), so a prompt may come in chunks behind what is
 * cached already.  seg_offset is a DEVICE array [n_seqs + 1], nondecreasing
 * from 0 to n_rows.  Rows of no segment are not written.
 */
int lora_attn_prompt(lora_attn_t a, const lora_kv_cache_t* c, int32_t layer, const lora_kv_seqs_t* s,
                     const int32_t* seg_offset, int32_t n_rows, int32_t n_heads, const void* q, int64_t ldq,
                     void* out, int64_t ldo, float scale, int32_t window, int32_t n_sinks, void* stream);

/* Device workspace of lora_kv_grow, _fork (with or without _step) and _compact for
 * this book, in bytes; any contents, 16-byte aligned, overwritten. */
int lora_kv_workspace_bytes(const lora_kv_book_t* b, size_t* bytes);

/*
 * lens[s] += add[s] (DEVICE array [n_seqs]; entries below 1 are read as 0) with
 * the pages that this takes: free pages in ascending order go to sequences in
 * ascending order.  A sequence whose table is too short stays as it is and
 * takes nothing.  From the first whose pages exceed the free ones that are
 * left, sequences that need a page stay as they are (a short one does not
 * overtake), and those that need none still grow.  info (DEVICE [2], may be
 * NULL): pages taken, sequences that stayed.
 */
int lora_kv_grow(const lora_kv_book_t* b, const int32_t* add, int32_t* info, void* ws, size_t ws_bytes,
                 void* stream);

/*
 * The same for the rows of one step, with what the step has to know.  No length
 * passes max_len (at most ld_table * page_rows; a sequence that would pass it
 * stays as it is).  step_lens (DEVICE [n_seqs], not the book's lens) gets
 * the new length of each sequence that grew, and 0 for one that stayed or had
 * nothing to add.
 *
 * A sequence that stayed has no room for its rows: with lens as the lengths of the
 * step, lora_kv_append would store them over its last tokens, which other
 * sequences may share.  With step_lens as the lengths (lora_kv_seqs_t.lens) such rows
 * are not stored and attention gives them zeros, also in a recorded step, where the host cannot
 * look at info in between.  The rows of a sequence in that step are at most add[s].
 */
int lora_kv_grow_step(const lora_kv_book_t* b, const int32_t* add, int32_t max_len, int32_t* step_lens, int32_t* info,
                      void* ws, size_t ws_bytes, void* stream);

/*
 * Sequence children[i] becomes a copy of parents[i] (HOST arrays of n, read
 * during the call; the children distinct and none a parent).  What a child
 * held is released first.  Full pages are shared; the rows of a partly filled
 * last page are copied, in every layer, into a page of the child's own: free
 * pages in ascending order go to the pairs in the order given.  A child whose page
 * does not fit is left empty.  So the tokens that a later grow gives never lie in a
 * shared page; for a sequence that got none, see lora_kv_grow_step.
 * info (DEVICE [2], may be NULL): pages taken, children left empty.
 */
int lora_kv_fork(const lora_kv_cache_t* c, const lora_kv_book_t* b, int32_t n, const int32_t* parents,
                 const int32_t* children, int32_t* info, void* ws, size_t ws_bytes, void* stream);

/* The same between steps that use step_lens: the children's become 0, so that they have
 * no rows before the next lora_kv_grow_step. */
int lora_kv_fork_step(const lora_kv_cache_t* c, const lora_kv_book_t* b, int32_t n, const int32_t* parents,
                      const int32_t* children, int32_t* step_lens, int32_t* info, void* ws, size_t ws_bytes,
                      void* stream);

/* Sequences seqs[0 .. n) (HOST array, distinct) release their pages: length 0,
 * table entries -1. */
int lora_kv_free(const lora_kv_book_t* b, int32_t n, const int32_t* seqs, void* stream);

/* Every sequence releases the pages in which no row still to come (position
 * len or later) sees a token with this window and these sinks; their table
 * entries become -1.  window >= 1.  Between a step and the next grow: once the lengths
 * have grown, the step's own rows are no longer to come. */
int lora_kv_trim(const lora_kv_book_t* b, int32_t window, int32_t n_sinks, void* stream);

/* Pages src[i] to dst[i], every layer, all rows (HOST arrays of n; the dst
 * distinct and none a src). */
int lora_kv_copy(const lora_kv_cache_t* c, int32_t n, const int32_t* src, const int32_t* dst, void* stream);

/*
 * The L pages in use move to ids [0, L): the pages in use from L on, in
 * ascending order, into the free ones below L, in ascending order, in every
 * layer (the others stay; what the pages from L on hold is not changed).
 * tables_out [n_seqs, ld_table] and refs_out [n_pages] receive the book for
 * the new ids and may be the book's own arrays, which are not written
 * otherwise; table entries without a page, and those past a sequence's
 * length, become -1.  info (DEVICE [2], may be NULL): L, pages moved.
 */
int lora_kv_compact(const lora_kv_cache_t* c, const lora_kv_book_t* b, int32_t* tables_out, int32_t* refs_out,
                    int32_t* info, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LORA_KV_H */
