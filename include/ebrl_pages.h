/*
 * ebrl_pages -- prefixes that grow: keys and values of many sequences in pages, and the operators that work on them.
 *
 * Action generation (ebrl_actgen.h, ebrl_prefix8.h) takes an environment's prefix as the backbone left it.  This is
 * where the backbone leaves it while an episode runs: an environment's observations arrive in chunks (one token, or
 * thousands), every chunk attends to all that came before, rollouts that start from one state share what they have in
 * common (paper section 4.2: environments progress independently, in groups that start and end at different times), and a
 * reset gives everything back.  A page holds page_tokens consecutive tokens of a sequence, for all layers:
 *
 *     elements  dtype  [kv_layers][2][n_kv_heads][page_tokens][head_dim]     plane 0 = K, plane 1 = V
 *     mask      uint32 [page_tokens / 32]                                    bit t % 32 of word t / 32: queries see token t
 *
 * padded to a multiple of 128 bytes (ebrl_pages_page_bytes).  A pool is n_pages pages in a row, 16-byte aligned.  A table names the
 * pages of a call's sequences: DEVICE int32, row i of it at table + i * table_stride, token t of sequence i lies in page
 * table[i][t / page_tokens].  An entry outside 0 .. n_pages - 1 says that the page is not there: its tokens are not seen, nothing is read from or
 * written to it.  Where all lengths are 0 the table may be NULL.  Lengths and numbers of tokens are host arrays, checked and copied before the call returns; pages are looked up
 * on the device.  Rows of a page that no token of a sequence has been written to may hold anything, NaN included.
 *
 * Sequences of a call may share pages that are only read.  append, copy and whatever else writes a page that another call uses are ordered by the
 * caller (one stream, or events).  The operators are asynchronous on `stream` and touch no memory but their arguments; the current
 * device must be the one that holds them.  All arguments are checked before anything is enqueued; a status other than EBRL_OK comes
 * with a text (ebrl_pages_last_error).  All operators may be captured into a CUDA graph (lengths, counts and pointers are then those of the
 * capture; pages are looked up at the replay).  sm_quota as in ebrl_actgen_submit: 0 = all SMs, else persistent grids of at most
 * that many CTAs.
 */
#ifndef EBRL_PAGES_H_
#define EBRL_PAGES_H_

#include "ebrl_actgen.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int32_t kv_layers;    /* 1 .. 4096                                                                 */
    int32_t n_kv_heads;   /* 1 .. 4096                                                                 */
    int32_t head_dim;     /* 32, 64 or 128                                                             */
    int32_t page_tokens;  /* 32, 64, 128 or 256                                                        */
    int32_t dtype;        /* EBRL_F32 or EBRL_BF16                                                     */
} ebrl_pages_layout_t;

/* Bytes of one page; 0 for a layout that is not covered. */
uint64_t ebrl_pages_page_bytes(const ebrl_pages_layout_t *layout);

/* Text of the last error of this thread's ebrl_pages calls; valid until its next one. */
const char *ebrl_pages_last_error(void);

/* Waits of the kernels on their own copies are bounded (4 s).  When one runs out, the rows that were not finished (of cut sequences, all rows that wanted a piece)
 * are left as they are, and the kernel notes it; this call waits for the current device's work, returns EBRL_ERR_TIMEOUT if that happened on it since the last call, and
 * forgets it. */
ebrl_status_t ebrl_pages_check(void);

/* Tests of that path only: with limit_ns > 0 (2 s at most) this thread's later attend calls issue no copies in the kernels that wait for them, so that the
 * waits run out after limit_ns and the kernels return; 0 ends it. */
void ebrl_pages_test_drop_copies(uint64_t limit_ns);

/* Writes the keys and values of new tokens of one layer.
 *   new_tokens  host [n], 0 .. len[i]: sequence i's new tokens are its last ones, positions len[i] - new_tokens[i] .. len[i] - 1
 *   len         host [n]: its length with them, at most table_stride * page_tokens
 *   k, v        DEVICE, layout dtype: the new tokens of sequence 0, then those of sequence 1, ...; token r, head h, element j at
 *               k + r * k_stride + h * head_dim + j (v likewise); addresses and strides multiples of 16 bytes; the stride of a single token is not looked at
 *   mask        NULL (all visible), or DEVICE bytes, one per new token in the same order: 0 hides it
 * Sets the tokens' mask bits, too (every layer's call writes the same ones).  A hidden token's rows become zeros whatever k and v hold.
 * Other tokens' rows and bits are left as they were.  Sequences of one call that write must not share the pages they write. */
ebrl_status_t ebrl_pages_append(const ebrl_pages_layout_t *layout, void *pool, int32_t n_pages, int32_t n, const int32_t *table,
                                int64_t table_stride, const int32_t *new_tokens, const int32_t *len, int32_t layer, const void *k, int64_t k_stride,
                                const void *v, int64_t v_stride, const uint8_t *mask, int32_t sm_quota, void *stream);

/* Softmax attention of each sequence's new tokens over the sequence, of one layer:
 *     out = softmax(scale * q k^T) v,   lse = log sum_t exp(scale * q k_t)
 * over the tokens t that query j of sequence i (position p = len[i] - new_tokens[i] + j) sees: t < len[i], its mask bit is set, its page is there, and
 *   causal      != 0: t <= p.  0: every one (tokens of an observation that see one another, or queries that are no tokens of the sequence: cross attention)
 *   window      > 0 (only with causal): t > p - window.  0, or any that is not below the longest length: no limit
 *   new_tokens  host [n], >= 0: number of queries (usually appended before; more than len[i] is allowed: with causal, those at negative positions see nothing)
 *   q           DEVICE, layout dtype, queries packed like the tokens of append: query r, head a at q + r * q_stride + a * head_dim
 *               (stride in elements, >= 0, a multiple of 16 bytes; not looked at for a single query).  Head a reads key/value head a / (n_heads / n_kv_heads).
 *   n_heads     a multiple of n_kv_heads, at most 65536, and n_heads / n_kv_heads at most 128
 *   out         DEVICE, layout dtype, laid out like q with its own stride; may be q itself.  Rows behind the last query are left as they were.
 *   lse         DEVICE fp32 [queries][n_heads], or NULL
 *   scale       softmax scale, of at most 2.3e38 either way (usually 1 / sqrt(head_dim)); scores, too, may be as large as that
 * A row that sees no token gives out = 0 and lse = -inf.  Keys and values of tokens that some query of the call sees must be finite; those of hidden
 * tokens, of missing pages and behind the length may hold anything.
 * Where sequences are few, a sequence is divided among warps, which are joined in shared memory, and a long one is cut into pieces besides, which a
 * second kernel joins.  split_tokens = 0 lets the call choose (a sequence's last bits can then depend on its company); -1 never divides or cuts (a
 * sequence's result then depends on nothing but itself); a positive multiple of 128 cuts every longer sequence into pieces of that many tokens.  The pieces' partial results need
 * ebrl_pages_attend_workspace bytes (of the same arguments) of DEVICE memory, 16-byte aligned, that no other call in flight uses (two captured graphs that
 * may run at once need one each); 0 bytes: workspace may be NULL.
 * bf16: products of bf16 operands, weights rounded to bf16.  fp32: operands and weights in two tf32 terms, three products
 * (21 bits, fewer of values below 2^-118; numbers next to the largest one, from 2^128 (1 - 2^-12) on, are no finite first terms).  Sums and softmax statistics are fp32.  Sums of weights times values
 * are divided by the sum of the weights at the end; until then a row's are at most 2^16, or the number of tokens that it sees if that is more, times the largest value,
 * so that values above 2^112 (5e33; 2^128 / tokens if that is less; with many bf16 rows whose scores are 2^26 and more up to 2^32 times less) may overflow. */
uint64_t ebrl_pages_attend_workspace(const ebrl_pages_layout_t *layout, int32_t n, const int32_t *new_tokens, const int32_t *len, int32_t n_heads,
                                     int32_t causal, int32_t window, int32_t split_tokens, int32_t sm_quota);
ebrl_status_t ebrl_pages_attend(const ebrl_pages_layout_t *layout, const void *pool, int32_t n_pages, int32_t n, const int32_t *table,
                                int64_t table_stride, const int32_t *new_tokens, const int32_t *len, int32_t layer, const void *q, int64_t q_stride,
                                int32_t n_heads, void *out, int64_t o_stride, float *lse, float scale, int32_t causal, int32_t window,
                                int32_t split_tokens, void *workspace, uint64_t workspace_bytes, int32_t sm_quota, void *stream);

/* Copies pages: page from[i] of src to page to[i] of dst (pools of one layout; dst is src, or memory that does not overlap it).
 *   tokens  NULL (all), or host [n], 0 .. page_tokens: only so many first tokens of each page, with their mask bits; the others are left as they were
 * Pages written must differ from one another and, within one pool, from the pages that are read. */
ebrl_status_t ebrl_pages_copy(const ebrl_pages_layout_t *layout, const void *src, int32_t src_pages, void *dst, int32_t dst_pages, int32_t n,
                              const int32_t *from, const int32_t *to, const int32_t *tokens, int32_t sm_quota, void *stream);

/* Writes sequences out as planes, the form that ebrl_actgen_submit and ebrl_prefix8_quantize take.
 *   planes      host [n] of DEVICE pointers; sequence i: element (layer l, plane p, token t, column c) goes to
 *               planes[i][((l * 2 + p) * plane_rows[i] + t) * row_stride + c], c = head * head_dim + j; 16-byte aligned, layout dtype
 *   len         host [n]; plane_rows host [n], at least len[i], NULL: len; row_stride as in ebrl_prefix8_quantize, 0: n_kv_heads * head_dim
 *   mask        NULL, or host [n] of DEVICE pointers (each may be NULL) to len[i] bytes: 1 where the token is visible, else 0
 * Rows of hidden tokens and of missing pages become zeros.  (Planes know no hidden tokens: quantize takes them along with the mask.)
 * Rows behind the length are left as they were.  Planes of one call must not overlap. */
ebrl_status_t ebrl_pages_gather(const ebrl_pages_layout_t *layout, const void *pool, int32_t n_pages, int32_t n, const int32_t *table,
                                int64_t table_stride, const int32_t *len, void *const *planes, const int32_t *plane_rows, int64_t row_stride,
                                uint8_t *const *mask, int32_t sm_quota, void *stream);

/* ---- the book: which page belongs to whom (host only, no device needed) ------------------------------------------------
 * Sequences are numbered 0 .. max_sequences - 1; each has a length and pages.  A page may belong to several sequences (after a fork); it is free
 * when the last of them lets go.  Free pages are handed out lowest number first.  Calls change all that they were asked to or, on an error, nothing.  One thread at a time
 * per book.  Functions that make data move return the moves (arrays as ebrl_pages_copy takes them); the caller enqueues that copy before anything that
 * relies on it, and reads the tables anew. */
typedef struct ebrl_pages_book *ebrl_pages_book_t;

ebrl_status_t ebrl_pages_book_create(int32_t n_pages, int32_t page_tokens, int32_t max_sequences, ebrl_pages_book_t *out);
ebrl_status_t ebrl_pages_book_clone(ebrl_pages_book_t book, ebrl_pages_book_t *out);
void ebrl_pages_book_destroy(ebrl_pages_book_t book);

/* Lengthens sequences to len[i] >= their length (a sequence may be named once), in the order of the call.  Where the first new token falls into a page that is shared, the
 * sequence gets its own copy of that page: a move of the tokens it has there.  from, to, tokens have room for n moves; *n_moves says how many there are.
 * EBRL_ERR_NOMEM: not enough free pages. */
ebrl_status_t ebrl_pages_book_extend(ebrl_pages_book_t book, int32_t n, const int32_t *seqs, const int32_t *len, int32_t *from, int32_t *to, int32_t *tokens,
                                     int32_t *n_moves);
/* Sequence to[i], empty before, becomes from[i]'s twin: the same length and pages.  Nothing is copied until one of them is extended. */
ebrl_status_t ebrl_pages_book_fork(ebrl_pages_book_t book, int32_t n, const int32_t *from, const int32_t *to);
/* Shortens sequences to len[i] <= their length (0: frees them); pages behind it are let go. */
ebrl_status_t ebrl_pages_book_shorten(ebrl_pages_book_t book, int32_t n, const int32_t *seqs, const int32_t *len);
/* Moves pages in use with the highest numbers to the lowest free ones until they are the first ones of the pool, or `room` moves are made. */
ebrl_status_t ebrl_pages_book_compact(ebrl_pages_book_t book, int32_t room, int32_t *from, int32_t *to, int32_t *tokens, int32_t *n_moves);

/* Host table of sequences: row i at out + i * stride, -1 behind a sequence's last page.  stride >= the most pages of one; where it is 0, out may be NULL. */
ebrl_status_t ebrl_pages_book_table(ebrl_pages_book_t book, int32_t n, const int32_t *seqs, int32_t *out, int64_t stride);
/* Length of a sequence, -1 if there is no such; pages in use (each counted once). */
int32_t ebrl_pages_book_len(ebrl_pages_book_t book, int32_t seq);
int32_t ebrl_pages_book_used(ebrl_pages_book_t book);

#ifdef __cplusplus
}
#endif
#endif /* EBRL_PAGES_H_ */
