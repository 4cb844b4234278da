/*
 * ssd_pages.h — a paged cache in 8 bits for a batch of sequences, and the
 * attention that reads it.
 *
 * ssd.h verifies the speculated tokens of one sequence over a dense cache.  A
 * batch of sequences, each somewhere else, that share prompts, grow by what is
 * accepted of each step (Sec. 2.3, 3.1 of arXiv 2308.04623) and end at any time
 * keeps its keys and values in pages of a pool instead:
 *   ssd_paged_attn    attention of every sequence's new rows (a chain or a tree's
 *                     nodes) over its cached rows and each other, optionally over a
 *                     window of them with the first few ("sinks") only;
 *   ssd_pages_take, ssd_pages_store, ssd_pages_load
 *                     pages for a prompt, its rows into them and back;
 *   ssd_pages_commit  appends the accepted path of each sequence's new rows;
 *   ssd_pages_fork    slots become copies of others (sharing pages) or are freed;
 *   ssd_pages_compact moves the pages in use to the front of the pool.
 *
 * Where a sequence's rows are.  With R0 = page_rows, the first
 * floor(length / R0) R0 of a sequence's `length` rows lie in pages, 8 bits an
 * element with a scale for each page, head, and keys or values; the others, of its open
 * page, lie in the batch's tail in the model's type, the row of position p at
 * p mod tail_rows.  A page is made once, from exact rows, when it is full: its scale knows
 * no rejected row, and pages never change, so sequences share them freely.
 * The new rows of a step are kept apart from both (Sec. 3.1) until they are committed.
 *
 * A page's block (R0 rows of one layer, head, and keys or values): a is the largest magnitude in
 * it, top is 127 (SSD_PAGE_INT8) or 448 (SSD_PAGE_E4M3, a float of 4 exponent
 * and 3 mantissa bits without infinities).  In float32, every operation rounded to nearest even:
 *   r = top / a, code = the code nearest to clamp(x r, -top, top), scale = a / top,
 * and an element reads as scale code.  a < 2^-100: scale and codes 0; a row that is
 * not finite: scale NaN.  SSD_PAGE_INT8 stores code + 128.  Bytes lie in
 * matrix-core order: with rows 32 a + 16 b + m of the keys and 32 a + 16 b + 4 g + r of
 * the values (every index running from the left, slowest, to the right)
 *   keys, head_dim >= 64  [a][b][head_dim / 64: c][g: 4][m: 16][i: 16], dim 64 c + 16 g + i
 *   keys, head_dim 32     [a][g: 4][m: 16][b][i: 8],                  dim 8 g + i
 *   values                [a][head_dim / 32: c][g: 4][m: 16][u: 2][b][r: 4], dim 32 c + 16 u + m
 *
 * The conventions of ssd.h and ssd_ops.h hold: device pointers are the caller's, work
 * goes onto the caller's stream, nothing synchronises the host or allocates, every
 * argument check runs on the host before anything is enqueued; calls that share a
 * workspace, or change what another reads, are ordered by the caller.  All can be captured into a
 * HIP graph.  Results are bitwise the same from run to run.  What tables, lengths,
 * paths and ids on the device hold is checked there: a page outside the pool or a row outside
 * its buffer is never read or written (what happens instead is said at each call).
 */
#ifndef SSD_PAGES_H
#define SSD_PAGES_H

#include "ssd_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SSD_PAGE_INT8 = 0, SSD_PAGE_E4M3 = 1 } ssd_page_code;

/* The pool.  data: n_layer n_page n_kv_head 2 page_rows head_dim bytes (16-byte
 * aligned), [layer][page][head][keys, values][block]; scale: [layer][page][head][2]
 * (8-byte aligned).  page_rows 32, 64 or 128; head_dim 32, 64 or 128; 1 <= n_layer <= 4096,
 * 1 <= n_page <= 2^20, 1 <= n_kv_head <= 1024. */
typedef struct {
  ssd_page_code code;
  int32_t n_layer, n_page, n_kv_head, page_rows, head_dim;
  void *data;
  float *scale;
} ssd_page_pool;

/* The batch's sequences, on the device: table [n_seq][n_col] (table_ld entries from
 * row to row), column c the page of rows c page_rows ..; -1: none.  length [n_seq]; below 0: a
 * slot without a sequence.  refs [n_page]: how many table entries name a page; 0: it is
 * free.  1 <= n_seq <= 4096, 0 <= n_col, n_col page_rows < 2^30. */
typedef struct {
  int32_t n_seq, n_col;
  int64_t table_ld;
  int32_t *table, *length, *refs;
} ssd_page_seqs;

/* Rows in the model's type.  Strides count elements; the head_dim elements of a
 * row lie side by side.  Pointers are 16-byte aligned, strides multiples of 16 bytes,
 * not negative.  Where rows are written they do not overlap: sorted by their strides, each
 * dimension steps over all that the smaller ones reach.
 *   tail          element (l, b, g, j, i) at l layer + b seq + g head + j row + i,  j < rows
 *   new rows      element (l, b, t, g, i) the same with t row,                      t < rows
 *   pages' rows   element (l, n, g, j, i) the same with n seq,                      j < page_rows */
typedef struct {
  ssd_dtype dtype;
  int32_t rows;
  int64_t layer, seq, head, row;
} ssd_rows_desc;

/* Attention of the n_query new rows of each sequence in one layer.  New row t of a
 * sequence of `length` rows sits at position length + depth, with depth = t for a chain (anc
 * NULL); for a tree anc (device, [n_seq][n_query]) says which new rows row t sees, bit i row i
 * (its ancestors and itself, as ssd_tree_prep's masks), and its depth is their number less one.  It sees
 *   cached rows j < length: all of them if window is 0, else those with
 *     j > position - window or j < sinks (n_query <= window, so that what it
 *     sees of the new rows is inside its window);
 *   new rows i <= t, or those of anc.
 * Head h reads the keys and values of head h / (n_head / n_kv_head).  out is the softmax of scale
 * q.k over the seen rows times their values; a query that sees no row (anc 0 and
 * nothing cached), or of a slot without a sequence, gives 0, and lse -infinity.  Rows that no query of
 * a sequence sees may hold anything (in pages of which it sees other rows, anything but e4m3's codes of NaN, which
 * ssd_pages_store never writes), and a cached row whose table entry is no page of the
 * pool is not seen.  A row whose score is -infinity counts as one that is not seen; a score
 * that is NaN or +infinity makes the query's out and lse NaN; an element that is not finite
 * among the values of a seen row makes that element of out NaN.  A page's scale that is not finite reads as NaN.
 * lse, if not NULL: float32 [n_seq][n_query][n_head], the log of the sum of exponentials of
 * the seen scores.
 *   q, out: element (b, t, h, i) at b seq + t row + h head + i.  dtype, of q, tail, new rows and
 * out, SSD_F32 or SSD_BF16; 1 <= n_query <= 64; n_head a multiple of n_kv_head and at most
 * 1024; tail_rows >= page_rows; pointers and strides as ssd_rows_desc says; out shares no
 * element with an input (it may lie between its rows, heads or tokens, where a step that divides the larger
 * ones of both tells them apart).  window and sinks >= 0.
 * Scores, softmax and sums are float32; 8-bit codes are multiplied exactly.  For the product with the cached values bfloat16 calls
 * hold the weights exp(x - max) in 20 bits or to 2^-24 of the largest weight of the same 32 rows (32 a .. 32 a + 31), float32
 * calls in 22 bits or to 2^-39 of it, and queries in 33 bits; for that with other values bfloat16 calls hold them in 16 bits.
 * No page takes bits from another's, whatever its scale.  Sums are finite where their quotient is (up to scores of 2^29;
 * beside seen values of 2^80 or scales of 2^48, weights are held in 19 bits).
 * Errors: SSD_E_INVALID_ARG, SSD_E_CAPACITY (workspace too small or not 16-byte aligned, or more than 2^24 workgroups),
 * SSD_E_UNSUPPORTED (page_rows, head_dim, alignment), SSD_E_DEVICE. */
typedef struct {
  ssd_dtype dtype;
  int32_t layer, n_query, n_head;
  int32_t tail_rows;
  int32_t window, sinks;
  float scale;
  int64_t q_seq, q_row, q_head;
  int64_t out_seq, out_row, out_head;
  int64_t tail_seq, tail_head, tail_row;
  int64_t new_seq, new_row, new_head;
} ssd_paged_attn_desc;

/* Bytes of workspace for a call with these shapes (0: none, it may be NULL). */
ssd_status ssd_paged_attn_workspace(const ssd_page_pool *pool, const ssd_page_seqs *seqs,
                                    const ssd_paged_attn_desc *a, size_t *bytes);
ssd_status ssd_paged_attn(const ssd_page_pool *pool, const ssd_page_seqs *seqs, const ssd_paged_attn_desc *a,
                          const void *q, const void *k_tail, const void *v_tail, const void *k_new,
                          const void *v_new, const int64_t *anc, void *out, float *lse, void *workspace,
                          size_t workspace_bytes, void *stream);

/* Rows into pages: block (l, n, g) of k and v becomes that of page ids[n] (device) in layer
 * first_layer + l, l < n_layer of the call, n < n.  Ids outside the pool are passed over.  A page that
 * ids names twice gets a block of either for each head, and keys or values: name it once.
 * ssd_pages_load is the way back: k and v get the values that the pages stand for, rounded once to
 * dtype; ids outside the pool give zeros.  rows of the desc is not used.  n_layer and n >= 0, n at most 2^20; 0
 * does nothing.  k and v of ssd_pages_load lie apart, one behind the other.
 * Errors: SSD_E_INVALID_ARG, SSD_E_UNSUPPORTED, SSD_E_DEVICE. */
ssd_status ssd_pages_store(const ssd_page_pool *pool, const int32_t *ids, int32_t n, int32_t first_layer,
                           int32_t n_layer, const ssd_rows_desc *d, const void *k, const void *v, void *stream);
ssd_status ssd_pages_load(const ssd_page_pool *pool, const int32_t *ids, int32_t n, int32_t first_layer,
                          int32_t n_layer, const ssd_rows_desc *d, void *k, void *v, void *stream);

/* Bytes of workspace for ssd_pages_take, _commit and _compact (16-byte aligned). */
ssd_status ssd_pages_workspace(const ssd_page_pool *pool, const ssd_page_seqs *seqs, size_t *bytes);

/* Pages for whole blocks of rows (a prompt's) that the caller stores.  Slot b with count[b] >= 0
 * (device) gets count[b] pages behind those it has: the lowest free ones, slots in order; its
 * length, below 0 counting as 0, grows by count[b] page_rows and got[b] (device) is
 * count[b].  got[b] is -1, and nothing of the slot changes, where count[b] < 0, the length is no multiple of
 * page_rows, the table has too few columns or too few pages are free (counting those that
 * slots before it asked for, whether they got them or not).
 * Errors: SSD_E_INVALID_ARG, SSD_E_CAPACITY (workspace), SSD_E_DEVICE. */
ssd_status ssd_pages_take(const ssd_page_pool *pool, const ssd_page_seqs *seqs, const int32_t *count, int32_t *got,
                          void *workspace, size_t workspace_bytes, void *stream);

/* Appends accepted new rows: rows path[b][0 .. path_len[b]-1] (device; path_ld entries from row to row, at
 * most max_path of them, and no more than k_new has rows, count, and none from the first outside [0, k_new's rows)
 * on) of sequence b become its rows length[b] .., in every layer, and length[b] grows by their number (n).
 * Pages that get full by it are taken as by ssd_pages_take and made from the tail's and the new
 * rows; rows behind them join the tail, whose other rows stay as they are.  full[b] (device): how many pages got full;
 * -1 where pages or columns of the table did not suffice, and nothing of the sequence changes; 0 for a slot without one.
 * window > 0: then the pages of the sequence that no later row sees (as ssd_paged_attn
 * with this window and these sinks: all of its rows are at sinks or behind, and at most length - window)
 * are given back: their entries become -1.
 * Tail and new rows have one dtype; tail rows >= page_rows + new rows - 1; 1 <= new rows <= 64;
 * layers are the pool's.  Buffers share no bytes.
 * Errors: SSD_E_INVALID_ARG, SSD_E_CAPACITY (workspace, or slots and layers for 2^24 workgroups), SSD_E_UNSUPPORTED,
 * SSD_E_DEVICE. */
ssd_status ssd_pages_commit(const ssd_page_pool *pool, const ssd_page_seqs *seqs, const ssd_rows_desc *tail,
                            void *k_tail, void *v_tail, const ssd_rows_desc *fresh, const void *k_new,
                            const void *v_new, const int32_t *path, int64_t path_ld, int32_t max_path,
                            const int32_t *path_len, int32_t window, int32_t sinks, int32_t *full, void *workspace,
                            size_t workspace_bytes, void *stream);

/* Copies and ends of sequences.  parents (device, [n_seq]): slot b with parents[b] = b stays as it is; with
 * parents[b] = s, where parents[s] = s, it becomes a copy of slot s: it gives back its pages, names
 * s's, and takes s's length and open rows (n_layer layers of the tail); with any other value it ends: its pages are
 * given back, its length becomes -1.  n_page and page_rows are the pool's, n_layer, n_kv_head and head_dim the
 * tail's.
 * Errors: SSD_E_INVALID_ARG, SSD_E_UNSUPPORTED, SSD_E_DEVICE. */
ssd_status ssd_pages_fork(const ssd_page_seqs *seqs, int32_t n_page, int32_t page_rows, const int32_t *parents,
                          const ssd_rows_desc *tail, int32_t n_layer, int32_t n_kv_head, int32_t head_dim,
                          void *k_tail, void *v_tail, void *stream);

/* Moves the pages in use to 0 .. *used - 1 (device): with U pages in use, the i-th page in
 * use from U on goes to the i-th free page below U, in every layer, and refs and table follow.  The pages
 * from U on are free then and the pool may be cut there.
 * Errors: SSD_E_INVALID_ARG, SSD_E_CAPACITY (workspace), SSD_E_DEVICE. */
ssd_status ssd_pages_compact(const ssd_page_pool *pool, const ssd_page_seqs *seqs, int32_t *used, void *workspace,
                             size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
