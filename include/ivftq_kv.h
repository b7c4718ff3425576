/*
 * ivftq_kv.h -- paged key-value cache for AMD MI355X (gfx950), part of libivftq.
 *
 * A model that answers keeps the keys and values of its tokens.  They are rows like those of an index: the rotation Pi
 * and the Lloyd-Max levels of ivftq.h depend on (b, d) only, so a cache can hold them in the same codes without training,
 *     gamma = |x| ; rho = Pi x / gamma ; code_j = level next to rho_j ; x^ = gamma Pi^T C[code]
 * and attention takes its products from the codes as the search does,
 *     <q, k^> = gamma_k <Pi q, C[code_k]>      sum_t p_t v^_t = Pi^T sum_t (p_t gamma_t) C[code_t].
 * The same pages can hold the rows in 16 bits instead.
 *
 * Conventions
 *   - The caller owns every buffer: pool, table, lengths, reference counts, workspace.  Device pointers unless stated.
 *     Nothing is kept from one call for the next.
 *   - Calls are asynchronous on `stream` (a hipStream_t passed as void*, NULL = the default stream), allocate nothing, issue
 *     kernel launches only and may be recorded into a HIP graph.  Buffers and stream belong to the current device.
 *   - Arguments that the host can see are checked before any launch; every call returns an ivftq_status and
 *     ivftq_last_error() has the message.  What only the device sees (table entries, lengths, starts, rows of a list) is
 *     bounded by the kernels: an entry that names no page of the pool holds no visible token and takes no row, a length
 *     counts up to columns * page, a row number outside the table is passed over.
 *
 * Pool: `pages` records, one after the other; a record holds for each key-value head, one after the other (page tokens t,
 * d coordinates j):
 *   IVFTQ_KV_F16, IVFTQ_KV_BF16   K[t][j], then V[t / 8][j][t % 8], 16 bits each
 *   IVFTQ_KV_CODE4                the two blocks in 4 bits, low half of a byte first (bit 3: sign, bits 0-2: magnitude m,
 *                                 level levels[8 + m] or its negative), in the coordinates of the rotated row; then the
 *                                 keys' norms and the values' norms, page float16 each
 * (values stand in groups of eight tokens because a matrix instruction takes eight neighbouring ones of one coordinate.)
 */
#ifndef IVFTQ_KV_H
#define IVFTQ_KV_H

#include "ivftq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { IVFTQ_KV_F16 = 0, IVFTQ_KV_BF16 = 1, IVFTQ_KV_CODE4 = 2 };

/* One layer's cache as a call sees it.  d: 64, 96, 128, 192 or 256; page: a power of two, 16 to 1024; heads: key-value
 * heads, 1 to 1024.  Sequence b's token t is token t % page of page table[b * table_stride + t / page].  lengths[b]: tokens
 * of the sequence, those of the present step included.  rotation (device, d x d, 16-byte aligned) and levels (16 values,
 * ascending, levels[15 - i] == -levels[i], as ivftq_build_codebook(4, d, ...) gives them) are read for IVFTQ_KV_CODE4 only.
 * pool is 16-byte aligned.
 * asked and granted (device, batch numbers each, or both NULL): counts and results of the present step's ivftq_kv_reserve.
 * ivftq_kv_append writes no row of a sequence with granted[b] < asked[b]: its length does not count them, so that they would
 * fall on the tokens before them.  No other call reads the two. */
typedef struct ivftq_kv_cache {
    void* pool;
    const int32_t* table;
    const int32_t* lengths;
    const float* rotation;
    int64_t pages;
    int64_t table_stride;
    int32_t batch;
    int32_t columns;
    int32_t format;
    int32_t page;
    int32_t heads;
    int32_t d;
    float levels[16];
    const int32_t* asked;
    const int32_t* granted;
} ivftq_kv_cache;

/* Rows of the present step: row r, head h, coordinate j at data[r * row_stride + h * head_stride + j] (strides in elements,
 * multiples of 8; data 16-byte aligned).  type: IVFTQ_KV_F16 or IVFTQ_KV_BF16. */
typedef struct ivftq_kv_rows {
    void* data;
    int64_t row_stride;
    int64_t head_stride;
    int64_t rows;
    int32_t heads;
    int32_t type;
} ivftq_kv_rows;

/* Bytes of one page's record, all heads; 0 for a shape that is not supported. */
int64_t ivftq_kv_page_bytes(int format, int page, int heads, int d);

/* Write the new rows of every sequence to its pages.  Sequence b's rows are starts[b] .. starts[b + 1] - 1 (device, batch + 1
 * numbers) and become its last tokens, positions lengths[b] - count .. lengths[b] - 1; starts NULL: one row per sequence.
 * k and v have the cache's heads and one type; for the 16-bit formats that type is the cache's.  Coded: a row's norm is
 * rounded to float16 (over 65504: infinite); a row of norm zero stands for zero.  A token whose page is missing is not
 * written. No two sequences may append to one page. */
ivftq_status ivftq_kv_append(const ivftq_kv_cache* cache, const ivftq_kv_rows* k, const ivftq_kv_rows* v,
                             const int32_t* starts, void* stream);

/* The opposite: the rows that the cache holds for these tokens, in the type of the outputs (coded: x^).  Tokens whose page is
 * missing give zeros. */
ivftq_status ivftq_kv_read(const ivftq_kv_cache* cache, const ivftq_kv_rows* k_out, const ivftq_kv_rows* v_out,
                           const int32_t* starts, void* stream);

/* Attention of the new rows over the cache.  q and out: rows x (heads * group), the group consecutive query heads h * group ..
 * of key-value head h share its keys; out has q's rows, heads and type, and does not overlap it (codes: may be the same rows).  The i-th of sequence b's n new rows stands at
 * position p = lengths[b] - n + i and sees the tokens t <= p with window == 0 or t > p - window or t < sinks.
 *     out = sum_t e^(scale <q, k_t> - max) v_t / sum_t e^(scale <q, k_t> - max)
 * A row that sees nothing gives zeros (lse: -infinity).  lse, NULL or rows x (heads * group) floats: the natural logarithm of
 * the sum of e^(scale <q, k_t>).  max_new: no sequence has more new rows than this (>= 1; rows beyond it get no result;
 * starts NULL: taken as 1, which is then what the workspace is asked for with).
 * workspace: ivftq_kv_attend_workspace bytes, 256-byte aligned, its content does not matter. */
ivftq_status ivftq_kv_attend(const ivftq_kv_cache* cache, const ivftq_kv_rows* q, const ivftq_kv_rows* out, float* lse,
                             const int32_t* starts, int32_t max_new, int32_t window, int32_t sinks, float scale,
                             void* workspace, int64_t workspace_bytes, void* stream);
/* -1 for arguments that ivftq_kv_attend refuses. */
int64_t ivftq_kv_attend_workspace(const ivftq_kv_cache* cache, int64_t rows, int32_t q_heads, int32_t max_new);

/* ---- attention over chosen pages ---------------------------------------------------------
 * Over a long cache a row needs few pages.  A page's digest bounds its keys,
 *     low[j] = min_t k_t[j]     high[j] = max_t k_t[j]     (codes: of the rotated keys, norm * level)
 * and a row's queries with it the products that they can have with any key of the page,
 *     score = sum_g sum_j max(q_g[j] low[j], q_g[j] high[j])  >=  sum_g max_t <q_g, k_t>     (g: the key-value head's query heads).
 * In 16 bits the digest is exact.  Over codes its ends are norm * level rounded to the nearest float16: the bounds hold to half a float16 step, 2^-11
 * of an end, of each coordinate.  Each row and key-value head attends to the pages of the highest scores.  A step of a model: ivftq_kv_append, ivftq_kv_digest,
 * ivftq_kv_score, ivftq_kv_select, ivftq_kv_attend_pages.
 * digests: for each page, one after the other, heads x (low[d], high[d]) in the cache's type (codes: float16), 16-byte aligned; an
 * array like a pool, whose pages ivftq_kv_fork_pools and ivftq_kv_compact_pools move with the pool's. */

/* Digests of the pages that hold the new rows, from the rows that ivftq_kv_append has written (same starts, asked and granted): a page
 * whose first token is new gets the digest of its new tokens, one that goes on has them added to the digest that it has.  With every
 * token of a sequence as a new row its digests are made afresh.  Coordinates that are no number count for nothing. */
ivftq_status ivftq_kv_digest(const ivftq_kv_cache* cache, void* digests, const int32_t* starts, void* stream);

/* scores: rows x heads x columns floats; -infinity where a page holds no token that the row sees (behind its position, no page).  A page with
 * an infinite key coordinate has the score +infinity, and so has one whose sum float32 has no number for: nothing bounds its products.
 * A query's coordinate that is no finite number counts for nothing (codes: the whole query, and one whose length float32 does not hold).
 * q, starts, max_new as in ivftq_kv_attend; rows that it gives no result keep their scores.  workspace: ivftq_kv_score_workspace
 * bytes (starts NULL: of max_new = 1), 256-byte aligned. */
ivftq_status ivftq_kv_score(const ivftq_kv_cache* cache, const ivftq_kv_rows* q, const void* digests, float* scores, const int32_t* starts,
                            int32_t max_new, void* workspace, int64_t workspace_bytes, void* stream);
/* -1 for arguments that ivftq_kv_score refuses. */
int64_t ivftq_kv_score_workspace(const ivftq_kv_cache* cache, int64_t rows, int32_t q_heads, int32_t max_new);

/* chosen: rows x heads x count numbers: of the columns that a row's position p reaches (column c: c * page <= p) the first `first` and
 * the last `last`, and those of the highest scores (ties: the lowest column; -infinity and what is no number: never), ascending, -1
 * behind them.  first + last <= count <= 4096.  Rows of no sequence get -1 throughout. */
ivftq_status ivftq_kv_select(const float* scores, const int32_t* lengths, const int32_t* starts, int64_t rows, int32_t batch, int32_t heads,
                             int32_t columns, int32_t page, int32_t count, int32_t first, int32_t last, int32_t* chosen, void* stream);

/* ivftq_kv_attend where a row and key-value head sees, of the tokens up to its own, those of the columns chosen[row][head][0 .. count - 1]
 * (count: 1 to 4096).  Columns ascend; an entry that is not above every one before it, or names no page, is passed over. */
ivftq_status ivftq_kv_attend_pages(const ivftq_kv_cache* cache, const ivftq_kv_rows* q, const ivftq_kv_rows* out, float* lse,
                                   const int32_t* starts, int32_t max_new, const int32_t* chosen, int32_t count, float scale,
                                   void* workspace, int64_t workspace_bytes, void* stream);
/* -1 for arguments that ivftq_kv_attend_pages refuses.  (starts NULL: of max_new = 1) */
int64_t ivftq_kv_attend_pages_workspace(const ivftq_kv_cache* cache, int64_t rows, int32_t q_heads, int32_t max_new, int32_t count);

/* ---- pages ------------------------------------------------------------------------------
 * refs[p]: how many table entries name page p, 0 = free.  Free pages are taken lowest first, rows are served in the order
 * given, so equal states give equal results.  table: rows x columns with stride table_stride, -1 = no page; lengths: rows.
 * Once a row holds pages, these calls alone change the three.  In particular a row is not cut back by a lower length: the entries
 * past it would be written over and their pages lost, and a page that a fork shares would be appended to. */
typedef struct ivftq_kv_pages {
    int32_t* table;
    int32_t* lengths;
    int32_t* refs;
    int64_t table_stride;
    int64_t pages;
    int32_t rows;
    int32_t columns;
    int32_t page;
} ivftq_kv_pages;

/* `layers` pools whose records have equal size: layer l's record of page p at pool + l * layer_stride + p * page_bytes.
 * Multiples of 16 bytes. */
typedef struct ivftq_kv_pools {
    void* pool;
    int64_t layer_stride;
    int64_t page_bytes;
    int64_t pages;
    int32_t layers;
} ivftq_kv_pools;

/* Room for counts[r] more tokens (device, negative counts as 0) in each row: pages taken, lengths raised; granted[r] = counts[r].
 * Where the table's columns or the free pages do not reach, granted[r] = 0 and the row stays as it is (new rows must not be
 * appended to it: see asked and granted above); once the pages have not
 * reached for one row, no later row that needs a page gets one.  scratch: pages int32. */
ivftq_status ivftq_kv_reserve(const ivftq_kv_pages* state, const int32_t* counts, int32_t* granted, int32_t* scratch,
                              void* stream);
/* children[i] becomes a copy of parents[i] (device, n row numbers each, n <= 65536): full pages are shared, a last page that is
 * not full is copied in every layer to a free one (entries that name no page become -1).  done[i] = 1, or 0 where nothing was done: a number out of range, a child
 * that is not empty, that an earlier entry names or that is any entry's parent, or no free page left.  scratch:
 * pages + 2 n + 2 rows int32. */
ivftq_status ivftq_kv_fork(const ivftq_kv_pages* state, const ivftq_kv_pools* pools, const int32_t* parents,
                           const int32_t* children, int32_t n, int32_t* done, int32_t* scratch, void* stream);
/* Rows (device, n row numbers; repeats count once) give their pages back and become empty.  The state's page
 * size is not read (any that is allowed). */
ivftq_status ivftq_kv_free(const ivftq_kv_pages* state, const int32_t* rows, int32_t n, void* stream);
/* Every row gives back the pages that no later token can see with this window (> 0) and these first tokens; the entries
 * become -1, lengths stay. */
ivftq_status ivftq_kv_trim(const ivftq_kv_pages* state, int32_t window, int32_t sinks, void* stream);
/* Moves pages in use to the lowest numbers: of `used` pages in use, those numbered `used` and above go, in ascending order, to
 * the free ones below.  Table, counts and every layer's records follow; *used_out (device) = used.  scratch: 3 pages + 64
 * int32.  The lengths and the page size of the state are not read (page: any that is allowed). */
ivftq_status ivftq_kv_compact(const ivftq_kv_pages* state, const ivftq_kv_pools* pools, int32_t* used_out, int32_t* scratch,
                              void* stream);
/* The two for `groups` arrays (1 to 8) of records whose pages are numbered alike: a cache's pools and its digests. */
ivftq_status ivftq_kv_fork_pools(const ivftq_kv_pages* state, const ivftq_kv_pools* pools, int32_t groups, const int32_t* parents,
                                 const int32_t* children, int32_t n, int32_t* done, int32_t* scratch, void* stream);
ivftq_status ivftq_kv_compact_pools(const ivftq_kv_pages* state, const ivftq_kv_pools* pools, int32_t groups, int32_t* used_out,
                                    int32_t* scratch, void* stream);
/* Record of page src[i] to page dst[i] in every layer (device, n numbers each; a pair with a number out of range is passed
 * over).  No page may be both source and destination, or destination twice. */
ivftq_status ivftq_kv_copy(const ivftq_kv_pools* pools, const int32_t* src, const int32_t* dst, int32_t n, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* IVFTQ_KV_H */
