/*
 * splice_pages.h -- K and V held in 4 bits, in pages of 64 tokens that cells of a
 * sweep share, copy on write and give back:
 *   splice_page_append   rotary positions of new tokens' q and k, and their K/V
 *                        written to pages in 4 bits;
 *   splice_page_read     rows of cells read back as bf16;
 *   splice_page_attn     the spliced attention of every cell's new tokens, one
 *                        or many, over such pages;
 *   splice_page_fork     cells take over the rows of others, give pages back and
 *                        get new ones;
 *   splice_page_compact  the rows of a cell that stay moved together.
 *
 * Pages.  A layer's pool is uint8 [n_pages][page_bytes], 16-byte aligned (the pools
 * of several layers layer_stride bytes apart, a multiple of 16); a page holds
 * 64 tokens of every KV head.  Row r of cell c is row r mod 64 of page
 * tables[c][r / 64] (device int32 [C][table_len]); prompt slot j is row j mod 64 of
 * page clean_table[j / 64] or donor_table[j / 64] (device int32
 * [ceil(T_p / 64)], pages of the same pool).  Pages may be shared by
 * any tables as long as nobody writes to them.  An entry outside [0, n_pages) is
 * an absent page: what lies in it is seen by nobody, and what is written to it is
 * dropped.  A call reads a table's entries for rows below gen_capacity only, which is at
 * most 64 * table_len.
 *
 * 4 bits a value.  Every 32 values of a (token, head) row share an exponent byte e;
 * a value is code * 2^(e - 127), its code a sign (bit 3) and one of 0, 1/2, 1,
 * 3/2, 2, 3, 4, 6 (OCP e2m1 under e8m0 scales, "MXFP4").  e - 127 is the smallest with
 * max |x| <= 6 * 2^(e - 127), at least -100 (blocks whose largest value is below
 * 2^-98 lose digits); codes are to the nearest, ties to the even code, and above
 * 3 * 2^126 they stop there (a rotated k beyond fp32's range, too).  Every stored value is
 * exact in bf16.  Where k or v of a token has an infinity or NaN in some head, every
 * byte e of that head's k and v row is 255: the rows read back as NaN, and out and lse
 * of a query that sees them are NaN.
 *
 * Bytes of a page: Hkv heads of 68 D bytes, each, with r a token of the page:
 *   K codes   [64][D / 2]: values 2 i (low half) and 2 i + 1 of token r at [r][i];
 *   V codes   [2][D / 64][4][16][2][4][2]: values 64 b + 4 d + 2 g (low half) and the next
 *             of token r = 32 a + 16 e + 4 c + f at [a][b][c][d][e][f][g];
 *   K scales  [D / (32 n)][16][n][4], n = min(4, D / 32): block n a + c of token
 *             r = 16 d + b at [a][b][c][d];
 *   V scales  [2][4][2][D / 64][2][4]: block 2 d + c of token r = 32 a + 16 e + 4 b + f
 *             at [a][b][c][d][e][f].
 * (The order in which the matrix instructions take them, see csrc/page_format.hpp.)
 *
 * Otherwise the conventions of splice_attn.h hold: shapes, splices, ownership,
 * streams, errors.  Every entry takes shape->dtype == SPLICE_BF16 only (that of q, k and v).
 * cell_step (host int32 [C]): rows that the cell has, s_c; < 0: a finished
 * cell, nothing of it is read or written.  cell_new (host int32 [C], 0..T;
 * NULL: T for all): its tokens in this pass.  Token t of cell c is that of decode
 * step s_c + t at position T_p + s_c + t, row s_c + t; what stands in a call's
 * tensors for tokens from cell_new[c] on is neither read nor written.
 * s_c + cell_new[c] <= gen_capacity (SPLICE_ESHAPE).  Results are deterministic.
 */
#ifndef SPLICE_PAGES_H
#define SPLICE_PAGES_H

#include "splice_attn.h"
#include "splice_tree.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPLICE_PAGE_ROWS 64
#define SPLICE_MAX_PAGE_TOKENS 32768

typedef struct {
    int32_t n_pages;    /* pages of a layer's pool, 1..2^24                       */
    int32_t table_len;  /* entries of a cell's table, 1..2^22                     */
    int32_t n_tokens;   /* T: tokens a cell (or entries of its list) in a call,
                           1..SPLICE_MAX_PAGE_TOKENS                              */
} splice_pages;

/* Bytes of one page of one layer: Hkv * 68 * D. */
SPLICE_API int64_t splice_page_bytes(const splice_shape *shape);

/*
 * For token t of active cell c, with the angles of splice_tree_append:
 *   q_out[c][t]  = the rotated q[c][t], bf16 [C][T][Hq][D] (rotated in fp32, one
 *                  rounding); q_out may be q when q is dense;
 *   row s_c + t  = the rotated k[c][t] and v[c][t] in 4 bits (rotated in 64 bits, by a sine
 *                  and cosine that are off by 2^-33 and 2^-51 of the angle at most).
 * q, k, v, their strides, pos (device int64 [C][T], or NULL) and freq: as
 * splice_tree_append takes them, with T = pages->n_tokens; q and q_out may both be NULL
 * (then only rows are written).  A page that is written
 * to is in one cell's table only (splice_page_fork sees to that).
 */
SPLICE_API int32_t splice_page_append(const splice_shape *shape, const splice_pages *pages, const splice_rope *rope,
                                      const int32_t *cell_step, const int32_t *cell_new, const int32_t *tables,
                                      const int64_t *pos, const double *freq,
                                      const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                      const void *v, int64_t v_stride, void *q_out, void *pool, void *stream);

/* rows_k, rows_v [C][Hkv][T][D] bf16: row i is row cell_step[c] + i of the cell, for i < cell_new[c]; rows of absent
 * pages are left as they were. */
SPLICE_API int32_t splice_page_read(const splice_shape *shape, const splice_pages *pages, const int32_t *cell_step,
                                    const int32_t *cell_new, const int32_t *tables, const void *pool, void *rows_k,
                                    void *rows_v, void *stream);

/*
 * out [C][T][Hq][D] bf16 and lse [C][T][Hq] fp32 (natural log) of the tokens of
 * every active cell; q [C][T][Hq][D] bf16, rotated.  Token t sees the prompt
 * slots and the cell's rows 0..s_c + t, with a window w > 0 only positions > p - w, and takes the
 * splice predicate of step s_c + t.  One that sees nothing has out = 0 and
 * lse = -inf.  What a query does not see does not reach its result.  call->step
 * and call->merge_wait are ignored; call->split_keys sets the keys a work group
 * takes (0: planned).  Scores are fp32; one that is NaN or +inf makes the query's
 * results NaN, one of -inf has weight 0.  Weights enter the second product as bf16, and weighted values are
 * summed in fp32 before the division by the weights' sum (a weight may be 2^8).
 * Calls of 2^24 work groups and more are SPLICE_EUNSUPPORTED (2^26 rows, tokens x q heads, of one cell).
 * workspace: 256-byte aligned, splice_page_attn_workspace_bytes(shape, call,
 * pages) bytes (enough for any steps; it may be 0), no initialisation.  Calls that
 * share a workspace must be ordered on one stream.
 */
SPLICE_API int64_t splice_page_attn_workspace_bytes(const splice_shape *shape, const splice_call *call,
                                                    const splice_pages *pages);
SPLICE_API int32_t splice_page_attn(const splice_shape *shape, const splice_call *call, const splice_pages *pages,
                                    const int32_t *cell_LW, const int32_t *cell_step, const int32_t *cell_new,
                                    const int32_t *tables, const int32_t *clean_table, const int32_t *donor_table,
                                    const void *q, const void *pool, void *out, float *lse, void *workspace,
                                    size_t workspace_bytes, void *stream);

/*
 * Who holds which pages next.  Cell c becomes the first rows[c] rows of cell
 * parent[c] as it was before the call (host int32 [C]; parent[c] < 0: empty, with
 * rows[c] == 0), with pages for want[c] >= rows[c] rows (host int32 [C]):
 * a fork, a beam that goes on from another, a cell that gives its rows back,
 * keeps fewer, or gets room for more are all calls of this kind.
 *   - Pages are counted: refs[p] (device int32 [n_pages]) is the number of table
 *     entries that name page p, plus what others hold of it; 0: the page is free.
 *   - new_tables, new_refs are the tables and counts after the call; they overlap no
 *     input.  Entries behind want[c] rows are -1.
 *   - A last page that rows[c] fills in part and that has other holders is
 *     copied, in every layer; where all its holders are such cells of this call, the
 *     first of them keeps it.  copied[c] (device int32 [C][2]) is (from, to),
 *     or (-1, -1).
 *   - New pages are the free ones from the lowest on, in the order of cells and of a cell's rows.
 *     *missing (device int32): how many there were too few; their entries are -1.  A cell's are then
 *     its last ones.  Entries below rows[c] rows that were absent stay so, and are not asked for: a later call
 *     that is to fill them names fewer rows.
 * rows[c], want[c] <= 64 * table_len; shape: n_cells, the heads and D; pool: the first
 * layer's, n_layers = shape->n_layers of them.  pages->n_tokens is ignored.  As everywhere, a call
 * without cells does nothing: new_refs too is then left as it was.
 */
SPLICE_API int32_t splice_page_fork(const splice_shape *shape, const splice_pages *pages, const int32_t *parent,
                                    const int32_t *rows, const int32_t *want, const int32_t *tables,
                                    const int32_t *refs, int32_t *new_tables, int32_t *new_refs, int32_t *missing,
                                    int32_t *copied, void *pool, int64_t layer_stride, void *stream);

/*
 * Row cell_step[c] + i = row cell_step[c] + keep[c][i] in every layer, for
 * i = 0, 1, ... (device int32 [C][T]): accepted tokens, or those that an
 * eviction leaves.  The list of a cell ends at its first entry that is negative, not
 * above the one before, or whose row is not below gen_capacity.  Rows behind those
 * that are written are left as they were.  Pages from row cell_step[c] on are in one
 * table only; rows from or to absent pages are dropped.
 */
SPLICE_API int32_t splice_page_compact(const splice_shape *shape, const splice_pages *pages, const int32_t *cell_step,
                                       const int32_t *keep, const int32_t *tables, void *pool, int64_t layer_stride,
                                       void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SPLICE_PAGES_H */
