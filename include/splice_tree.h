/*
 * splice_tree.h -- several candidate tokens per sweep cell judged in one pass:
 * a tree of T drafted tokens hangs below each cell's last token, every node is
 * one row of a forward pass, and the entries below do what such a pass needs
 * beside the weight products:
 *   splice_tree_append   rotary positions of the nodes' q and k, and their K/V
 *                        written as rows of the generated caches;
 *   splice_tree_attn     the spliced attention of every node;
 *   splice_token_scores  log probability, entropy, rank and top alternatives
 *                        of given tokens, from the logits;
 *   splice_tree_keep     the rows of the accepted nodes moved together, so that
 *                        the cell goes on behind them;
 *   splice_tree_read     the T rows of each cell read back as bf16.
 *
 * The tree.  Cell c has s_c = cell_step[c] generated rows (host int32 [C];
 * < 0: a finished cell, nothing of it is read or written).  Node t of 0..T-1
 * has its K/V in row s_c + t of the cell's generated caches, depth
 * depth[c][t] >= 0 (its distance from the root of the tree: the root's depth
 * is 0) and a word visible[c][t], bit u of which says that node t sees node u;
 * a node that sees itself has its own bit set.  depth and visible are device
 * memory, [C][T] int32 and [C][T] uint64.  A depth < 0 marks padding: such a
 * node is no query, no other node sees it, and its rows and outputs are left
 * as they were.  A depth of T or more counts as T - 1, bits from T on as 0.
 * Node t is the token of decode step s_c + depth: it sits at position
 * p = T_p + s_c + depth, the splice predicate takes that step (the nodes of
 * one cell may differ in it), and it sees the prompt slots, the cell's
 * rows below s_c and the nodes of its word, of these with a window w > 0
 * only positions > p - w (a node's position is that of its depth).  A query
 * that sees nothing has out = 0 and lse = -inf.  What a query does not see
 * does not reach its result, whatever it holds (NaN and infinities too).
 *
 * Generated caches are bf16, or 8 bits a value (SPLICE_KV_E4M3): gen_k, gen_v
 * uint8 [C][Hkv][cap][D] hold OCP e4m3 codes and gen_k_exp, gen_v_exp uint8
 * [C][Hkv][cap] one exponent a row; a value is code * 2^(exponent - 127).  The
 * exponent of a row is the smallest with max |x| <= 448 * 2^(e - 127), at least
 * 27 (rows whose largest value is below 2^-92 lose digits), so every
 * stored value is exact in bf16 and an attention over such a cache is that over
 * the bf16 cache of the same values.  A row with an infinity or NaN reads
 * back as NaN.  Prompt caches are bf16.
 *
 * Otherwise the conventions of splice_attn.h hold: shapes, splices, ownership,
 * alignment (16 bytes; exponents, depth, lse and logits as their types),
 * streams, errors.  Every entry takes shape->dtype == SPLICE_BF16 only
 * and fewer than 2^16 query heads (SPLICE_EUNSUPPORTED otherwise).  s_c + T <=
 * gen_capacity for every active cell (SPLICE_ESHAPE).  Results are deterministic.
 */
#ifndef SPLICE_TREE_H
#define SPLICE_TREE_H

#include "splice_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPLICE_MAX_NODES 64
#define SPLICE_MAX_TOP 64

typedef enum { SPLICE_KV_BF16 = 0, SPLICE_KV_E4M3 = 1 } splice_kv_format;
typedef enum { SPLICE_ROPE_HALF = 0, SPLICE_ROPE_INTERLEAVED = 1 } splice_rope_layout;

typedef struct {
    int32_t n_nodes;    /* T, 1..SPLICE_MAX_NODES                  */
    int32_t kv_format;  /* splice_kv_format of the generated caches */
} splice_tree;

typedef struct {
    int32_t layout;      /* splice_rope_layout: pairs (i, i + R / 2), or (2 i, 2 i + 1)       */
    int32_t rotary_dim;  /* R: the first R values of a head turn; a multiple of 16 in 0..D  */
    double mscale;       /* factor on cos and sin (1, or a long-context scaling's), finite  */
} splice_rope;

/*
 * For node t of active cell c, with angle_i = p * freq[i] (device, R / 2
 * doubles; the product and its reduction are computed in 64 bits):
 *   q_out[c][t]  = the rotated q[c][t], bf16 [C][T][Hq][D]; q_out may be q
 *                  when q is dense;
 *   row s_c + t of gen_k, gen_v = the rotated k[c][t], and v[c][t], in
 *                  tree->kv_format (bf16: one rounding from the rotation in fp32;
 *                  e4m3: codes and exponents of the rotation in 64 bits).
 * q, k, v: bf16, a token's heads dense ([heads][D]) and q_stride, k_stride,
 * v_stride values from one token to the next (multiples of 8, at least
 * heads * D), so they may be parts of one projection's rows.  pos: device
 * int64 [C][T] positions, or NULL for T_p + s_c + depth; positions of
 * magnitude up to 2^31.  gen_k_exp, gen_v_exp: as the format says (NULL for
 * bf16).  freq may be NULL if R is 0.
 */
SPLICE_API int32_t splice_tree_append(const splice_shape *shape, const splice_tree *tree, const splice_rope *rope,
                                      const int32_t *cell_step, const int32_t *depth, const int64_t *pos,
                                      const double *freq,
                                      const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                      const void *v, int64_t v_stride, void *q_out, void *gen_k, void *gen_v,
                                      uint8_t *gen_k_exp, uint8_t *gen_v_exp, void *stream);

/* rows_k, rows_v [C][Hkv][T][D] bf16 = rows s_c .. s_c + T - 1 of the generated caches of every active cell. */
SPLICE_API int32_t splice_tree_read(const splice_shape *shape, const splice_tree *tree, const int32_t *cell_step,
                                    const void *gen_k, const void *gen_v, const uint8_t *gen_k_exp,
                                    const uint8_t *gen_v_exp, void *rows_k, void *rows_v, void *stream);

/*
 * out [C][T][Hq][D] bf16 and lse [C][T][Hq] fp32 (natural log) of the nodes
 * of every active cell; q [C][T][Hq][D] bf16, rotated.  call->step and
 * call->merge_wait are ignored.  Weighted values are summed in fp32 before the
 * division by the weights' sum, and a weight may be 2^8: values of a size that
 * times 2^8 times the number of keys passes fp32's range may give infinities.
 * workspace: 256-byte aligned,
 * splice_tree_attn_workspace_bytes(shape, call, tree) bytes (enough for any
 * steps; it may be 0), no initialisation.  Calls that share a workspace must
 * be ordered on one stream.
 */
SPLICE_API int64_t splice_tree_attn_workspace_bytes(const splice_shape *shape, const splice_call *call,
                                                    const splice_tree *tree);
SPLICE_API int32_t splice_tree_attn(const splice_shape *shape, const splice_call *call, const splice_tree *tree,
                                    const int32_t *cell_LW, const int32_t *cell_step, const int32_t *depth,
                                    const uint64_t *visible, const void *q,
                                    const void *clean_k, const void *clean_v, const void *donor_k, const void *donor_v,
                                    const void *gen_k, const void *gen_v, const uint8_t *gen_k_exp,
                                    const uint8_t *gen_v_exp, void *out, float *lse,
                                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * Row s_c + i of the generated caches = row s_c + keep[c][i], for
 * i = 0, 1, ... (device int32 [C][T]): the ascending nodes of an accepted path.  The
 * list of a cell ends at its first entry that is negative, not below T or not
 * above the one before.
 */
SPLICE_API int32_t splice_tree_keep(const splice_shape *shape, const splice_tree *tree, const int32_t *cell_step,
                                    const int32_t *keep, void *gen_k, void *gen_v, uint8_t *gen_k_exp,
                                    uint8_t *gen_v_exp, void *stream);

/*
 * What a model's logits say about given tokens.  Per row r of logits
 * [rows][vocab] (dtype: SPLICE_BF16 or SPLICE_F32, row_stride values from row
 * to row), with x = scale * logit (scale finite, > 0) and token = tokens[r]:
 *   lse       log sum exp x
 *   logp      x[token] - lse            (NaN for a token outside [0, vocab))
 *   entropy   of softmax(x), in nats
 *   rank      how many tokens come before this one, by the larger logit, among
 *             equals by the lower index  (-1 for a token outside [0, vocab))
 *   top, top_logp  [rows][k]: the first k tokens of that order and their log
 *             probabilities; 0 <= k <= min(vocab, SPLICE_MAX_TOP), both may be
 *             NULL when k is 0.
 * Logits of -inf have probability 0 (a row of nothing else: lse -inf,
 * entropy and logp NaN).  Logits of NaN or +inf make the row's lse, entropy and log
 * probabilities NaN (with +inf the softmax is inf / inf); NaN ones come first in its
 * order, and ranks count them as above every number.  Finite logits may be
 * as large as a float: what a row's have in common does not reach its
 * probabilities.  What passes a float (lse, logp, a distance between two logits) is infinite.
 * Sums are fp32; rows < 2^24, vocab <= 2^28.  logp, lse, entropy fp32 [rows]; rank, tokens, top int64.
 * workspace: 16-byte aligned, splice_token_scores_workspace_bytes bytes, no
 * initialisation.
 */
SPLICE_API int64_t splice_token_scores_workspace_bytes(int64_t rows, int64_t vocab, int32_t k);
SPLICE_API int32_t splice_token_scores(const void *logits, int32_t dtype, int64_t rows, int64_t vocab,
                                       int64_t row_stride, float scale, const int64_t *tokens, int32_t k, float *logp,
                                       float *lse, float *entropy, int64_t *rank, int64_t *top, float *top_logp,
                                       void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SPLICE_TREE_H */
