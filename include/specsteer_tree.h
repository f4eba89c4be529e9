/*
 * specsteer_tree.h -- C ABI of trees of drafted tokens on MI355X (gfx950): the attention that scores a tree's rows over a
 * paged cache, the verify-and-recover step down a tree, and the commit of the accepted path to the cache.
 *
 *   specsteer_tree_attention  attention of the last token and the drafts behind it over the cache and their own ancestors
 *   specsteer_tree_verify     specsteer_verify_block of specsteer.h for a tree
 *   specsteer_tree_commit     keys and values of the accepted path into the cache
 *
 * A tree of sequence b has N_b nodes, the drafted tokens, in any order with every node behind its parent: parents[b][i] is
 * in [-1, i), -1 for a child of the last token.  Rows are counted as in specsteer.h: row 0 is the last token, whose
 * next-token distribution scores the children of -1, and row i + 1 is node i.  parents may be NULL: a chain, every node the
 * child of the one before it, which is what specsteer_verify_block takes; without nodes a call is one for single tokens.
 * Rows past N_b belong to nobody: nothing that inputs hold there matters, and outputs have 0 there.
 *
 * Pointers, streams, workspaces and errors are as in specsteer.h: all arrays are device memory but for the parameters,
 * nothing is allocated, owned or waited for, argument errors return before anything is enqueued and leave every output
 * untouched.  All calls may be captured into a graph.  Sums are formed in a fixed order: the same call gives the same bits.
 * Data errors that only the GPU can see mark their sequence alone, as each call says; no out-of-range address is formed.
 * No output shares memory with an input or another output: workgroups read the one while others write the other
 * (SS_ERR_PARAM where two of the small arrays are one).
 *
 * Cache.  Keys and values lie in pages of page_size positions, [pages, page_size, kv_heads, head_dim] each; position t of
 * sequence b is slot t % page_size of page block_table[b][t / page_size].  Pages may be shared between sequences.
 */
#ifndef SPECSTEER_TREE_H
#define SPECSTEER_TREE_H

#include "specsteer.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SS_TREE_F16 2         /* besides SS_BF16: the type of queries, keys, values and outputs */
#define SS_TREE_MAX_HEADS 1024
#define SS_TREE_MAX_ROWS (1 << 20) /* largest batch * (nodes + 1) */

typedef struct {
    int32_t batch;       /* B >= 0 (0 is a no-op)                                                       */
    int32_t nodes;       /* N, 0..SS_MAX_K: most nodes of a tree; arrays of rows hold N + 1             */
    int32_t heads;       /* query heads, a multiple of kv_heads, up to SS_TREE_MAX_HEADS                */
    int32_t kv_heads;    /* query head h reads key and value head h / (heads / kv_heads)                */
    int32_t head_dim;    /* attention: 64 or 128; commit: any multiple of 8 up to 1024                  */
    int32_t dtype;       /* SS_BF16 or SS_TREE_F16                                                      */
    int32_t pages;       /* of the cache, >= 0                                                          */
    int32_t page_size;   /* >= 1                                                                        */
    int32_t table_width; /* columns of block_table, >= 0                                                */
    float scale;         /* of the products of queries and keys; finite (commit: not read)              */
    /* Element strides, 0 for those of a dense array.  head_dim is contiguous.  All are multiples of 8, and so are the
     * arrays' addresses of 16 bytes.                                                                    */
    int64_t q_stride[3];     /* sequence, row, head of q                                                */
    int64_t k_stride[3];     /* of k; v has the same                                                    */
    int64_t out_stride[3];   /* of out                                                                  */
    int64_t cache_stride[3]; /* page, slot, head of k_cache; v_cache has the same.  attention: pages    */
                             /* and slots less than 2^31 apart                                          */
    int64_t table_stride;    /* of block_table's rows                                                   */
} ss_tree_params;

/* Bytes of device scratch (256-byte aligned) that specsteer_tree_attention needs; 0 for invalid params. */
size_t specsteer_tree_attention_workspace_bytes(const ss_tree_params *params);

/*
 * For row r of sequence b and query head h, with G = heads / kv_heads:
 *     out = sum_j p_j v_j,   p = softmax_j(scale * q . k_j)
 * over j in positions [0, cache_len[b]) of the cache and the rows of the block that are r or its ancestors, row 0 among
 * them.  Softmax statistics and sums are fp32; the weights p are rounded to the type of the values for their product.
 *
 *   q            device, [B, N + 1, heads, head_dim]
 *   k, v         device, [B, N + 1, kv_heads, head_dim]: the block's own rows, not in the cache yet
 *   k_cache, v_cache, block_table  device, see above; block_table is int32
 *   cache_len    device, [B] int32, 0..table_width * page_size
 *   parents      device, [B, N] int32, or NULL: chains
 *   tree_len     device, [B] int32, 0..N, or NULL: N for all
 *   out          device, [B, N + 1, heads, head_dim] out; no input's memory
 *
 * A sequence whose cache_len or tree_len is out of range, or a parent or a page that is needed, has NaN in all its rows.  A
 * row never takes anything from positions that it does not see, whatever they hold.  What it sees is expected to be finite,
 * the sums q . k to be numbers of fp32, and scale * q . k to be below 2^30 in size: a row that sees other values has NaN, or
 * what they make of it.  A call whose work may reach 2^31 tiles (keys times heads times rows, by 64 keys times 32 to 256 rows)
 * is refused with SS_ERR_SHAPE.
 */
ss_status specsteer_tree_attention(const void *q, const void *k, const void *v, const void *k_cache, const void *v_cache,
                                   const int32_t *block_table, const int32_t *cache_len, const int32_t *parents,
                                   const int32_t *tree_len, const ss_tree_params *params, void *out, void *workspace,
                                   size_t workspace_bytes, void *stream);

/* Bytes of device scratch that specsteer_tree_verify needs; 0 for invalid params. */
size_t specsteer_tree_verify_workspace_bytes(const ss_params *params);

/*
 * The walk down a tree, by Eq. 7 and Eq. 8 as in specsteer_verify_block:
 *     cur = -1
 *     for the children c of cur by increasing index:
 *         accept iff uniforms[b][c] <= min(1, P_LLM(y_c) / (lambda * P_SLM^-(y_c)))  at row cur + 1
 *         the first that is accepted: append it to the path, cur = c, and go on with its children
 *     next_token ~ Softmax((h_LLM + beta * (h_SLM^+ - h_SLM^-)) / T)  at row cur + 1, by uniforms[b][N]
 * For a chain these are the block's results; a leaf's row yields the bonus token.  Params are those of the block, with
 * k_max = N and flags 0 or SS_FLAG_GREEDY; logits are [B, N + 1, V], with the block's masked tokens, and rows that the
 * walk does not come through are not needed, though any row up to N_b may be read.
 *
 *   tokens              device, [B, N] int32
 *   parents, tree_len   as above
 *   uniforms            device, [B, N + 1] fp32 in [0, 1)
 *   accepted_len        device, [B] int32 out: nodes on the path
 *   path                device, [B, N] int32 out: the path's nodes, -1 behind them
 *   next_token          device, [B] int32 out
 *   next_token_logprob  device, [B] fp32 out, or NULL
 *
 * A sequence whose tree_len, a parent or a token (of any node i < N_b) is out of range has -1 in accepted_len, path and
 * next_token, and NaN in next_token_logprob.
 */
ss_status specsteer_tree_verify(const void *G, const void *S_ctx, const void *S_noctx, const int32_t *tokens,
                                const int32_t *parents, const int32_t *tree_len, const float *uniforms,
                                const ss_params *params, int32_t *accepted_len, int32_t *path, int32_t *next_token,
                                float *next_token_logprob, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Rows 0, path[b][0] + 1, ..., path[b][accepted_len[b] - 1] + 1 of k and v go to positions cache_len[b], cache_len[b] + 1, ...
 * of the cache; new_len[b] = cache_len[b] + accepted_len[b] + 1.  Other positions keep what they hold.
 *
 *   k, v              device, [B, N + 1, kv_heads, head_dim]
 *   k_cache, v_cache  device, laid out as described above; no memory of k, v or each other
 *   accepted_len      device, [B] int32, 0..N
 *   path              device, [B, N] int32, or NULL: 0, 1, 2, ..., a chain's
 *   new_len           device, [B] int32 out; neither cache_len nor accepted_len itself
 *
 * A sequence whose accepted_len, cache_len, path or pages are out of range, or whose positions pass table_width * page_size,
 * has -1 in new_len, and nothing of it is written.  Sequences that would write the same slot of the same page race.
 */
ss_status specsteer_tree_commit(const void *k, const void *v, void *k_cache, void *v_cache, const int32_t *block_table,
                                const int32_t *cache_len, const int32_t *accepted_len, const int32_t *path,
                                const ss_tree_params *params, int32_t *new_len, void *stream);

/* What a status of these calls means (the codes are those of specsteer.h). */
const char *specsteer_tree_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* SPECSTEER_TREE_H */
