/* Several continuations of one sequence over the paged KV pool: trees of drafted tokens that one pass of the model
 * verifies, and beams.  The paper (arxiv 2504.14775) schedules sequences with one continuation each; what stands here is the
 * public arithmetic of speculative decoding with token trees and of beam search, on the pool layout of gllm_stage.h.
 *
 * A step with drafted tokens: gllm_stage_forward_tree (gllm_stage.h) runs the layers over the trees, gllm_head_logits and
 * gllm_op_sample give one token for every node, gllm_op_tree_commit walks down each tree along these tokens and puts the
 * keys and values of the accepted nodes behind the prefix.  Since the sampler draws from the model's own distribution at
 * every node, what is accepted is distributed as without drafts.  A step with beams: gllm_stage_forward with one decode row per
 * beam, gllm_head_logits, gllm_op_beam_select; the caller forks the block tables of the chosen beams (whole pages are shared)
 * and gives each its own copy of the last, partly filled page by gllm_op_copy_pages.
 *
 * Same conventions as gllm_stage.h: plain C, every pointer marked HOST or DEVICE, DEVICE pointers belong to the current
 * HIP device, calls enqueue on `stream`, allocate nothing and return a gllm_status; there is no CPU fallback.  What lies on
 * the device is not read by the host: the calls can be recorded into a graph and replayed with other contents, and contents
 * that break a rule below are left out of the work as stated there, never followed out of the buffers.
 *
 * Trees.  Sequence s has the rows row_start[s] .. row_start[s+1]-1 of the row arrays, node i of its tree is row row_start[s]+i,
 * and parents[] holds, for every row, the index of its parent node in the same tree, smaller than its own, or -1 for a
 * root.  Any other value makes the node unused, and with it every node below it.  A tree has up to 256 nodes.  The keys and
 * values of node i lie in the pool at position cached_len[s] + i of the sequence: slot position % 16 of page
 * block_tables[s][position / 16].  (The rotary position of a node is cached_len[s] + its depth.)
 */
#ifndef GLLM_BRANCH_H
#define GLLM_BRANCH_H

#include <stddef.h>
#include <stdint.h>

#include "gllm_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { GLLM_TREE_MAX_NODES = 256, GLLM_BEAM_MAX_BEAMS = 32, GLLM_BEAM_MAX_KEEP = 64 };

/* Attention of one layer: row r of `out` = softmax over the visible positions of (q[r] . k * scale), times v, per query head; node i
 * of sequence s sees the positions 0 .. cached_len[s]-1 and those of its ancestors and of itself.
 *   q             DEVICE bf16 [num_rows][ld_q], rotated queries, head h in columns h*head_dim .. (ld_q a multiple of 8, 16-byte
 *                 aligned)
 *   k_pool,v_pool DEVICE bf16, one layer of the pool (layout: gllm_stage_bind_kv_pool), num_blocks pages, 16-byte aligned
 *   block_tables  DEVICE int32 [num_seqs][block_table_stride]; a page id outside [0, num_blocks) is read as the nearest one inside
 *   cached_len    DEVICE int32 [num_seqs]
 *   row_start     DEVICE int32 [num_seqs + 1], ascending, from 0 up to at most num_rows (otherwise no row is written)
 *   parents       DEVICE int32 [num_rows]
 *   max_nodes     HOST: most nodes of any tree, 1 .. 256; the kernels are chosen by it
 *   out           DEVICE bf16 [num_rows][ld_out] (ld_out a multiple of 4, 8-byte aligned)
 *   workspace     DEVICE, 16-byte aligned, at least gllm_op_tree_attention_workspace_bytes() of it; contents need not survive
 *                 between calls, and calls that may overlap in time need one each
 * Unused nodes, and all nodes of a sequence with more than max_nodes, with cached_len < 0 or with more positions than its table row
 * has entries for (or than 2^31 - 64), receive zeros.  Rows outside every sequence are left as they are.  The keys and values of unused nodes and of slots
 * past the last node may hold anything; those of the prefix and of used nodes have to be finite for every row that sees them, and a value
 * that is not finite spoils the rows that see it only.
 * Supported: head_dim 64 or 128, n_q_heads a multiple of n_kv_heads with at most 16 query heads per KV head (else
 * GLLM_E_UNSUPPORTED); scale > 0 and at most 2.3e38 (else GLLM_E_INVALID), q . k finite in float, and q . k * scale between -5e29 and 2e38.
 * GLLM_E_CAPACITY for a workspace that is too small and for more than 2^22 sequences. */
gllm_status gllm_op_tree_attention(const void* q, int64_t ld_q, const void* k_pool, const void* v_pool, int64_t num_blocks,
                                   const int32_t* block_tables, int32_t block_table_stride, const int32_t* cached_len,
                                   const int32_t* row_start, const int32_t* parents, int32_t num_seqs, int32_t num_rows,
                                   int32_t max_nodes, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                                   void* out, int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream);
/* HOST only; 0 for head counts, a head size or max_nodes that the call does not take. */
size_t gllm_op_tree_attention_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_nodes);

/* Acceptance: from node 0, a root, the walk goes on to the lowest child whose token is the one sampled at the node, until there is
 * none.  The nodes passed are accepted (node 0 always is), path[row_start[s] ..] receives their indices in order and -1 behind
 * them, count[s] their number, next_token[s] the token sampled at the last of them; count 0, next_token -1 and a path of -1 for a
 * sequence without rows, with more than 256, whose node 0 is no root, or whose positions do not fit its table row (cached_len < 0
 * and more than 2^31 - 64 positions among them).
 * Then, in all layers, the keys and values of the i-th accepted node move to position cached_len[s] + i: the sequence goes on with
 * cached_len[s] + count[s] positions and next_token[s] as its next root.  Other slots are left as they are; a move from or to a page id
 * outside [0, num_blocks) is left out.  No page that holds a node may belong to two sequences of the call.
 *   tokens   DEVICE int32 [num_rows]: the drafted token of every node
 *   sampled  DEVICE int32 [num_rows]: the token drawn at every node (gllm_op_sample)
 *   k_pool, v_pool  DEVICE bf16, num_layers layers of num_blocks pages (16-byte aligned); both NULL: nothing is moved, and
 *            num_layers, num_blocks, n_kv_heads, head_dim are not looked at
 *   path DEVICE int32 [num_rows], count, next_token DEVICE int32 [num_seqs]
 * head_dim 64 or 128, else GLLM_E_UNSUPPORTED; num_layers * n_kv_heads * num_seqs below 2^31, else GLLM_E_CAPACITY. */
gllm_status gllm_op_tree_commit(const int32_t* tokens, const int32_t* parents, const int32_t* sampled, const int32_t* row_start,
                                const int32_t* cached_len, const int32_t* block_tables, int32_t block_table_stride,
                                int32_t num_seqs, int32_t num_rows, void* k_pool, void* v_pool, int32_t num_layers,
                                int64_t num_blocks, int32_t n_kv_heads, int32_t head_dim, int32_t* path, int32_t* count,
                                int32_t* next_token, void* stream);

/* Beam search: for every sequence the `keep` best continuations (beam b, token v) by
 *   scores[s][b] + logits[s*beams + b][v] - log sum_u exp logits[s*beams + b][u],
 * best first.  They are compared, and the sum is taken, in 64 bits (log sum exp is good to some 1e-10); those that agree there are in order of
 * the beam, in a beam of the logit, the largest first, and equal logits in order of the token.
 *   logits  DEVICE float [num_seqs*beams][ld_logits]; scores DEVICE float [num_seqs][beams]: log probability of each beam so far
 *   out_scores DEVICE float, out_beams, out_tokens DEVICE int32, [num_seqs][keep]
 * A beam whose score is not finite has no continuations (fewer beams than room: -infinity).  A logit that is not a number counts as
 * -infinity, and a logit of -infinity is no continuation; where logits are +infinity, the row's probability is shared among them.
 * Where there are fewer than `keep` continuations the places behind them receive -infinity, -1 and -1.
 * beams 1 .. 32, keep 1 .. 64 (twice the beams leaves room for those that end), vocab 1 .. 2^24, else GLLM_E_UNSUPPORTED;
 * workspace as above, GLLM_E_CAPACITY for one that is too small. */
gllm_status gllm_op_beam_select(const float* logits, int64_t ld_logits, const float* scores, int32_t num_seqs, int32_t beams,
                                int32_t vocab, int32_t keep, float* out_scores, int32_t* out_beams, int32_t* out_tokens,
                                void* workspace, size_t workspace_bytes, void* stream);
/* HOST only; 0 for sizes that the call does not take. */
size_t gllm_op_beam_select_workspace_bytes(int32_t num_seqs, int32_t beams, int32_t vocab, int32_t keep);

/* Copies page src[i] to page dst[i] in all layers of both pools, for i in [0, n).  src, dst: HOST, read before the call returns.
 * A page may be copied several times, but each destination is written once and none of them is a source as well
 * (GLLM_E_BLOCK_ALIAS); ids outside [0, num_blocks) give GLLM_E_BLOCK_RANGE.  Nothing is enqueued then.  Recorded into a graph, a
 * call copies the same pages at every replay. */
gllm_status gllm_op_copy_pages(void* k_pool, void* v_pool, int32_t num_layers, int64_t num_blocks, int32_t n_kv_heads,
                               int32_t head_dim, const int32_t* src, const int32_t* dst, int32_t n, void* stream);

#ifdef __cplusplus
}
#endif
#endif
