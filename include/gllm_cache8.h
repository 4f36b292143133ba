/* A KV cache held in 8 bits: the arrays of a step from its lengths, the store of a layer's keys and values, and the attention
 * that reads them.  The paper (arxiv 2504.14775, section 4.1) holds weights and activations in bf16 and says nothing of smaller
 * caches; what stands here is the public arithmetic of such a cache, for hybrid batches of prompt chunks and decode rows.
 *
 * A step: gllm_op_step_maps once, then for each layer gllm_op_gemm_bf16 (the QKV projection, float), gllm_op_norm_rope_store8 and
 * gllm_op_attention8.
 *
 * Same conventions as gllm_stage.h: plain C, every pointer marked HOST or DEVICE, DEVICE pointers belong to the current HIP
 * device, calls enqueue on `stream`, allocate nothing and return a gllm_status; there is no CPU fallback.  What lies on the device
 * is not read by the host: the calls can be recorded into a graph and replayed with other contents, and contents that break a
 * rule below are left out of the work as stated there, never followed out of the buffers.
 *
 * The pool of a layer: pages of 16 tokens; a value is its e4m3 code (OCP: 4 exponent bits, 3 mantissa bits, largest 448, no infinities)
 * times the float scale of its page, KV head and side.
 *   k_pool  DEVICE uint8 [num_blocks][n_kv][4][head_dim/16][4][16]: dim e of slot t of a page at [t / 4][e / 16][t % 4][e % 16]
 *   v_pool  DEVICE uint8 [num_blocks][n_kv][head_dim][16]
 *   scales  DEVICE float [num_blocks][n_kv][2]: of the keys, of the values; positive and finite
 * Attention counts a scale that is not, or that lies outside 2^-100 .. 2^100, as the nearest of these bounds (one that is not a number as
 * 2^-100).  Position p of a sequence is slot p % 16 of page block_tables[s][p / 16].  All pools are 16-byte aligned, scales 8-byte.
 */
#ifndef GLLM_CACHE8_H
#define GLLM_CACHE8_H

#include <stddef.h>
#include <stdint.h>

#include "gllm_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { GLLM_CACHE8_MAX_BLOCKS = 134217727 };  /* pages of a pool, so that a slot fits 31 bits */
enum { GLLM_ROWS_F32 = 0, GLLM_ROWS_BF16 = 1 };

/* What the operators below need to know of a step, from the lengths of its sequences.
 * Sequence s has new_tokens[s] rows (0: none) at positions cached_len[s] .. ; the pages of its new tokens that it does not hold yet,
 * those behind the first ceil(cached_len[s] / 16), are taken from free_pages in order of the sequences and positions.
 *   new_tokens, cached_len  DEVICE int32 [num_seqs]
 *   free_pages              DEVICE int32 [num_free]
 *   block_tables            DEVICE int32 [num_seqs][block_table_stride]: the entries of the pages taken are written (-1 where the
 *                           list has ended), the others are left as they are
 *   row_start               DEVICE int32 [num_seqs + 1] out
 *   positions, slots        DEVICE int32 [num_rows] out: of every row; slot = page * 16 + position % 16, or -1 where the page id is
 *                           outside [0, num_blocks).  Rows behind the last sequence (padding) receive 0 and -1
 *   needed                  DEVICE int32 [2] out: rows and pages that the lengths ask for (at most 2^31 - 1 is said), whether there are as many or not
 * A sequence with new_tokens < 0 counts as one without rows.  One with cached_len < 0 or more positions than its table row
 * has entries for (or than 2^31 - 64) takes no pages, its rows have position 0 and slot -1.  From the first sequence on whose rows would end
 * behind num_rows, sequences have no rows and take no pages.
 * GLLM_E_UNSUPPORTED above GLLM_CACHE8_MAX_BLOCKS blocks, GLLM_E_CAPACITY above 2^20 sequences. */
gllm_status gllm_op_step_maps(const int32_t* new_tokens, const int32_t* cached_len, int32_t num_seqs, const int32_t* free_pages,
                              int32_t num_free, int32_t* block_tables, int32_t block_table_stride, int64_t num_blocks, int32_t num_rows,
                              int32_t* row_start, int32_t* positions, int32_t* slots, int32_t* needed, void* stream);

/* One layer's queries, keys and values from its QKV projection: every query and key head h of a row becomes
 *   h * gain / sqrt(mean(h^2) + eps)           (where there is a gain; per head, over its head_dim elements)
 * and is rotated, elements i and i + head_dim/2 as a pair, by the angle of its position.  Queries are rounded to bf16; keys and values
 * to the nearest code (even where two are as near) of their page's scale, into their slots.
 *   qkv       DEVICE float or bf16 (rows_type) [num_rows][ld_qkv]: query heads, key heads, value heads (ld_qkv a multiple of 4, 16-byte
 *             aligned, bf16 8-byte)
 *   q_gain, k_gain  DEVICE bf16 [head_dim], 8-byte aligned, or NULL: heads as they are
 *   eps       0, or positive and inside float's range (else GLLM_E_INVALID)
 *   rope      DEVICE float [max_position][head_dim/2][2]: cosine and sine, 16-byte aligned; a position outside [0, max_position) is read
 *             as the nearest one inside
 *   positions, slots  DEVICE int32 [num_rows], as gllm_op_step_maps writes them.  Nothing is written for a row with a slot outside
 *             [0, num_blocks * 16).  The rows of a page stand within 16 rows, in any order, and have slots of their own
 *   q_out     DEVICE bf16 [num_rows][ld_q] (ld_q a multiple of 4, 8-byte aligned)
 * Scales: with m the largest finite magnitude that a page receives for a head and side, a page whose slot 0 is written has the scale
 * max(m / 448, 2^-100).  Any other keeps the tokens of the slots in front of those written: its scale grows by the least power of two
 * (at least 1) with which m / 448 fits, and the kept codes are divided by it and rounded; a scale that is not positive and finite counts as
 * 2^-100 there.  All other slots are left as they are.  A value that is not finite becomes the code that is not a number.
 * Supported: head_dim 64 or 128, any head counts with n_q_heads + 2 * n_kv_heads <= 65535 (else GLLM_E_UNSUPPORTED), at most
 * GLLM_CACHE8_MAX_BLOCKS blocks.  The mean of squares is held in float: with a gain, magnitudes up to 1e17, and sqrt(mean(h^2) + eps) from 1e-18 on
 * or 0 (then a head of zeros becomes 0 / 0).  GLLM_E_CAPACITY for more rows than a launch takes (there are none too many up to
 * num_rows * (n_q_heads + 2 * n_kv_heads) = 2^25). */
gllm_status gllm_op_norm_rope_store8(const void* qkv, int64_t ld_qkv, int32_t rows_type, const void* q_gain, const void* k_gain, double eps,
                                     const float* rope, int32_t max_position, const int32_t* positions, const int32_t* slots,
                                     int32_t num_rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, void* q_out, int64_t ld_q,
                                     void* k_pool, void* v_pool, float* scales, int64_t num_blocks, void* stream);

/* Attention of one layer: row r of `out` = softmax over the visible positions of (q[r] . k * scale), times v, per query head.  Row i of
 * sequence s stands at position p = cached_len[s] + i and sees the positions j <= p with j > p - window or j < sinks, all j <= p
 * where window is 0.
 *   q             DEVICE bf16 [num_rows][ld_q], rotated queries, head h in columns h*head_dim .. (ld_q a multiple of 8, 16-byte aligned)
 *   block_tables  DEVICE int32 [num_seqs][block_table_stride]; a page id outside [0, num_blocks) is read as the nearest one inside.  Entries
 *                 of blocks of four pages that no row of the sequence sees any position of are not followed; of other pages that no row sees
 *                 any position of, memory may be read, but what it holds reaches no result.  Both may have been given back
 *   cached_len    DEVICE int32 [num_seqs]: positions in front of the call's rows.  The keys and values of the rows themselves are in the
 *                 pool already
 *   row_start     DEVICE int32 [num_seqs + 1], ascending, from 0 up to at most num_rows (otherwise no row is written)
 *   max_new       HOST: most rows of any sequence; the kernels are chosen by it
 *   window, sinks HOST, >= 0 (sinks without a window: GLLM_E_INVALID)
 *   out           DEVICE bf16 [num_rows][ld_out] (ld_out a multiple of 4, 8-byte aligned)
 *   workspace     DEVICE, 16-byte aligned, at least gllm_op_attention8_workspace_bytes() of it; contents need not survive between calls,
 *                 and calls that may overlap in time need one each
 * All rows of a sequence with more than max_new, with cached_len < 0 or with more positions than its table row has entries for (or than
 * 2^31 - 64) receive zeros.  Rows outside every sequence are left as they are.  Codes in slots that no row sees may be anything; one that is
 * not a number spoils the rows that see it only.
 * Supported: head_dim 64 or 128, n_q_heads a multiple of n_kv_heads with at most 16 query heads per KV head, at most
 * GLLM_CACHE8_MAX_BLOCKS blocks (else GLLM_E_UNSUPPORTED); scale > 0 and at most 2.3e38 (else GLLM_E_INVALID), |q . k * scale| at most 1e8
 * and the values' magnitude at most 1e15 (beyond these, results are not).
 * GLLM_E_CAPACITY, with nothing enqueued, for a workspace that is too small, for more than 2^20 sequences and for more work than a launch takes
 * (there is none too much up to (num_rows * n_q_heads / n_kv_heads / 256 + num_seqs) * n_kv_heads = 2^22 and below 2^20 KV heads). */
gllm_status gllm_op_attention8(const void* q, int64_t ld_q, const void* k_pool, const void* v_pool, const float* scales, int64_t num_blocks,
                               const int32_t* block_tables, int32_t block_table_stride, const int32_t* cached_len,
                               const int32_t* row_start, int32_t num_seqs, int32_t num_rows, int32_t max_new, int32_t window, int32_t sinks,
                               int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float scale, void* out, int64_t ld_out,
                               void* workspace, size_t workspace_bytes, void* stream);
/* HOST only; 0 for head counts, a head size or max_new that the call does not take. */
size_t gllm_op_attention8_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_new);

#ifdef __cplusplus
}
#endif
#endif
