/*
 * ooco_batch.h -- C ABI of the operators of one step of a continuous batch.
 *
 * A serving instance whose sequences come, go, share prefixes and bring different numbers of tokens
 * (one of a decode, thousands of a prompt, a draft tree) runs
 *
 *   ooco_fork_pages             a child takes a parent's cache pages                 (between steps)
 *   ooco_release_pages          pages of finished or cut sequences become free       (between steps)
 *   ooco_plan_slots             (ooco_spec.h) blocks, slots and positions, packed     (once a step)
 *   ooco_norm_rope_kv_append    norms of q and k, rotary positions, append           (per layer)
 *   ooco_chunk_attention        the new tokens of all sequences over the paged cache (per layer)
 *   ooco_shape_logits           penalties, biases, grammar masks, probabilities      (once a step)
 *
 * (section 2.1 of the paper: continuous batching over a non-contiguous KV pool; section 3.4.1: pages of
 * evicted requests are freed; section 3.3: one iteration mixes prefill and decode tokens).  Conventions are
 * those of ooco.h and ooco_spec.h: the caller owns every buffer, work is enqueued on `cuda_stream` of the
 * current device, nothing is allocated and nothing synchronises, arguments are checked on the host before
 * anything is enqueued, the return value is OOCO_OK or a negative OOCO_E_* code, every call can be captured
 * into a graph, and two calls that may overlap on the GPU need outputs and workspaces of their own.
 */
#ifndef OOCO_BATCH_H_
#define OOCO_BATCH_H_

#include "ooco_spec.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Pages that several sequences hold.  shares[id] counts the sequences that hold block `id` beyond the
 * first: 0 for a block with one holder and for a free block, so blocks that ooco_plan_slots hands out need
 * no entry made.  Free ids lie in free_ids[free_head .. num_free), as ooco_plan_slots takes them; released
 * ids are put back in front of free_head.
 *
 * ooco_fork_pages: fork c gives row children[c] the first L tokens of row parents[c]; L = context_lens of
 * the parent, or the smaller of that and shared_lens[c].  The L / block_size full blocks are shared (the
 * child's row gets their ids, each one's count goes up); the tokens behind them lie in a block of the
 * child's own from the free list, and (copy_src[c], copy_dst[c]) names the copy to be made (the two lists
 * are arguments of ooco_kv_copy_blocks, which passes over the -1 of forks without one; make it before either
 * sequence goes on).  Blocks are taken in the order of the forks, with the rule of ooco_plan_slots: a fork
 * whose block the list does not hold on top of those of the forks before it is refused, takes nothing and
 * changes nothing (its need counts for the ones behind it; forks that need none are served).  A fork is
 * refused, too, and needs nothing, when a row lies outside [0, batch), its child is named twice, is a parent
 * of the call or holds blocks, or when the parent holds fewer blocks than L tokens need.
 *
 *   shape          batch (at most OOCO_MAX_PAGE_ROWS), block_size, num_blocks and max_blocks_per_seq are used
 *   num_forks      0 .. OOCO_MAX_PAGE_ROWS (OOCO_E_UNSUPPORTED beyond), num_forks * max_blocks_per_seq <= 2^30
 *   parents, children, shared_lens   device, int32 [num_forks]; shared_lens may be NULL, negative counts as 0
 *   context_lens, blocks_held        device, int32 [B]
 *   block_table    device, int32 [B, max_blocks_per_seq]; the children's entries are written
 *   free_ids       device, int32 [num_free]; free_head: device, int32 [1]
 *   shares         device, int32 [num_blocks]
 *   context_lens_out, blocks_held_out, free_head_out, shares_out   device, written whole; NULL = in place
 *   copy_src, copy_dst   device, int32 [num_forks], written: block ids, or -1 and -1 where nothing is to be copied
 *   granted        device, int32 [num_forks], written: 1, or 0 for a refused fork
 *   workspace      device, >= ooco_pages_workspace_bytes(shape, num_forks), 256-byte aligned
 *   status         device, int32 [1], may be NULL: OOCO_STATUS_REFUSED, OOCO_STATUS_BAD_BLOCK (an id outside the
 *                  pool: it is handed on, but not counted and not copied)
 * Nothing written may share memory with an input or another output, but for the in-place ones
 * (OOCO_E_SHAPE).  One launch for few table entries, two for many.
 *
 * ooco_release_pages: row rows[c] keeps its first keep_lens[c] tokens (NULL: none) and gives back the blocks
 * behind the last one that these need: a block with other holders loses one of them, a block without becomes
 * free.  The free blocks' ids are put into free_ids in front of free_head in the order of the list and, within
 * a row, of the table (a block that several rows of the list give back stands at the first of these places),
 * ending at free_head; ids for which the list has no room are dropped with OOCO_STATUS_REFUSED.  context_lens
 * becomes the smaller of itself and keep_lens, blocks_held the blocks kept; table entries stay.  A row outside
 * [0, batch) or named twice is refused; a row's blocks_held is clamped to [0, max_blocks_per_seq].
 *   free_ids is written in [new free_head, free_head); the rest as above.  One launch, or five for many table entries
 *   (num_rows * max_blocks_per_seq: the width of the table counts, as for the forks).
 * The last block that a cut row keeps may have other holders (shares of block_table[row, (keep - 1) / block_size] above 0, where
 * keep is no multiple of block_size): new tokens must not be written into it, though ooco_plan_slots would hand out its slots.
 * Such a row goes on as a fork of itself into an empty row (whose partly filled block is a copy).
 */
#define OOCO_MAX_PAGE_ROWS (1 << 18)
size_t ooco_pages_workspace_bytes(const ooco_shape_t* shape, int32_t num_rows);
int ooco_fork_pages(const ooco_shape_t* shape, int32_t num_forks, const int32_t* parents, const int32_t* children,
                    const int32_t* shared_lens, int32_t* context_lens, int32_t* block_table, int32_t* blocks_held,
                    const int32_t* free_ids, int32_t num_free, int32_t* free_head, int32_t* shares,
                    int32_t* context_lens_out, int32_t* blocks_held_out, int32_t* free_head_out, int32_t* shares_out,
                    int32_t* copy_src, int32_t* copy_dst, int32_t* granted, void* workspace, size_t workspace_bytes,
                    int32_t* status, void* cuda_stream);
int ooco_release_pages(const ooco_shape_t* shape, int32_t num_rows, const int32_t* rows, const int32_t* keep_lens,
                       int32_t* context_lens, const int32_t* block_table, int32_t* blocks_held, int32_t* free_ids,
                       int32_t num_free, int32_t* free_head, int32_t* shares, int32_t* context_lens_out,
                       int32_t* blocks_held_out, int32_t* free_head_out, int32_t* shares_out, void* workspace,
                       size_t workspace_bytes, int32_t* status, void* cuda_stream);

/* Norms of the heads of q and of k before they are turned. */
typedef struct {
  float eps;              /* >= 0, finite                                                            */
  float weight_offset;    /* added to every weight (1 for models that store weight - 1); finite      */
  const void* q_weight;   /* device, bf16 [head_dim], 16-byte aligned; NULL: no weights              */
  const void* k_weight;
} ooco_head_norm_t;

/*
 * ooco_rope_kv_append with a norm of every head of q and of k before the rotation:
 *     x  <-  x / sqrt(mean(x^2) + eps) * (weight + weight_offset)        over the head_dim values of a head
 * (weight + weight_offset = 1 where the weights are NULL).  v is taken as it is.  Computed in fp32, rounded
 * once, behind the rotation.  Everything else as for ooco_rope_kv_append and ooco_rope_kv_append_fp8.
 */
int ooco_norm_rope_kv_append(const ooco_shape_t* shape, const ooco_rope_t* rope, const ooco_head_norm_t* norm,
                             int32_t num_tokens, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, const int32_t* positions, const int32_t* slot_map,
                             void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache, void* cuda_stream);
int ooco_norm_rope_kv_append_fp8(const ooco_shape_t* shape, const ooco_rope_t* rope, const ooco_head_norm_t* norm,
                                 int32_t num_tokens, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                 const void* v, int64_t v_stride, const int32_t* positions, const int32_t* slot_map,
                                 void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache, float k_scale,
                                 float v_scale, void* cuda_stream);

typedef struct {
  int32_t batch;            /* B, 1 .. 2^24                                                            */
  int32_t max_nodes;        /* N rows per sequence, 1 .. OOCO_TREE_MAX_NODES                           */
  int32_t vocab;            /* V, 1 .. OOCO_MAX_SHAPED_VOCAB                                           */
  int32_t logits_fp32;      /* 0: bf16 logits, 1: fp32                                                 */
  int32_t history_width;    /* row width of `history`, 0 .. OOCO_MAX_HISTORY                            */
  int32_t max_bias;         /* entries per sequence of bias_tokens, 0 .. OOCO_MAX_BIAS                 */
  int64_t logits_seq_stride, logits_node_stride;  /* elements; rows of V consecutive values            */
  int64_t out_seq_stride, out_node_stride;
  int64_t probs_seq_stride, probs_node_stride;
  int64_t mask_seq_stride, mask_node_stride;      /* 32-bit words; 0 = one mask for all                */
} ooco_logits_t;
#define OOCO_MAX_SHAPED_VOCAB 409600
#define OOCO_MAX_BIAS 1024
#define OOCO_MAX_HISTORY (1 << 30)

/*
 * From logits to what a sampler, or ooco_verify_drafts, takes: for every row (sequence b, node i) and token v
 *   1. repetition: a token of the text gets  l > 0 ? l / repetition[b] : l * repetition[b]
 *   2. l <- l - frequency[b] * n(v) - presence[b] * [n(v) > 0],  n(v) = generated occurrences of v
 *   3. l <- l + sum of the biases listed for v, in their order
 *   4. l <- -inf where the mask has no bit for v
 *   5. probs = softmax over v of l / temperature[b]; a temperature that is not above 0: 1 at the lowest index
 *      of the largest l, 0 elsewhere.
 * The text of sequence b is history[b, 0 .. history_lens[b]), its first prompt_lens[b] tokens the prompt, the
 * rest generated.  With `tokens` the drafts of a node's branch (itself and its ancestors, the root, node 0, left
 * out: the history ends with it) count as generated text, too.  Steps 1 to 4 are done in fp32, every operation
 * rounded; a NaN counts as -inf from then on.  out_logits holds the result of step 4.  A row of which nothing is
 * left has probabilities of 0.  Equal infinite logits share the probability.
 *   logits         device, bf16 or fp32 with the strides of the struct
 *   temperature, repetition, frequency, presence   device, fp32 [B]; NULL: 1, 1, 0, 0 (a repetition that is not
 *                  above 0 counts as 1)
 *   history        device, int32 [B, history_width]; history_lens, prompt_lens: device, int32 [B], clamped to
 *                  [0, history_width]; prompt_lens NULL: 0.  Read only when one of the three penalties is given,
 *                  which needs history and history_lens
 *   tokens, parents   device, int32 [B, N] or NULL (parents NULL: a chain); tree_sizes: device, int32 [B] or NULL: N
 *   bias_tokens, bias_values   device, int32 and fp32 [B, max_bias], both or neither; a token outside [0, V) is
 *                  passed over, as in the history and the drafts
 *   mask           device, int32 words, bit v % 32 of word v / 32 set = v allowed; NULL: everything is
 *   out_logits, out_probs   device, fp32; one of them may be NULL.  Rows i >= tree_sizes[b] are left as they were
 * fp32 logits may be one of the outputs (same address and strides); otherwise the spans from the first to the last
 * element of an output, of another output and of an input do not meet, and an output's rows are distinct, with either of
 * its two strides the larger one (OOCO_E_SHAPE).  One launch.
 */
int ooco_shape_logits(const ooco_logits_t* shape, const void* logits, const float* temperature, const float* repetition,
                      const float* frequency, const float* presence, const int32_t* history, const int32_t* history_lens,
                      const int32_t* prompt_lens, const int32_t* tokens, const int32_t* parents, const int32_t* tree_sizes,
                      const int32_t* bias_tokens, const float* bias_values, const int32_t* mask, float* out_logits,
                      float* out_probs, void* cuda_stream);

/*
 * Causal attention of the new tokens of all sequences over the paged cache, rows packed as ooco_plan_slots packs
 * them: the query tokens of sequence b are rows first_row[b] .. of q and out, and are the LAST n_b tokens of its
 * context (their K / V are in the cache, context_lens[b] counts them); query i attends to tokens
 * [0, T_b - n_b + i + 1), with the formula of ooco_decode_attention.  A query that sees no token gives a zero row.
 *   n_b            first_row[b + 1] - first_row[b], or the smaller of that and chunk_lens[b]; negative counts as 0,
 *                  rows at or beyond num_rows do not exist and are not counted
 *   num_rows       rows of q and out; rows that belong to no query token are left as they were
 *   max_chunk      the caller's bound of n_b, 1 .. num_rows (which always is one): it decides which kernels are
 *                  launched and how large the workspace is.  A sequence that brings more is passed over, its rows left
 *                  as they were, and sets OOCO_STATUS_REFUSED in the workspace's status word
 *   q, out         device, bf16 [num_rows, Hq, head_dim], rows q_stride (out_stride) elements apart: multiples of 8, at
 *                  least the row's length; they share no memory (OOCO_E_SHAPE)
 *   first_row      device, int32 [B + 1]; chunk_lens: device, int32 [B] or NULL.  (ooco_plan_slots writes first_token,
 *                  granted_lens, and total_lens for context_lens.)  Rows of different sequences are distinct: where claims
 *                  of the same rows need more room than the workspace has for num_rows, all sequences, or all with one
 *                  new token, are passed over, and the status word is 1 (work list overflow)
 *   workspace      >= ooco_chunk_workspace_bytes(shape, num_rows, max_chunk), 256-byte aligned, read by
 *                  ooco_workspace_status
 * num_rows = 0 launches nothing.  Slots at or beyond T_b, table entries behind the last block used, and entries outside
 * the pool are treated as in ooco_decode_attention.  The K / V of a sequence's context must be finite, those of its later
 * new tokens among them: the products that the causal mask gives weight 0 are still formed inside a sequence.  The 8-bit
 * variant as ooco_decode_step_mq_fp8, but that a value x of q is rounded to f16 relative to the largest finite magnitude M of the
 * rows of its sequence and kv head: it is off by at most 2^-11 |x|, 2^-40 M or 2^-125.  One launch for few
 * sequences over a narrow table (of at most 2048 tokens, whatever the contexts), else up to five (plan, the kernels that
 * max_chunk asks for, merge).
 */
size_t ooco_chunk_workspace_bytes(const ooco_shape_t* shape, int32_t num_rows, int32_t max_chunk);
int ooco_chunk_attention(const ooco_shape_t* shape, int32_t num_rows, int32_t max_chunk, const void* q, int64_t q_stride,
                         const void* k_cache, const void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                         const int32_t* first_row, const int32_t* chunk_lens, float scale, void* out, int64_t out_stride,
                         void* workspace, size_t workspace_bytes, void* cuda_stream);
int ooco_chunk_attention_fp8(const ooco_shape_t* shape, int32_t num_rows, int32_t max_chunk, const void* q,
                             int64_t q_stride, const void* k_cache, const void* v_cache, const int32_t* block_table,
                             const int32_t* context_lens, const int32_t* first_row, const int32_t* chunk_lens, float scale,
                             float k_scale, float v_scale, void* out, int64_t out_stride, void* workspace,
                             size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* OOCO_BATCH_H_ */
