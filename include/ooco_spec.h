/*
 * ooco_spec.h -- C ABI of the operators of one speculative decoding step.
 *
 * A serving instance that drafts several tokens per request and step runs, per step:
 *
 *   ooco_plan_slots       blocks for the new tokens, their cache slots and positions   (once)
 *   ooco_rope_kv_append   rotary positions of q and k, k and v into the cache          (per layer)
 *   ooco_tree_attention   every drafted token attends to the context and its branch    (per layer)
 *   ooco_verify_drafts    the drafts against the target's probabilities                (once)
 *   ooco_kv_keep_path     the accepted branch's cache rows move together               (per layer)
 *
 * They work on the paged pool, the block tables and the shapes of ooco.h (section 2.1 of the paper:
 * a non-contiguous KV pool under continuous batching; section 2.3: a decode step's cost is the
 * reading of the cache, which a step of several tokens shares) and follow its conventions: the
 * caller owns every buffer, work is enqueued on `cuda_stream` of the current device, nothing is
 * allocated and nothing synchronises, arguments are checked on the host before anything is enqueued,
 * the return value is OOCO_OK or a negative OOCO_E_* code.  Every call can be captured into a graph.
 * Two calls that may overlap on the GPU need buffers (outputs, workspaces) of their own.
 *
 * The draft tree.  A sequence brings n nodes.  Node 0 is the root: the last token the sequence is
 * sure of, whose K / V are not in the cache yet.  parents[i] is the node above node i, with
 * parents[i] < i, or -1 for a node without one; a value outside [0, i) counts as -1.  A chain of
 * drafts is the tree parents[i] = i - 1.  Trees have at most OOCO_TREE_MAX_NODES nodes and lie in
 * padded rows of max_nodes entries per sequence; tree_sizes[b] (clamped to [0, max_nodes]) says how
 * many are real, NULL says all.  In the cache, node i of sequence b is token base + i, where base is
 * the sequence's context before the tree.
 */
#ifndef OOCO_SPEC_H_
#define OOCO_SPEC_H_

#include "ooco.h"

#ifdef __cplusplus
extern "C" {
#endif

#define OOCO_TREE_MAX_NODES 256
#define OOCO_MAX_VOCAB (1 << 20)

/* Bits of the optional status words below: OR-ed in, never cleared by the library. */
#define OOCO_STATUS_BAD_BLOCK 4   /* a block id outside [0, num_blocks) was met                   */
#define OOCO_STATUS_REFUSED 128   /* ooco_plan_slots: a sequence got no room for its new tokens   */

/*
 * Block tables and slot maps from request lengths.  Sequence b holds context_lens[b] tokens in
 * blocks_held[b] blocks (the first entries of its row of block_table) and brings new_lens[b] tokens.
 * In the order of the sequences each takes the blocks that it lacks,
 *     need_b = max(0, ceil((context_lens[b] + new_lens[b]) / block_size) - blocks_held[b]),
 * from free_ids[free_head ...], writes them behind the ones it holds, and every new token i gets
 *     slot = block * block_size + offset of token context_lens[b] + i,
 *     position = context_lens[b] + i, or context_lens[b] + depth of node i with `parents`.
 * A sequence is refused as a whole, takes nothing and has slots of -1 (positions are still written)
 * when the free list does not hold its blocks on top of those of the sequences before it (a refused
 * sequence's need counts for the ones behind it: blocks are not handed out past it, while sequences
 * that need none are served), when its table row, its padded row or the packed rows are too short,
 * when blocks_held does not cover its context, or when a block that it would use lies outside the pool
 * (the last only makes the slots of that block -1, and sets OOCO_STATUS_BAD_BLOCK).
 *
 *   shape          batch, block_size, num_blocks and max_blocks_per_seq are used; the other fields
 *                  must merely be valid; num_blocks * block_size < 2^31 (OOCO_E_UNSUPPORTED)
 *   context_lens, new_lens   device, int32 [B]; negative values count as 0
 *   block_table    device, int32 [B, max_blocks_per_seq]; the new entries are written
 *   blocks_held    device, int32 [B]
 *   free_ids       device, int32 [num_free]; free_head: device, int32 [1], index of the first free id
 *   blocks_held_out, free_head_out   device, int32 [B] and [1], written; NULL = in place
 *   row_len        0: packed rows, token i of sequence b is row first_token[b] + i;
 *                  > 0: padded rows, it is row b * row_len + i
 *   num_rows       rows of slot_map and positions: capacity (packed), or B * row_len (padded;
 *                  OOCO_E_SHAPE otherwise).  Rows without a token get slot and position -1.
 *   parents        device, int32 [num_rows], the tree of each sequence in the rows of its tokens;
 *                  NULL: positions count up
 *   slot_map, positions      device, int32 [num_rows], written
 *   first_token    device, int32 [B + 1], written: first row of each sequence, then the rows in use
 *                  (packed: saturates at num_rows)
 *   granted_lens, total_lens device, int32 [B], written: new_lens or 0, and the context with them
 *   workspace      device, >= ooco_plan_slots_workspace_bytes(shape), 256-byte aligned
 *   status         device, int32 [1], may be NULL
 * Nothing written may share memory with an input or another output, but for the two in-place ones
 * (OOCO_E_SHAPE).  One launch for few rows, two for many.
 */
size_t ooco_plan_slots_workspace_bytes(const ooco_shape_t* shape);
int ooco_plan_slots(const ooco_shape_t* shape, const int32_t* context_lens, const int32_t* new_lens,
                    int32_t* block_table, int32_t* blocks_held, const int32_t* free_ids, int32_t num_free,
                    int32_t* free_head, int32_t* blocks_held_out, int32_t* free_head_out, int32_t row_len,
                    int32_t num_rows, const int32_t* parents, int32_t* slot_map, int32_t* positions,
                    int32_t* first_token, int32_t* granted_lens, int32_t* total_lens, void* workspace,
                    size_t workspace_bytes, int32_t* status, void* cuda_stream);

/* How the frequencies of rotary positions are scaled for contexts longer than the trained one. */
enum {
  OOCO_ROPE_PLAIN = 0,     /* inv_freq[j] = base^(-2 j / rot_dim)                                       */
  OOCO_ROPE_LINEAR = 1,    /* every frequency divided by `factor` (interpolated positions)               */
  OOCO_ROPE_STRETCH = 2,   /* base replaced by base * factor^(rot_dim / (rot_dim - 2))                   */
  OOCO_ROPE_BANDS = 3,     /* by wavelength w = 2 pi / inv_freq: w < original_len / high: kept;
                              w > original_len / low: divided by factor; between: blended linearly in
                              original_len / w                                                          */
  OOCO_ROPE_RAMP = 4       /* by index: the frequencies that turn more than `high` times over
                              original_len are kept, those that turn less than `low` times divided by
                              factor, a linear ramp over the index between (its ends the whole indices
                              around it, in [0, rot_dim - 1]: it may end beyond the last frequency);
                              magnitude = 0.1 ln(factor) + 1                                             */
};
typedef struct {
  int32_t kind;          /* OOCO_ROPE_*                                        */
  int32_t original_len;  /* trained context (BANDS, RAMP)                      */
  double factor;         /* >= 1 (all but PLAIN)                               */
  double low, high;      /* BANDS: low < high; RAMP: low < high (turns)        */
} ooco_rope_scaling_t;

/*
 * Host arithmetic in 64 bits: the rot_dim / 2 frequencies, rounded to fp32 once, and the factor that
 * cosine and sine are multiplied by (1 except with OOCO_ROPE_RAMP).  scaling = NULL: plain.
 */
int ooco_rope_frequencies(int32_t rot_dim, double base, const ooco_rope_scaling_t* scaling,
                          float* inv_freq_host, float* magnitude_host);

typedef struct {
  int32_t rot_dim;        /* leading dims of each head that turn: a multiple of 16, <= head_dim        */
  int32_t interleaved;    /* 1: pairs (2 j, 2 j + 1); 0: pairs (j, j + rot_dim / 2)                    */
  float magnitude;        /* cosine and sine are multiplied by this; finite                           */
  int32_t reserved;       /* must be 0                                                                */
  const float* inv_freq;  /* device, fp32 [rot_dim / 2]                                               */
} ooco_rope_t;

/*
 * Rotary positions of the new tokens' q and k, and the append of k and v to the paged cache by slot:
 *     angle_j = positions[r] * inv_freq[j],   (x1, x2) -> (x1 c - x2 s, x2 c + x1 s) * magnitude
 * for every pair of the leading rot_dim dims of every head; the other dims and v are taken as they are.
 * The angle is formed and reduced in 64 bits, the rotation is computed in fp32 and rounded once.
 *   q, k, v      device, bf16 [num_tokens, Hq | Hkv | Hkv, head_dim], rows q_stride (k_stride,
 *                v_stride) elements apart, so they may be parts of one projection's output
 *   positions, slot_map   device, int32 [num_tokens] (as ooco_plan_slots writes them).  A row with a
 *                negative position is padding: nothing is written for it.  A row with a slot outside
 *                [0, num_blocks * block_size) leaves the cache alone (its q is still written).  No two
 *                rows may share a slot.
 *   q_out        device, bf16 rows q_out_stride apart, written; q itself is allowed (with its stride), rows that
 *                share memory with q's otherwise, with k's or with v's are not (OOCO_E_SHAPE)
 *   k_cache, v_cache      the pool of `shape`; word i of head h goes to
 *                block * kv_block_stride + h * kv_head_stride + offset * kv_token_stride + i
 * num_tokens = 0 launches nothing.  Strides are multiples of 8 elements, at least the row's length, and
 * addresses 16-byte aligned (OOCO_E_UNSUPPORTED).  _fp8: 8-bit caches as in ooco.h: the stored code is
 * e4m3(x / scale), x the rotated value in fp32 (no bf16 rounding before it), one division, round to
 * nearest even, saturating at 448; restrictions as for ooco_kv_append_fp8.  One launch.
 */
int ooco_rope_kv_append(const ooco_shape_t* shape, const ooco_rope_t* rope, int32_t num_tokens, const void* q,
                        int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                        const int32_t* positions, const int32_t* slot_map, void* q_out, int64_t q_out_stride,
                        void* k_cache, void* v_cache, void* cuda_stream);
int ooco_rope_kv_append_fp8(const ooco_shape_t* shape, const ooco_rope_t* rope, int32_t num_tokens, const void* q,
                            int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            const int32_t* positions, const int32_t* slot_map, void* q_out, int64_t q_out_stride,
                            void* k_cache, void* v_cache, float k_scale, float v_scale, void* cuda_stream);

/*
 * Attention of a draft tree over the paged cache: ooco_decode_attention_mq with another mask.  The last
 * n_b = tree_sizes[b] tokens of sequence b's context_lens[b] tokens are its tree's nodes; query i < n_b
 * attends to the tokens before the tree, to node i's ancestors and to node i itself.
 *   q, out        device, bf16 [B, max_nodes, Hq, head_dim], contiguous; rows i >= n_b of `out` are left
 *                 as they were, rows of q there are never used
 *   parents       device, int32 [B, max_nodes]
 *   tree_sizes    device, int32 [B], or NULL
 *   workspace     >= ooco_tree_workspace_bytes(shape, max_nodes), 256-byte aligned
 * A sequence with n_b = 0 reads nothing.  A node whose token index is negative (context_lens[b] < n_b)
 * does not exist: nobody attends to it; a query that sees no token gives a zero row.  The K / V of the
 * nodes must be finite, as must those of the context: the products that a mask gives weight 0 are
 * still formed inside a sequence (slots beyond context_lens[b] may hold anything).
 * 1 <= max_nodes <= OOCO_TREE_MAX_NODES (OOCO_E_UNSUPPORTED beyond).  Status word, launches (three) and
 * everything else as for ooco_decode_attention_mq; of the launch-shape knobs only 3, 4, 5, 8 and 13 apply.
 * The 8-bit variant as for ooco_decode_step_mq_fp8.
 */
size_t ooco_tree_workspace_bytes(const ooco_shape_t* shape, int32_t max_nodes);
int ooco_tree_attention(const ooco_shape_t* shape, int32_t max_nodes, const void* q, const void* k_cache,
                        const void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                        const int32_t* parents, const int32_t* tree_sizes, float scale, void* out,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);
int ooco_tree_attention_fp8(const ooco_shape_t* shape, int32_t max_nodes, const void* q, const void* k_cache,
                            const void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                            const int32_t* parents, const int32_t* tree_sizes, float scale, float k_scale,
                            float v_scale, void* out, void* workspace, size_t workspace_bytes, void* cuda_stream);

typedef struct {
  int32_t batch;              /* B                                                                    */
  int32_t max_nodes;          /* N, 1 .. OOCO_TREE_MAX_NODES                                          */
  int32_t vocab;              /* V, 1 .. OOCO_MAX_VOCAB                                               */
  int32_t reserved;           /* must be 0                                                            */
  int64_t target_seq_stride, target_node_stride;  /* elements; rows of V consecutive fp32 values      */
  int64_t draft_seq_stride, draft_node_stride;
} ooco_verify_t;

/*
 * Verification of drafted tokens against the target's probabilities from given random numbers: the
 * accepted tokens and the one drawn behind them are distributed as the target alone would draw them.
 * p_i is the target's distribution after node i (row i of target_probs), q_i the draft's, from which
 * node i's children were drawn independently of one another.  From the root on, the children of the
 * current node are asked in the order of their indices, with weights w = p, w's mass Z = 1 and S = 0:
 *     child c with token x is accepted iff  uniforms[c] * Z * q(x) < w(x),   w(x) = max(p(x) - S q(x), 0);
 *     otherwise S <- S + Z, then Z <- sum of w with that S (which is w <- max(w - Z q, 0)).
 * An accepted child becomes the current node.  When no child is left, the last token is
 *     the lowest index whose cumulative sum of w exceeds uniforms[0] * sum of w
 * at the current node (w = p again where w's sum is 0; token 0 where that sum is 0, too, or not finite).
 * With draft_probs = NULL the drafts were not drawn but chosen: a child is accepted iff
 * uniforms[c] * Z < w(x), and a refused one's token leaves w (w(x) <- 0, Z <- Z - w(x)).
 * Products, differences and sums are unevaluated pairs of fp32 values, which carry about 46 bits (24 where
 * the pair's low part falls below fp32's range: products under about 2^-102).  So a decision is that of the
 * exact formula unless the two sides of its comparison, or uniforms[0] * sum and the border of a cumulative
 * sum, are nearer than about 2^-40 * (1 + S).
 *   target_probs, draft_probs   device, fp32, [B, N, V] with the strides of the struct.  Rows sum to 1; a NaN or
 *                  negative value counts as 0, in either.  Of every node with children one value per child is
 *                  read in both, whether the walk reaches it or not (its value is used only then); whole rows are
 *                  read of nodes that are reached: in draft_probs where a child was refused, in target_probs
 *                  there and where the last token is drawn.  Rows of leaves in draft_probs are never read
 *   tokens         device, int32 [B, N]: the drafted tokens (entry 0 is not read); a token outside
 *                  [0, V) is never accepted
 *   parents        device, int32 [B, N]; NULL: a chain
 *   tree_sizes     device, int32 [B]; NULL: all N nodes
 *   uniforms       device, fp32 [B, N], in [0, 1): entry i for node i, entry 0 for the last token
 *   path           device, int32 [B, N], written: the root, then the accepted nodes, then -1
 *   out_tokens     device, int32 [B, N], written: the accepted tokens, the last token, then -1
 *   num_accepted   device, int32 [B], written: accepted drafts (the root and the last token not counted)
 * A sequence without nodes gets -1 everywhere and num_accepted 0.  One launch (a thread-block cluster per
 * sequence).
 */
int ooco_verify_drafts(const ooco_verify_t* shape, const float* target_probs, const float* draft_probs,
                       const int32_t* tokens, const int32_t* parents, const int32_t* tree_sizes,
                       const float* uniforms, int32_t* path, int32_t* out_tokens, int32_t* num_accepted,
                       void* cuda_stream);

/*
 * Keeps the accepted branch: the cache rows (K and V, every head) of token base_lens[b] + path[b, j] move
 * to token base_lens[b] + j, for j = 1 .. num_accepted[b], so that the context goes on without gaps;
 * rows behind it are left as they were.
 *   path          device, int32 [B, max_nodes], increasing, path[b, 0] = 0 (as ooco_verify_drafts writes
 *                 it); a row that starts with -1 keeps nothing.  The branch ends before the first entry
 *                 that does not lie above the one before it and below max_nodes.
 *   num_accepted  device, int32 [B], clamped to [0, max_nodes - 1]
 *   base_lens     device, int32 [B]: context before the tree
 *   context_lens_out  device, int32 [B], written: base + 1 + accepted (base where nothing is kept);
 *                 may be NULL; shares no memory with an input (OOCO_E_SHAPE)
 * A move whose token lies beyond the block table or in a block outside the pool is skipped.  The sequences'
 * blocks that hold nodes are distinct.  One launch; words are copied as they are (_fp8: bytes).
 */
int ooco_kv_keep_path(const ooco_shape_t* shape, int32_t max_nodes, void* k_cache, void* v_cache,
                      const int32_t* block_table, const int32_t* base_lens, const int32_t* path,
                      const int32_t* num_accepted, int32_t* context_lens_out, void* cuda_stream);
int ooco_kv_keep_path_fp8(const ooco_shape_t* shape, int32_t max_nodes, void* k_cache, void* v_cache,
                          const int32_t* block_table, const int32_t* base_lens, const int32_t* path,
                          const int32_t* num_accepted, int32_t* context_lens_out, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* OOCO_SPEC_H_ */
