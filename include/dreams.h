/*
 * dreams.h -- C ABI of libdreams.so, the MI355X (gfx950) tree-verification step of DREAM-S speculative
 * decoding for vision-language models.
 *
 * The step has three verbs (acceptance in three forms), run back to back on one HIP stream:
 *   dreams_tree_verify_attn  tree-masked attention of the draft-token tree against the KV cache
 *   dreams_tree_accept       greedy acceptance of the longest target-consistent root-to-node path
 *   dreams_tree_accept_sampled  acceptance at temperature tau > 0 (accept-or-resample down the tree)
 *   dreams_tree_accept_lm_head  greedy acceptance from final hidden states (LM head fused with the argmax)
 *   dreams_kv_commit         compaction of the accepted path's K/V into the cache
 * The cache is one slab of slots per sequence and KV head, or pages of a pool that sequences share ("Paged cache" below:
 * the attention of a tree and of a prompt over pages, the rows that go into them, and the tables' upkeep), in 16 or 32 bits
 * or in 8 ("Pages of 8 bits").  Queries and keys get their positions by rotation ("Rotary positions"), on their way into
 * pages or by themselves.
 *
 * Conventions shared by every entry point
 *   - Pointers named as "device" point to device memory the caller owns (allocated on the current HIP
 *     device).  The library never allocates or frees inside a call; scratch memory comes in through a
 *     caller-owned workspace sized by the matching *_workspace_size query.
 *   - Calls are asynchronous and stream-ordered: they enqueue kernels on `stream` and return.  Outputs are
 *     valid once the stream has reached that point.  Calls that share a workspace must be ordered (same
 *     stream, or synchronised streams).
 *   - Host-visible arguments (sizes, flags, null pointers) are checked before anything is enqueued; on a
 *     failed check the call returns a negative status, sets the thread's last error message and enqueues
 *     nothing.  Values that live in device memory (kv_len, parent, accept_path, ...) cannot be checked on the
 *     host; the kernels clamp or skip out-of-range entries so that no access leaves the caller's buffers,
 *     and the results for such entries are unspecified.
 *   - A HIP launch error returns DREAMS_ERR_HIP.
 *   - Element types: DREAMS_BF16 tensors hold bfloat16 bit patterns (round-to-nearest-even); DREAMS_F32
 *     tensors hold IEEE binary32; DREAMS_E4M3 pages hold 8-bit codes with a scale for each 16 slots of a head.
 */
#ifndef DREAMS_H
#define DREAMS_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DREAMS_OK = 0,
  DREAMS_ERR_INVALID_ARG = -1,  /* a host-visible argument is out of range or a required pointer is NULL */
  DREAMS_ERR_UNSUPPORTED = -2,  /* valid in principle but not built (e.g. a head_dim other than 64/128)   */
  DREAMS_ERR_WORKSPACE = -3,    /* workspace NULL or too small (*_workspace_size bytes are always enough)  */
  DREAMS_ERR_HIP = -4,          /* the HIP runtime reported an error (device query or kernel launch)     */
  DREAMS_ERR_DEVICE = -5        /* a kernel of an earlier call flagged a failure (dreams_workspace_status) */
} dreams_status_t;

/* (DREAMS_E4M3: pages of 8 bits, in the calls named *_e4m3 only) */
typedef enum { DREAMS_F32 = 0, DREAMS_BF16 = 1, DREAMS_E4M3 = 2 } dreams_dtype_t;

/*
 * Workspaces.  Every workspace (of either verb that takes one) begins with DREAMS_WORKSPACE_COUNTER_BYTES
 * bytes of arrival counters.  Zero-fill that region once, before the workspace is first used (zeroing the
 * whole buffer after allocating it does this).  Every call, of any shape, leaves the region zero again when it
 * completes, so one workspace of sufficient size can serve calls of different shapes and of every verb one
 * after another.  The region's last 128 bytes hold failure flags instead of counters: a kernel that meets a
 * condition it cannot complete under (listed at dreams_workspace_status) sets one and leaves it set until
 * dreams_workspace_status reads and clears it.  Calls that overlap in time on one workspace (different
 * streams without synchronisation) race and give unspecified results.  Workspaces must be 256-byte aligned.
 */
#define DREAMS_WORKSPACE_COUNTER_BYTES 65536

/*
 * dreams_workspace_status -- the failures kernels flagged in `workspace` (device, 256-byte aligned, a workspace
 * of any verb, workspace_bytes >= DREAMS_WORKSPACE_COUNTER_BYTES, else DREAMS_ERR_WORKSPACE) since the last
 * check.  Synchronises `stream`, reads the flags, clears them, and returns DREAMS_OK if none was set, else
 * DREAMS_ERR_DEVICE with a message naming each flag.  The flags:
 *   attention (more than one piece per row set): the pieces of one set did not all run on one XCD, so the
 *       merge could not read their partial results from its XCD's L2 -- the rows of that set are NaN.  Not
 *       expected on an MI355X (consecutive workgroups of a dispatch run on consecutive XCDs, so workgroups
 *       whose ids agree mod 8 share one).
 *   a wait for another workgroup's results gave up (dreams_set_wait_limit; attention merges, sampled
 *       acceptance): that call's results are unspecified (attention rows NaN).
 * After a flagged failure, zero the workspace's counter region before it serves another call: arrivals that
 * came after a wait gave up can remain there.  Not for use under stream capture (it copies to the host and
 * synchronises).
 */
dreams_status_t dreams_workspace_status(void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * dreams_set_wait_limit -- the bound, in seconds (0 .. 60, default 0.2), on every wait of one workgroup for
 * another's results inside the library's kernels: the merging workgroups of dreams_tree_verify_attn (several
 * pieces per row set) and the pieces of dreams_tree_accept_sampled.  Those waits always end in normal operation
 * (a workgroup only waits for ones dispatched before it); a wait that reaches the bound gives up, its call's
 * results are unspecified, and the workspace's failure flag is set (dreams_workspace_status).  A limit of 0
 * makes every such wait give up at once, which exercises that path.  Applies to calls enqueued after it;
 * process-wide.
 */
dreams_status_t dreams_set_wait_limit(double seconds);

/*
 * Shape of one tree-verification attention call.
 *   batch            B >= 0 sequences
 *   num_q_heads      Hq >= 1 query heads
 *   num_kv_heads     Hkv >= 1 KV heads, Hq % Hkv == 0 (query head h reads KV head h / (Hq/Hkv))
 *   head_dim         D, 64 or 128
 *   num_nodes        T, 1..128 tree nodes per sequence, root included (node 0 = the last emitted token)
 *   cache_capacity   S_cap >= T slots per (sequence, KV head)
 *   max_kv_len       host-side upper bound on every kv_len[b], used only to plan the work split;
 *                    0 means S_cap - T.  Must satisfy 0 <= max_kv_len <= S_cap - T.
 *   num_splits       number of pieces the key axis of each (sequence, KV head) is cut into; 0 lets the
 *                    library choose from the shape and the device's compute-unit count.  Any value gives
 *                    the same result up to floating-point rounding order.
 *   dtype            type of q, the caches and out: DREAMS_BF16 (matrix-core path) or DREAMS_F32
 *   scale            softmax scale applied to q.k (normally 1/sqrt(D))
 */
typedef struct {
  int32_t batch;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t num_nodes;
  int32_t cache_capacity;
  int32_t max_kv_len;
  int32_t num_splits;
  dreams_dtype_t dtype;
  float scale;
} dreams_attn_desc_t;

/* Bytes of workspace dreams_tree_verify_attn needs for `desc` on the current device (0 if none: then the
 * call accepts a NULL workspace).  Non-zero when the key axis is cut into pieces: the pieces' partial
 * results live there, after the counter region every workspace starts with.
 * Where the library chooses the pieces (num_splits 0), a call that brings less than this, but room for as many
 * pieces as leave each 384 keys or more, is not refused: it is cut into those, and its results differ from those
 * with a whole workspace by the pieces' rounding.  Results that must not depend on the workspace's size take
 * num_splits from dreams_tree_verify_attn_splits. */
dreams_status_t dreams_tree_verify_attn_workspace_size(const dreams_attn_desc_t* desc, size_t* bytes);

/* Number of pieces dreams_tree_verify_attn cuts the key axis of every (sequence, KV head) into for `desc` on
 * the current device (desc->num_splits, clamped, or the library's choice when it is 0, for a workspace of
 * dreams_tree_verify_attn_workspace_size bytes). */
dreams_status_t dreams_tree_verify_attn_splits(const dreams_attn_desc_t* desc, int32_t* splits);

/*
 * dreams_tree_verify_attn -- the target model's parallel verification pass, attention part (the paper,
 * Section 2, "Speculative decoding": the target checks all draft tokens in one pass; Section 3.2 defines the
 * attention matrix softmax(Q K^T / sqrt(z))).  For every sequence b, query head h and tree node i:
 *
 *     out[b,h,i,:] = softmax_j( scale * q[b,h,i,:] . k[b,g,j,:] ) v[b,g,j,:],   g = h / (Hq/Hkv)
 *
 * over the visible slots j: every committed prefix slot 0..L_b-1 (image and text tokens alike -- the
 * paper's Section 2, "Vision-Language Models", notes every visual token stays in the KV cache and is
 * attended at each decoding step), plus slot L_b + n for every tree node n that is node i itself or one of
 * its ancestors.  lse[b,h,i] = log(sum_j exp(scale * q.k_j)) (natural log).  A row with no visible slot
 * (possible only with a tree_mask and L_b = 0) gives out = 0 and lse = -inf.
 *
 *   q          device [B, Hq, T, D]      queries of the tree nodes (after any positional rotation)
 *   k_cache    device [B, Hkv, S_cap, D] keys: slots [0, L_b) committed prefix, [L_b, L_b+T) the tree
 *                                         nodes' own keys in node order (written by the caller beforehand)
 *   v_cache    device [B, Hkv, S_cap, D] values, same layout
 *   kv_len     device [B] int32          L_b; the kernel clamps it into [0, S_cap - T]
 *   parent     device [B, T] int32       parent[b,0] = -1, 0 <= parent[b,i] < i; ignored when tree_mask is
 *                                         given.  An entry breaking these rules ends that node's ancestor walk.
 *   tree_mask  device [B, T, ceil(T/64)] uint64, or NULL: bit n of row i set <=> slot L_b+n is visible to
 *                                         node i.  Takes precedence over parent.
 *   out        device [B, Hq, T, D]      same dtype as q
 *   lse        device [B, Hq, T] float, or NULL
 *   workspace  device, >= dreams_tree_verify_attn_workspace_size bytes (see "Workspaces" above, and that
 *              function for a smaller one), or NULL when that size is 0.
 * Arithmetic: bf16 products accumulated in fp32 on the matrix cores, softmax statistics in fp32, one
 * rounding of the probabilities to bf16 before the value product; output rounded to the nearest bf16.  With
 * more than one piece of the key axis (dreams_tree_verify_attn_splits), each piece's output is rounded to
 * bf16 once more before the pieces are merged in fp32.
 */
dreams_status_t dreams_tree_verify_attn(const dreams_attn_desc_t* desc, const void* q, const void* k_cache,
                                        const void* v_cache, const int32_t* kv_len, const int32_t* parent,
                                        const uint64_t* tree_mask, void* out, float* lse, void* workspace,
                                        size_t workspace_bytes, hipStream_t stream);

/*
 * dreams_tree_verify_attn_noalloc -- dreams_tree_verify_attn for callers that cannot allocate device memory
 * (code under stream capture, tight serving loops, harnesses that forbid hipMalloc): the same arguments without
 * a workspace, the same kernels and the same results.  The scratch memory lives in a fixed array of
 * DREAMS_NOALLOC_SCRATCH_BYTES bytes inside the library, one per device, held until the process ends; the
 * call allocates and frees nothing.  Shapes whose workspace (dreams_tree_verify_attn_workspace_size) exceeds
 * that size return DREAMS_ERR_UNSUPPORTED before anything is enqueued.  The first call on a device also
 * enqueues one small kernel that clears the array's counters.  Every call on a device shares that device's
 * array, so calls that overlap in time on one device (different streams without synchronisation) race and
 * give unspecified results.  A failure a kernel flags (see dreams_workspace_status) stays in the array and
 * is not reported; the rows concerned are NaN.
 */
#define DREAMS_NOALLOC_SCRATCH_BYTES (16u << 20)
dreams_status_t dreams_tree_verify_attn_noalloc(const dreams_attn_desc_t* desc, const void* q, const void* k_cache,
                                                const void* v_cache, const int32_t* kv_len, const int32_t* parent,
                                                const uint64_t* tree_mask, void* out, float* lse, hipStream_t stream);

/*
 * dreams_tree_verify_attn_entropy -- dreams_tree_verify_attn, plus the attention entropy of every row: the
 * per-row term of the average attention entropy AE(l) by which the paper's Section 3.2 ("Adaptive
 * Intermediate Feature Distillation") ranks target layers.
 *
 *   entropy[b,h,i] = - sum_j A[j] ln A[j]   over the slots row (b,h,i) sees, A = its attention probabilities
 *                    (natural log; 0 for a row with no visible slot)
 *
 * Arguments, layouts, workspace and errors as dreams_tree_verify_attn; entropy is device [B, Hq, T] float
 * (required, 4-byte aligned).  The entropy is computed in the same pass over the keys as out and lse (one
 * more fp32 sum per row next to the softmax denominator), from the fp32 probabilities before their bf16
 * rounding.
 */
dreams_status_t dreams_tree_verify_attn_entropy(const dreams_attn_desc_t* desc, const void* q, const void* k_cache,
                                                const void* v_cache, const int32_t* kv_len, const int32_t* parent,
                                                const uint64_t* tree_mask, void* out, float* lse, float* entropy,
                                                void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * dreams_attn_entropy_mean -- AE of one layer (Section 3.2): the mean of `count` >= 1 row entropies, e.g. the
 * B*Hq*T values one dreams_tree_verify_attn_entropy call wrote (every head and sequence counts alike).
 * entropy: device [count] float; ae: device, one float (out).  Summed in fp64 in a fixed order.
 */
dreams_status_t dreams_attn_entropy_mean(int64_t count, const float* entropy, float* ae, hipStream_t stream);

/*
 * dreams_attn_entropy_select -- the distillation layer of Section 3.2: the layer l minimising
 * AE(l) + |AE(l) - AE(l-1)| (entropy plus its change from the layer below).  The change needs a
 * predecessor, so the candidates are l = 1 .. num_layers-1 (num_layers >= 2); scores are fp32 and ties go to
 * the smaller l.  ae: device [num_layers] float; best: device, one int32 (out).
 */
dreams_status_t dreams_attn_entropy_select(int32_t num_layers, const float* ae, int32_t* best, hipStream_t stream);

/*
 * Target-aware visual-token selection (the paper's Section 3.1, "Visual Token Compression", Eq. 2).
 *
 * dreams_visual_importance -- the importance of visual token j (cache slot vis_begin + j of every sequence):
 *   importance[b,j] = (1 / (Hq*T)) * sum over query heads h and rows i of A[b,h,i,vis_begin+j]
 * where A[b,h,i,.] is row (b,h,i)'s attention as dreams_tree_verify_attn defines it (same desc, q, k_cache and
 * kv_len; lse = that call's log-sum-exp output, [B, Hq, T]).  A visual slot at or past a sequence's prefix
 * length has importance 0; a row whose lse is -inf contributes nothing.  bf16 only (DREAMS_ERR_UNSUPPORTED
 * otherwise).  importance: device [B, vis_count] float (out).  Requires vis_begin >= 0, vis_count >= 1,
 * vis_begin + vis_count <= cache_capacity and B * ceil(vis_count / 256) <= (DREAMS_WORKSPACE_COUNTER_BYTES - 128) / 4
 * (DREAMS_ERR_UNSUPPORTED otherwise).  workspace: device, 256-byte aligned, >=
 * dreams_visual_importance_workspace_size bytes: the arrival-counter region every workspace starts with (see
 * "Workspaces" above), then B*Hkv*vis_count floats of per-KV-head partial sums.  Arithmetic: bf16 products, fp32
 * sums; the heads are summed in head order, so results are reproducible.
 */
dreams_status_t dreams_visual_importance_workspace_size(int32_t batch, int32_t num_kv_heads, int32_t vis_count,
                                                        size_t* bytes);
dreams_status_t dreams_visual_importance(const dreams_attn_desc_t* desc, const void* q, const void* k_cache,
                                         const int32_t* kv_len, const float* lse, int32_t vis_begin,
                                         int32_t vis_count, float* importance, void* workspace,
                                         size_t workspace_bytes, hipStream_t stream);

/*
 * dreams_visual_topk -- the keep_count most important visual tokens of every sequence: keep[b] lists them in
 * increasing token order.  Ranking: larger importance first, the smaller token index among equal values
 * (exact fp32 comparisons; importance must not hold NaN).  importance device [B, vis_count] float, with
 * 1 <= vis_count <= DREAMS_VISUAL_MAX_TOKENS and 1 <= keep_count <= vis_count; keep device [B, keep_count] int32.
 */
#define DREAMS_VISUAL_MAX_TOKENS 8192
dreams_status_t dreams_visual_topk(int32_t batch, int32_t vis_count, int32_t keep_count, const float* importance,
                                   int32_t* keep, hipStream_t stream);

/*
 * dreams_visual_gather -- the kept tokens' K/V rows, for a cache that holds only them:
 *   k_out[b,g,m,:] = k_cache[b,g,vis_begin + keep[b,m],:]   (same for v), bit for bit
 * k_cache, v_cache device [B, Hkv, S_cap, D] of dtype; keep device [B, keep_count] int32 (as dreams_visual_topk
 * writes it); k_out, v_out device [B, Hkv, keep_count, D].  head_dim * element size must be a multiple of 16.
 * A kept token whose slot falls outside the cache leaves its output rows unwritten.
 */
dreams_status_t dreams_visual_gather(int32_t batch, int32_t num_kv_heads, int32_t head_dim, int32_t cache_capacity,
                                     dreams_dtype_t dtype, const void* k_cache, const void* v_cache,
                                     int32_t vis_begin, const int32_t* keep, int32_t keep_count, void* k_out,
                                     void* v_out, hipStream_t stream);

/*
 * Prefill statistics: the same quantities over a prompt's own causal attention, which is where the paper reads
 * them -- Eq. 2 (Section 3.1, "Visual Token Compression") scores visual tokens with the final layer's attention
 * weights of the prefilling pass, and AE(l) (Section 3.2) averages the attention entropy of a layer's rows over
 * the n prompt tokens.  Prompt b holds n_b = prompt_len[b] tokens (clamped to [0, num_rows]): queries in rows
 * 0..n_b-1 of q [B, Hq, num_rows, D], keys in slots 0..n_b-1 of k_cache [B, Hkv, cache_capacity, D], both bf16,
 * caller-owned device buffers; query head h reads KV head h / (Hq/Hkv).  Row i attends slots 0..i:
 *   A[b,h,i,j] = exp(scale * q_i . k_j - lse[b,h,i]),  lse[b,h,i] = log sum_{j <= i} exp(scale * q_i . k_j).
 * Arithmetic: bf16 products, fp32 sums.  head_dim 64 or 128 (DREAMS_ERR_UNSUPPORTED otherwise).
 */
typedef struct {
  int32_t batch;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t num_rows;        /* N: rows per head of q, the longest prompt */
  int32_t cache_capacity;  /* slots per (sequence, KV head) of k_cache, >= num_rows */
  float scale;
} dreams_prefill_desc_t;

/*
 * dreams_prefill_attn_stats -- lse[b,h,i] (natural log) and entropy[b,h,i] = -sum_{j<=i} A log A (nats) of every
 * prompt row; rows i >= n_b get lse = -inf and entropy 0.  lse and entropy: device [B, Hq, num_rows] float,
 * either may be NULL.  Nothing is allocated; no workspace.
 */
dreams_status_t dreams_prefill_attn_stats(const dreams_prefill_desc_t* desc, const void* q, const void* k_cache,
                                          const int32_t* prompt_len, float* lse, float* entropy,
                                          hipStream_t stream);

/*
 * dreams_prefill_attn_entropy_mean -- AE of one layer over prompts (Section 3.2): the sum of entropy
 * [B, Hq, num_rows] (as dreams_prefill_attn_stats wrote it: 0 past each prompt) over Hq * sum_b n_b rows, summed
 * in fp64 in a fixed order; 0 when no prompt has a row.  ae: device, one float (out).
 */
dreams_status_t dreams_prefill_attn_entropy_mean(int32_t batch, int32_t num_q_heads, int32_t num_rows,
                                                 const float* entropy, const int32_t* prompt_len, float* ae,
                                                 hipStream_t stream);

/*
 * dreams_prefill_visual_importance -- Eq. 2 over the prompt: for visual token j (slot vis_begin + j),
 *   importance[b,j] = (1 / (Hq * n_b)) * sum_h sum_{i < n_b} A[b,h,i,vis_begin+j]
 * (a slot past row i gets nothing from it; a slot at or past n_b has importance 0; n_b = 0 gives 0).  lse: the
 * [B, Hq, num_rows] output of dreams_prefill_attn_stats on the same inputs.  Requires vis_begin >= 0,
 * vis_count >= 1, vis_begin + vis_count <= num_rows.  workspace: as for dreams_visual_importance (at least
 * dreams_visual_importance_workspace_size(batch, num_kv_heads, vis_count) bytes; its counter region zero, and left
 * zero).  importance: device [B, vis_count] float (out).  The heads are summed in head order (reproducible).
 *
 * With few KV heads or visual tokens the rows of a head are cut into pieces for more workgroups, each with partial
 * sums of its own in the workspace: dreams_prefill_visual_importance_workspace_size bytes hold all of them.  A
 * smaller workspace gets as many pieces as it holds (a slower call, sums of fewer pieces in the same order).
 */
dreams_status_t dreams_prefill_visual_importance_workspace_size(int32_t batch, int32_t num_kv_heads, int32_t vis_count,
                                                                size_t* bytes);

dreams_status_t dreams_prefill_visual_importance(const dreams_prefill_desc_t* desc, const void* q, const void* k_cache,
                                                 const int32_t* prompt_len, const float* lse, int32_t vis_begin,
                                                 int32_t vis_count, float* importance, void* workspace,
                                                 size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace dreams_tree_accept needs (0 only when batch is 0).  DREAMS_ERR_UNSUPPORTED if batch
 * exceeds (DREAMS_WORKSPACE_COUNTER_BYTES - 128) / 4 (one arrival counter per sequence, plus up to 8 group counters
 * per sequence while batch * 9 counters fit).  After the counters: one (value, index) pair per piece of each
 * row (rows of long vocabularies are cut into pieces). */
dreams_status_t dreams_tree_accept_workspace_size(int32_t batch, int32_t num_nodes, int32_t vocab,
                                                  size_t* bytes);

/*
 * dreams_tree_accept -- greedy acceptance (the paper, Section 2, "Speculative decoding": a draft token is
 * kept while it equals the target's own token at its position; at the first mismatch the target's token is
 * used instead), applied to every root-to-node path of the tree.
 *
 *   tgt[i]  = the smallest vocabulary index attaining max_v target_logits[b,i,v]   (-0.0 equals +0.0)
 *   node i is consistent iff i = 0, or its parent is consistent and draft_tokens[b,i] == tgt[parent[i]]
 *   last    = the consistent node of greatest depth, smallest index among equals
 *   accept_len[b]  = depth(last) = number of accepted draft tokens a  (the step emits a + 1 tokens)
 *   accept_path[b] = node ids root .. last (a + 1 entries), then -1 up to T entries
 *   next_token[b]  = tgt[last], the target's token emitted after the accepted drafts
 *
 *   target_logits  device [B, T, V] float, finite (NaN gives unspecified results)
 *   draft_tokens   device [B, T] int32 (entry 0 = root token, not checked)
 *   parent         device [B, T] int32, as for dreams_tree_verify_attn; a node whose ancestor walk
 *                  breaks the parent rules is never consistent
 *   accept_len     device [B] int32 (out)
 *   accept_path    device [B, T] int32 (out)
 *   next_token     device [B] int32 (out)
 *   target_argmax  device [B, T] int32 (out) or NULL: tgt[i] for every node
 *   workspace      device, >= dreams_tree_accept_workspace_size bytes (see "Workspaces" above).
 * Bit-exact: integer results only; every comparison is an fp32 comparison of the caller's logits.
 */
dreams_status_t dreams_tree_accept(int32_t batch, int32_t num_nodes, int32_t vocab, const float* target_logits,
                                   const int32_t* draft_tokens, const int32_t* parent, int32_t* accept_len,
                                   int32_t* accept_path, int32_t* next_token, int32_t* target_argmax,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace dreams_tree_accept_sampled needs (0 only when batch is 0).  DREAMS_ERR_UNSUPPORTED if
 * vocab exceeds 2^23 or if the arrival counters (one word per sequence, then 16 bytes per row: batch *
 * num_nodes rows) do not fit in DREAMS_WORKSPACE_COUNTER_BYTES - 128 (about 4000 rows).  After the counters: per row
 * 8 bytes of flags plus 40 bytes per piece of the vocabulary (pieces of 4096 entries, or of 8192 once
 * batch * num_nodes * ceil(vocab / 4096) exceeds 4096). */
dreams_status_t dreams_tree_accept_sampled_workspace_size(int32_t batch, int32_t num_nodes, int32_t vocab,
                                                          size_t* bytes);

/*
 * dreams_tree_accept_sampled -- acceptance at temperature tau > 0 (the paper reports its speedups at
 * temperature 1, Table 2): speculative sampling's accept-or-resample rule (Section 1; Section 2,
 * "Speculative decoding"), walked down the tree.  For every sequence b:
 *
 *   p_i = softmax(target_logits[b,i,:] / tau), q_i = softmax(draft_logits[b,i,:] / tau): the target's and the
 *         draft's distribution of the token that follows node i (node i's children are the draft's samples
 *         from q_i)
 *   walk: node = 0 (the root), r = p_node; the children c of node are tested in increasing index order:
 *         with x = draft_tokens[b,c], c is kept iff uniforms[b,c] * q_node(x) < r(x) (probability
 *         min(1, r(x)/q_node(x))); the walk moves to the first kept child and starts again there; after a
 *         rejection r becomes max(r - q_node, 0) / sum(max(r - q_node, 0)) (r is kept if that sum is 0)
 *   stop: at a node none of whose children is kept (a leaf included), with that node's residual r
 *   accept_len[b]  = number of kept children on the walk (the step emits accept_len + 1 tokens)
 *   accept_path[b] = node ids root .. last (accept_len + 1 entries), then -1 up to T entries
 *   next_token[b]  = the smallest x with sum_{y <= x} r(y) > uniforms[b,0] * sum_y r(y)
 *
 *   temperature    tau > 0, finite
 *   target_logits  device [B, T, V] float, finite
 *   draft_logits   device [B, T, V] float, finite
 *   draft_tokens   device [B, T] int32 (entry 0 = root token, not read); a token outside [0, V) is rejected
 *   parent         device [B, T] int32, as for dreams_tree_verify_attn; a node whose parent breaks the rules
 *                  (parent[i] outside [0, i)) is never kept
 *   uniforms       device [B, T] float in [0, 1): entry 0 draws the emitted token, entry c decides child c
 *   accept_len     device [B] int32 (out)
 *   accept_path    device [B, T] int32 (out)
 *   next_token     device [B] int32 (out)
 *   workspace      device, >= dreams_tree_accept_sampled_workspace_size bytes (see "Workspaces" above)
 * Probabilities are computed in fp64; the integer results equal those of the rule evaluated in fp64 except
 * where a uniform falls within rounding (about 1e-15 relative) of a decision threshold.
 */
dreams_status_t dreams_tree_accept_sampled(int32_t batch, int32_t num_nodes, int32_t vocab, double temperature,
                                           const float* target_logits, const float* draft_logits,
                                           const int32_t* draft_tokens, const int32_t* parent,
                                           const float* uniforms, int32_t* accept_len, int32_t* accept_path,
                                           int32_t* next_token, void* workspace, size_t workspace_bytes,
                                           hipStream_t stream);

/* Bytes of workspace dreams_tree_accept_lm_head needs (0 only when batch is 0): the 64 KiB counter region
 * (unused by this verb, kept so that one workspace serves every verb) and 8 bytes per row per tile of the
 * vocabulary (tiles of 128 entries while batch * num_nodes <= 64, else of 256).  DREAMS_ERR_UNSUPPORTED if
 * hidden is not a multiple of 256. */
dreams_status_t dreams_tree_accept_lm_head_workspace_size(int32_t batch, int32_t num_nodes, int32_t hidden,
                                                          int32_t vocab, size_t* bytes);

/*
 * dreams_tree_accept_lm_head -- dreams_tree_accept with the LM head fused in: the target logits of every tree
 * node are formed from its final hidden state and the LM head's weight (the paper, Section 2, "Speculative
 * decoding": the target's token at each position is the argmax of its logits),
 *
 *   logit[b,i,v] = sum_k hidden_states[b,i,k] * lm_weight[v,k]      (bf16 operands, fp32 accumulation)
 *
 * and the greedy rule of dreams_tree_accept is applied to them, without the logits ever being written to
 * memory.  tgt[i] is the smallest index attaining the row maximum of the logits as computed here (fp32, a
 * fixed order of accumulation); results are otherwise exactly those of dreams_tree_accept on these logits.
 *
 *   hidden         H, a multiple of 256
 *   hidden_states  device [B, T, H] bfloat16, 16-byte aligned
 *   lm_weight      device [V, H] bfloat16 (one row per vocabulary entry), 16-byte aligned
 *   draft_tokens, parent, accept_len, accept_path, next_token, target_argmax: as for dreams_tree_accept
 *   workspace      device, >= dreams_tree_accept_lm_head_workspace_size bytes (see "Workspaces" above).
 */
dreams_status_t dreams_tree_accept_lm_head(int32_t batch, int32_t num_nodes, int32_t hidden, int32_t vocab,
                                           const void* hidden_states, const void* lm_weight,
                                           const int32_t* draft_tokens, const int32_t* parent,
                                           int32_t* accept_len, int32_t* accept_path, int32_t* next_token,
                                           int32_t* target_argmax, void* workspace, size_t workspace_bytes,
                                           hipStream_t stream);

/*
 * dreams_kv_commit -- keeps the accepted path in the cache: for every layer, sequence b and KV head, and
 * k = 0 .. accept_len[b], slot kv_len_in[b] + k receives (bit for bit) the K and V rows of slot
 * kv_len_in[b] + accept_path[b,k]; then kv_len_out[b] = kv_len_in[b] + accept_len[b] + 1 (the root and the
 * accepted drafts are now committed; the bonus token's K/V is produced by the next step, where it is the
 * root).  Slots outside [kv_len_in[b], kv_len_in[b] + accept_len[b]] are not written.
 *
 *   num_layers          NL >= 1 caches; layer l starts layer_stride_elems elements after layer l-1
 *   k_cache, v_cache    device, per layer [B, Hkv, S_cap, D] of `dtype` (in place)
 *   kv_len_in           device [B] int32
 *   accept_path         device [B, path_stride] int32, as written by dreams_tree_accept
 *   accept_len          device [B] int32, clamped into [0, path_stride - 1]
 *   kv_len_out          device [B] int32 (out); must not alias kv_len_in
 * A path entry that is not a valid source (accept_path[b,k] < k, or kv_len_in[b] + accept_path[b,k] outside
 * the cache) is skipped.
 */
dreams_status_t dreams_kv_commit(int32_t num_layers, int64_t layer_stride_elems, int32_t batch,
                                 int32_t num_kv_heads, int32_t head_dim, int32_t cache_capacity,
                                 dreams_dtype_t dtype, void* k_cache, void* v_cache, const int32_t* kv_len_in,
                                 const int32_t* accept_path, const int32_t* accept_len, int32_t path_stride,
                                 int32_t* kv_len_out, hipStream_t stream);

/*
 * Paged cache.  A pool holds num_pages pages of page_size slots; per layer, k_pages and v_pages are
 * [num_pages, Hkv, page_size, D], the pages page_stride elements apart (so that one buffer may hold a page's K and V side
 * by side), each page dense.  Slot j of sequence b is row j % page_size of page page_table[b, j / page_size] (table:
 * device [B, table_width] int32).  A sequence's table need only name the pages of the slots that a call reads or writes;
 * entries past them may hold anything.  A named page outside [0, num_pages) is never accessed: attention reads another
 * page of the pool in its place (results unspecified), writes of rows leave it out.
 *   page_size   a power of two, 16 .. 32768 (DREAMS_ERR_UNSUPPORTED otherwise)
 *   table_width * page_size <= 2^30 slots
 * Offsets are 64-bit: a pool may be larger than 4 GiB.
 */

/*
 * Attention over pages.
 *   num_rows     T tree nodes (1..128) or N prompt rows per sequence, <= table_width * page_size
 *   max_kv_len   host-side upper bound on every kv_len[b], used only to plan the work split (results do not depend on it
 *                beyond rounding order).  0 means unknown: table_width * page_size - num_rows, so that a prompt without a
 *                prefix in a wide table is cut into pieces for keys that are not there (8 x 187 rows, 24 heads, a table
 *                of 32768 slots: 34 us instead of 10).  1 is the bound of no prefix: max(1, longest) is always accepted.
 *                0 <= max_kv_len <= max(1, table_width * page_size - num_rows).
 *   num_splits   pieces of the key axis, 0: the library's choice.  Any value gives the same result up to rounding order.
 *   window       0: every key is in sight.  W >= 1: a key at position p is in sight of a row at position P iff P - p < W
 *   sinks        or p < sinks (the first tokens of a sequence that stay visible; >= 0, no effect without a window)
 *   page_stride  elements from a page to the next, >= Hkv * page_size * D; 0 means just that
 * Other fields as in dreams_attn_desc_t.
 */
typedef struct {
  int32_t batch;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t num_rows;
  int32_t num_pages;
  int32_t page_size;
  int32_t table_width;
  int32_t max_kv_len;
  int32_t num_splits;
  int32_t window;
  int32_t sinks;
  dreams_dtype_t dtype;
  float scale;
  int64_t page_stride;
} dreams_paged_desc_t;

/* Bytes of workspace dreams_paged_verify_attn / dreams_paged_prompt_attn need for `desc` on the current device (0 if
 * none: then the call accepts a NULL workspace). */
dreams_status_t dreams_paged_verify_attn_workspace_size(const dreams_paged_desc_t* desc, size_t* bytes);
dreams_status_t dreams_paged_prompt_attn_workspace_size(const dreams_paged_desc_t* desc, size_t* bytes);

/*
 * dreams_paged_verify_attn -- dreams_tree_verify_attn over a paged cache, with an optional sliding window: for every
 * sequence b, query head h and tree node i, softmax attention over the prefix slots 0 .. L_b-1 and the slots L_b + n of
 * the nodes n that are i or its ancestors (the caller has written the nodes' K/V there, dreams_paged_append), of these
 * the ones in sight.  The position of prefix slot j is j, that of node n is L_b + depth(n).  T = 1 is a decode step.
 *   q            device [B, Hq, T, D]
 *   k_pages, v_pages, page_table: see "Paged cache"
 *   kv_len       device [B] int32     L_b, clamped into [0, table_width * page_size - T]
 *   parent       device [B, T] int32  as for dreams_tree_verify_attn (an entry breaking the rules ends that node's walk,
 *                                     and its depth); may be NULL if tree_mask is given and window is 0
 *   tree_mask    device [B, T, ceil(T/64)] uint64 or NULL: bit n of row i set <=> node n is visible to node i (if in
 *                                     sight; the window needs parent for the depths)
 *   out          device [B, Hq, T, D] same dtype as q;  lse: device [B, Hq, T] float or NULL
 * A row that sees nothing (a mask without a prefix in sight) gives out = 0 and lse = -inf, as does one whose scores are all
 * -inf; a score of NaN or +inf makes its row's out and lse NaN.  Values in slots that no row sees do not matter (NaN and
 * infinities included), but for the rows' own slots: their V, and that of slots which a window leaves to some of a
 * sequence's rows only, is to be finite.  Where it is not, rows that do not see it may be NaN too.  K may hold anything
 * where a row does not see it.  Arithmetic as for dreams_tree_verify_attn, but for the pieces' rows, which are merged in fp32
 * unrounded.  The workspace is dreams_paged_verify_attn_workspace_size bytes at least (fewer: DREAMS_ERR_WORKSPACE).
 */
dreams_status_t dreams_paged_verify_attn(const dreams_paged_desc_t* desc, const void* q, const void* k_pages,
                                         const void* v_pages, const int32_t* page_table, const int32_t* kv_len,
                                         const int32_t* parent, const uint64_t* tree_mask, void* out, float* lse,
                                         void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * dreams_paged_prompt_attn -- the attention of a prompt's rows (or of a piece of a prompt behind kv_len[b] cached slots)
 * over a paged cache that holds their K/V already: row i of sequence b is at position L_b + i and sees the slots
 * 0 .. L_b + i in sight.
 *   q          device [B, Hq, N, D]
 *   kv_len     device [B] int32   L_b, slots before the rows' own; clamped into [0, table_width * page_size - n_b]
 *   row_len    device [B] int32   n_b, live rows (clamped into [0, N]), or NULL: N each
 *   out, lse   as above; rows i >= n_b get out = 0 and lse = -inf (their q, and the slots from
 *              L_b + n_b on, may hold anything)
 */
dreams_status_t dreams_paged_prompt_attn(const dreams_paged_desc_t* desc, const void* q, const void* k_pages,
                                         const void* v_pages, const int32_t* page_table, const int32_t* kv_len,
                                         const int32_t* row_len, void* out, float* lse, void* workspace,
                                         size_t workspace_bytes, hipStream_t stream);

/*
 * A pool's geometry for the calls that write it or keep its tables.  layer_stride and page_stride are in elements, 0
 * means dense (page_stride Hkv * page_size * D, layer_stride num_pages * page_stride); both times the element size must be
 * multiples of 16 bytes, as must head_dim times it (<= 512 bytes).
 * dreams_pages_reserve and dreams_pages_release read only batch, num_pages, page_size and table_width.
 */
typedef struct {
  int32_t num_layers;
  int32_t batch;         /* rows of the page table */
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t num_pages;
  int32_t page_size;
  int32_t table_width;
  dreams_dtype_t dtype;
  int64_t layer_stride;
  int64_t page_stride;
} dreams_page_pool_t;

/*
 * dreams_paged_append -- new rows into their slots, bit for bit: for every layer, KV head and i < n_b, slot
 * kv_len[b] + i of sequence b receives K and V row (layer, b, head, i) of k_new and v_new.  kv_len is not changed.  Rows
 * past the table or on pages outside the pool, and sequences with kv_len[b] < 0, are left out.  k_new and v_new are no rows
 * that the call writes.
 *   k_new, v_new   device, num_rows rows a sequence; strides[4] (host): elements between layers, sequences, KV heads and
 *                  rows (so [NL, B, Hkv, N, D] and [NL, B, N, Hkv, D] both serve), multiples of 16 bytes; rows dense
 *   row_len        device [B] int32 n_b (at most num_rows), or NULL: num_rows each
 */
dreams_status_t dreams_paged_append(const dreams_page_pool_t* pool, const void* k_new, const void* v_new,
                                    int32_t num_rows, const int64_t* strides, const int32_t* page_table,
                                    const int32_t* kv_len, const int32_t* row_len, void* k_pages, void* v_pages,
                                    hipStream_t stream);

/* dreams_paged_kv_commit -- dreams_kv_commit over pages: slot kv_len_in[b] + k receives slot kv_len_in[b] +
 * accept_path[b,k] for k = 0 .. accept_len[b], in every layer and KV head; kv_len_out[b] = kv_len_in[b] + accept_len[b] + 1.
 * Arguments and skipped entries as there (an entry whose slot the table does not cover is skipped too). */
dreams_status_t dreams_paged_kv_commit(const dreams_page_pool_t* pool, void* k_pages, void* v_pages,
                                       const int32_t* page_table, const int32_t* kv_len_in, const int32_t* accept_path,
                                       const int32_t* accept_len, int32_t path_stride, int32_t* kv_len_out,
                                       hipStream_t stream);

/*
 * Page tables.  page_count[b] is the number of pages that sequence b holds, the first entries of its row; refcount[p] the
 * number of sequences that hold page p, 0 marking it free (device int32 [B] and [num_pages]; a new pool is all zeros).
 * Pages are taken lowest number first and the calls read nothing but the state before them, so that the same calls
 * always give the same tables.  Limits: num_pages <= DREAMS_PAGES_MAX, batch and list lengths <=
 * DREAMS_PAGES_MAX_SEQUENCES, batch * table_width < 2^31 (DREAMS_ERR_UNSUPPORTED otherwise).  Calls on one pool are
 * ordered by the caller (one stream, or synchronised ones).
 *
 * Pages are shared by forks only, and only pages filled to the end are: as long as kv_len[b] is only raised (and lowered by
 * dreams_pages_release), the slots from kv_len[b] on are the sequence's own.
 */
#define DREAMS_PAGES_MAX 524288
#define DREAMS_PAGES_MAX_SEQUENCES 4096

/* dreams_pages_reserve -- room: every sequence b, in order, that holds fewer than ceil(want_len[b] / page_size) pages takes
 * as many as it lacks, if that many are free by then (all or none) and its row is wide enough.  granted[b] (out): 1 if the
 * sequence holds want_len[b] slots, else 0 and nothing of it changes.  want_len[b] <= 0 asks for nothing. */
dreams_status_t dreams_pages_reserve(const dreams_page_pool_t* pool, int32_t* page_table, int32_t* page_count,
                                     int32_t* refcount, const int32_t* want_len, int32_t* granted, hipStream_t stream);

/* dreams_pages_fork -- copies of sequences: for i < count, sequence dst[i] becomes a copy of sequence src[i], sharing its
 * pages filled to the end and taking a page of its own (lowest free, pairs in order) for the copied rows of a partly filled
 * one; kv_len[dst[i]] = kv_len[src[i]].  granted[i] (out): 1, or 0 and nothing changes: dst[i] holds pages or was named
 * before in dst, dst[i] = src[i], an index is outside the table, src[i]'s pages do not cover its kv_len, or no page is free.
 * Sources are read as they are before the call.  A table of no sequences (batch 0) enqueues nothing: granted is not
 * written. */
dreams_status_t dreams_pages_fork(const dreams_page_pool_t* pool, void* k_pages, void* v_pages, int32_t* page_table,
                                  int32_t* page_count, int32_t* kv_len, int32_t* refcount, int32_t count,
                                  const int32_t* src, const int32_t* dst, int32_t* granted, hipStream_t stream);

/* dreams_pages_release -- sequences seqs[0 .. count-1] give up their pages: all of them (trim 0; kv_len becomes 0), or those
 * past the ones that kv_len slots need (trim 1; kv_len stays).  Their entries become -1.  An index outside the table is
 * skipped, one named again too. */
dreams_status_t dreams_pages_release(const dreams_page_pool_t* pool, int32_t* page_table, int32_t* page_count,
                                     int32_t* kv_len, int32_t* refcount, int32_t count, const int32_t* seqs, int32_t trim,
                                     hipStream_t stream);

/*
 * Rotary positions.  A head's first rotary_dim columns are rotary_dim / 2 pairs, of which pair i of a row at position p is
 * turned by the angle p * frequencies[i] (radians):
 *     (x, y)  becomes  (amplitude * (x cos - y sin), amplitude * (y cos + x sin))
 * The other columns stay as they are.  Cosines and sines, times the amplitude, are computed in 64 bits and rounded once to 32;
 * two products and their sum in 32 bits follow (one of the products unrounded), and the result is rounded
 * once to the type of the output.
 *   rotary_dim    R, a multiple of 16, 16 .. head_dim
 *   interleaved   0: pair i is columns i and i + R/2;  1: columns 2i and 2i + 1
 *   frequencies   device [R/2] double (dreams_rope_frequencies, or any others), 8-byte aligned
 *   positions     device [B, N] int32 or NULL: every row's position (a negative one turns back)
 *   parent        device [B, N] int32 or NULL: rows are tree nodes (N <= 128), as for dreams_tree_verify_attn
 *                 Without positions, row i of sequence b is at kv_len[b] + depth(i) (parent) or kv_len[b] + i.
 *   amplitude     finite factor of the rotated columns (stretched contexts; normally 1)
 */
typedef struct {
  int32_t rotary_dim;
  int32_t interleaved;
  const double* frequencies;
  const int32_t* positions;
  const int32_t* parent;
  float amplitude;
} dreams_rope_t;

/* Scalings of the frequencies f_i = base^(-2i/R) for contexts beyond the trained one:
 *   DREAMS_ROPE_PLAIN    none
 *   DREAMS_ROPE_LINEAR   f_i / factor
 *   DREAMS_ROPE_PARTS    by parts: f_i (g + (1 - g) / factor), where g rises from 0 to 1 as the turns that the pair makes
 *                        within the trained context, trained_len * f_i / (2 pi), go from `low` to `high` */
typedef enum { DREAMS_ROPE_PLAIN = 0, DREAMS_ROPE_LINEAR = 1, DREAMS_ROPE_PARTS = 2 } dreams_rope_scaling_t;

/* dreams_rope_frequencies -- fills frequencies (HOST memory, rotary_dim / 2 doubles; rotary_dim even and >= 2).  base > 0 and
 * factor > 0 finite; trained_len > 0 and 0 <= low < high finite (read for DREAMS_ROPE_PARTS only). */
dreams_status_t dreams_rope_frequencies(int32_t rotary_dim, double base, dreams_rope_scaling_t scaling, double factor,
                                        double trained_len, double low, double high, double* frequencies);

/*
 * dreams_rope -- rows rotated by their positions: out[b,h,i,:] = rotation of x[b,h,i,:] for every sequence b < batch, head h
 * < num_heads and row i < num_rows.
 *   head_dim      D, a multiple of 8, <= 512; dtype DREAMS_BF16 or DREAMS_F32
 *   x, out        device; x_strides[3], out_strides[3] (host): elements between sequences, heads and rows, multiples of 16
 *                 bytes (so [B, H, N, D] and [B, N, H, D] both serve); rows dense.  out = x with the same strides works in
 *                 place; else they must not overlap.
 *   kv_len        device [B] int32, the position of row 0 (of the root); may be NULL where rope->positions is given
 */
dreams_status_t dreams_rope(const dreams_rope_t* rope, int32_t batch, int32_t num_heads, int32_t num_rows, int32_t head_dim,
                            dreams_dtype_t dtype, const void* x, const int64_t* x_strides, const int32_t* kv_len,
                            void* out, const int64_t* out_strides, hipStream_t stream);

/*
 * The queries that go with new rows.  q: device [B, num_q_heads, N, D] of the new rows' type at strides[3] (elements between
 * sequences, heads and rows, multiples of 16 bytes, rows dense); out: device, dense [B, num_q_heads, N, D], the layout that the
 * attention calls take; must not overlap q.  Rows i >= row_len[b] of out become 0.
 */
typedef struct {
  const void* q;
  void* out;
  int32_t num_q_heads;
  int64_t strides[3];
} dreams_rope_queries_t;

/* dreams_paged_append_rope -- dreams_paged_append with k_new rotated on its way into the pages, and, where queries is not
 * NULL (num_layers 1), the rows' queries rotated in the same launch.  Other arguments as there. */
dreams_status_t dreams_paged_append_rope(const dreams_page_pool_t* pool, const dreams_rope_t* rope,
                                         const dreams_rope_queries_t* queries, const void* k_new, const void* v_new,
                                         int32_t num_rows, const int64_t* strides, const int32_t* page_table,
                                         const int32_t* kv_len, const int32_t* row_len, void* k_pages, void* v_pages,
                                         hipStream_t stream);

/*
 * Pages of 8 bits.  Pages as above in the codes of e4m3 (OCP: 1 sign, 4 exponent and 3 fraction bits, bias 7, largest 448, no
 * infinity, 0x7f and 0xff NaN), pool dtype DREAMS_E4M3, and for each block of 16 slots of a head (slots 16 j .. 16 j + 15 of
 * its page) one scale byte s of K and one of V, in e8m0: a row's values are its codes times 2^(s - 127).  head_dim is a
 * multiple of 16, <= 512 (attention: 64 or 128).
 * A block takes the least scale (s >= 1) at which the largest finite magnitude in it is at most 448 times it.  Powers of two
 * lose nothing here: codes have an exponent of their own, and rows that move to a larger scale change only where they
 * fall below the codes' normal range (2^-14 of the block's largest value and less).  The bytes that these calls write are 1 ..
 * 247; 0 and 255 give unspecified values.  An infinity or NaN becomes NaN; a magnitude from 1.9375 * 2^127 on rounds to 2^128,
 * an infinity as it is read.
 *   k, v           device uint8 [NL][num_pages, Hkv, page_size / 16]
 *   layer_stride, page_stride   bytes, 0 means dense (page_stride Hkv * page_size / 16)
 */
typedef struct {
  uint8_t* k;
  uint8_t* v;
  int64_t layer_stride;
  int64_t page_stride;
} dreams_page_scales_t;

/*
 * dreams_paged_append_e4m3 -- dreams_paged_append (rope NULL) or dreams_paged_append_rope into pages of 8 bits: every
 * block that new rows go into takes the larger of its rows' scale and, where it holds slots before kv_len[b], the one it has;
 * their codes are then moved to it.  A block's later slots are dead: their values may change.
 *   new_dtype   type of k_new, v_new and the queries: DREAMS_BF16 or DREAMS_F32 (strides in its elements)
 *   queries     needs rope
 */
dreams_status_t dreams_paged_append_e4m3(const dreams_page_pool_t* pool, const dreams_page_scales_t* scales,
                                         const dreams_rope_t* rope, const dreams_rope_queries_t* queries,
                                         dreams_dtype_t new_dtype, const void* k_new, const void* v_new, int32_t num_rows,
                                         const int64_t* strides, const int32_t* page_table, const int32_t* kv_len,
                                         const int32_t* row_len, void* k_pages, void* v_pages, hipStream_t stream);

/* dreams_paged_kv_commit_e4m3 -- dreams_paged_kv_commit over pages of 8 bits.  A block that rows move into takes the largest
 * scale of the rows it keeps (slots before kv_len_in[b], path entries that stay where they are or are skipped) and of those
 * that come, and their codes are moved to it.  A block's slots past the path are dead: their values may change. */
dreams_status_t dreams_paged_kv_commit_e4m3(const dreams_page_pool_t* pool, const dreams_page_scales_t* scales, void* k_pages,
                                            void* v_pages, const int32_t* page_table, const int32_t* kv_len_in,
                                            const int32_t* accept_path, const int32_t* accept_len, int32_t path_stride,
                                            int32_t* kv_len_out, hipStream_t stream);

/* dreams_paged_read_e4m3 -- the cached rows as values: k_out, v_out device bfloat16 [NL, B, Hkv, num_slots, D] (16-byte
 * aligned): slot j < kv_len[b] of sequence b, exactly; 0 from kv_len[b] on, past the table, and for a page outside the pool.
 * (Values below bfloat16's normal range may be flushed.)  What reads a cache as one slab (the visual-token statistics, a pool
 * of another type) takes it from there. */
dreams_status_t dreams_paged_read_e4m3(const dreams_page_pool_t* pool, const dreams_page_scales_t* scales,
                                       const void* k_pages, const void* v_pages, const int32_t* page_table,
                                       const int32_t* kv_len, int32_t num_slots, void* k_out, void* v_out,
                                       hipStream_t stream);

/*
 * dreams_paged_verify_attn_e4m3, dreams_paged_prompt_attn_e4m3 -- dreams_paged_verify_attn and dreams_paged_prompt_attn over
 * pages of 8 bits: attention of bf16 queries over the values that the codes stand for (exact in bf16; those below its normal
 * range may be flushed), with the same arithmetic (scores and sums in fp32, the probabilities rounded to bf16 once before the
 * value product), masks, windows, and rules for slots out of sight.
 *   desc->dtype        type of q and out, DREAMS_BF16 (DREAMS_F32: DREAMS_ERR_UNSUPPORTED)
 *   desc->page_stride  codes (bytes) from a page to the next
 *   scales             of this layer (layer_stride is not read)
 * The workspace is of the matching size query; splits may differ from those over bf16 pages.
 */
dreams_status_t dreams_paged_verify_attn_e4m3_workspace_size(const dreams_paged_desc_t* desc, size_t* bytes);
dreams_status_t dreams_paged_prompt_attn_e4m3_workspace_size(const dreams_paged_desc_t* desc, size_t* bytes);
dreams_status_t dreams_paged_verify_attn_e4m3(const dreams_paged_desc_t* desc, const void* q, const void* k_pages,
                                              const void* v_pages, const dreams_page_scales_t* scales,
                                              const int32_t* page_table, const int32_t* kv_len, const int32_t* parent,
                                              const uint64_t* tree_mask, void* out, float* lse, void* workspace,
                                              size_t workspace_bytes, hipStream_t stream);
dreams_status_t dreams_paged_prompt_attn_e4m3(const dreams_paged_desc_t* desc, const void* q, const void* k_pages,
                                              const void* v_pages, const dreams_page_scales_t* scales,
                                              const int32_t* page_table, const int32_t* kv_len, const int32_t* row_len,
                                              void* out, float* lse, void* workspace, size_t workspace_bytes,
                                              hipStream_t stream);

/* dreams_pages_fork_e4m3 -- dreams_pages_fork over pages of 8 bits: the copied rows' scales go with them. */
dreams_status_t dreams_pages_fork_e4m3(const dreams_page_pool_t* pool, const dreams_page_scales_t* scales, void* k_pages,
                                       void* v_pages, int32_t* page_table, int32_t* page_count, int32_t* kv_len,
                                       int32_t* refcount, int32_t count, const int32_t* src, const int32_t* dst,
                                       int32_t* granted, hipStream_t stream);

/* Static description of a status code. */
const char* dreams_status_string(dreams_status_t status);

/* Message describing the calling thread's most recent failure ("" if none). Valid until its next call. */
const char* dreams_last_error_message(void);

/* Host-side check of a parent array (host memory): DREAMS_OK iff parent[0] == -1 and 0 <= parent[i] < i. */
dreams_status_t dreams_check_tree_host(const int32_t* parent, int32_t num_nodes);

/*
 * Measurement helper, not part of the method: reads `bytes` bytes at `src` once, with non-temporal 16-byte loads,
 * one contiguous chunk per workgroup over every compute unit, and writes one word per wave to `sink`
 * (DREAMS_STREAM_READ_SINK_WORDS words) so
 * that the loads cannot be elided.  Timed around, it gives the device's plain read bandwidth, the reference for
 * the share of the measured peak that the kernels above reach.
 *   src    device, 16-byte aligned; bytes a multiple of 16 (DREAMS_ERR_INVALID_ARG otherwise)
 *   sink   device, DREAMS_STREAM_READ_SINK_WORDS uint32 words (contents unspecified afterwards)
 */
#define DREAMS_STREAM_READ_SINK_WORDS 2048
dreams_status_t dreams_stream_read(const void* src, size_t bytes, uint32_t* sink, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DREAMS_H */
