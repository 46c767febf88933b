/*
 * fkv - budgeted KV-cache eviction and decode attention for one B200 (sm_100a).
 *
 * C ABI of the library built from paper_2602_03203_b200/csrc.  The calls are
 * the paper's statement of the problem (Section 3.1): a cache with budget B
 * that grows by appended (k, v) pairs, is pruned back to B by a learned
 * per-(layer, KV-head) scorer, and is attended over by the decode queries:
 *
 *     fkv_init_cache(shapes, budget)  fkv_append(k, v)  fkv_evict(layer)  fkv_decode_attn(q)
 *
 * Conventions
 *   - Every function returns FKV_OK (0) or a negative fkv_status.  Nothing
 *     throws, nothing is printed.
 *   - "dev" pointers are CUDA device pointers, "host" pointers are host
 *     pointers; a pointer documented "host or dev" may be either.
 *   - All device work is enqueued on the caller's stream (a cudaStream_t passed
 *     as void*); calls return without synchronising unless they say "syncs".
 *     Calls on one cache must be issued on ONE stream, or be ordered by the
 *     caller; two calls on one cache that overlap on the GPU race.
 *   - Host threads: a handle keeps a host-side mirror of the lengths and is not
 *     thread-safe; use one host thread per handle at a time.  The first launch
 *     of each kernel in a process sets its attributes without a lock, so make
 *     the first calls on a device from one thread.
 *   - The library never allocates device memory for a cache.  The caller owns
 *     one device workspace (fkv_workspace_bytes) and keeps it alive until
 *     fkv_destroy; per-call tensors (k, v, q, out, ...) are borrowed until the
 *     enqueued work has run.
 *   - Device-side failures (page pool exhausted, capacity exceeded, a bounded
 *     wait that ran out) do not fault: the kernel skips the work and sets a
 *     bit in a status word that fkv_device_status reads.
 *
 * Terms: one "segment" is the cache of one (sequence, layer, KV head); it
 * holds n "pairs" (slots 0..n-1 in position order).  D = head_dim, g =
 * group_size (query heads per KV head), F = 6g attention features per pair
 * (Appendix B.1), H = scorer_hidden.  bf16 tensors are passed as raw 16-bit
 * patterns.
 */
#ifndef FKV_H
#define FKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  FKV_OK = 0,
  FKV_ERR_INVALID_ARG = -1,
  FKV_ERR_WORKSPACE_TOO_SMALL = -2,
  FKV_ERR_CAPACITY = -3,   /* a sequence would exceed max_tokens_per_head */
  FKV_ERR_CUDA = -4,       /* a CUDA call failed; see fkv_last_cuda_error */
  FKV_ERR_NOT_READY = -5,  /* e.g. evict before the scorers are loaded */
  FKV_ERR_DEVICE = -6      /* fkv_device_status found error bits */
} fkv_status;

/* Bits of the device status word (fkv_device_status). */
#define FKV_DEV_POOL_EXHAUSTED 1u /* no free page: the step that needed it was skipped */
#define FKV_DEV_CAPACITY 2u       /* append past max_tokens_per_head was skipped */
#define FKV_DEV_WAIT_TIMEOUT 4u   /* a bounded wait in a kernel ran out */
#define FKV_DEV_BAD_INDEX 8u      /* fkv_compact was given an index outside the segment; a replayed chunk call met a shorter one;
                                   a tree's parents or path are out of order */

/* Scorer activation sigma.  The paper does not name it (Appendix B.1); ReLU is the default. */
enum { FKV_ACT_RELU = 0, FKV_ACT_SILU = 1, FKV_ACT_GELU_TANH = 2, FKV_ACT_SIGMOID = 3 };

#define FKV_ALL_LAYERS (-1)

typedef struct fkv_cache fkv_cache; /* opaque, host side */

typedef struct {
  int32_t num_layers;
  int32_t num_kv_heads;
  int32_t group_size;          /* g, 1..8 */
  int32_t head_dim;            /* D, 64 or 128 */
  int32_t max_batch;           /* sequences, at most 256 (the efficiency table of Section 4.3 runs up to 96) */
  int32_t page_size;           /* pairs per page; must be 16 */
  int32_t scorer_hidden;       /* H; must be 16 (Section 4.1) */
  int32_t activation;          /* FKV_ACT_* */
  int32_t budget;              /* B for every sequence (fkv_set_budget overrides per sequence) */
  int32_t recent_keep;         /* R: most recent pairs never evicted (the paper's L; 0 = plain top-B) */
  int32_t max_tokens_per_head; /* capacity of one segment, n <= this */
  int32_t num_pages;           /* pages in the pool; 0 = enough for every segment at capacity
                                  plus the transient copies of an all-layer eviction */
  int32_t feature_window;      /* W: decode queries kept on record per (layer, sequence) for the attention
                                  features of Appendix B.1 (a multiple of 8, at most 256;
                                  the paper's update length L, e.g. 256); 0 = the library does not
                                  maintain the features */
} fkv_config;

/* Bytes of device workspace fkv_init_cache needs for this config (39 MB of them, 20 with head_dim 64, for the partial results
 * of fkv_chunk_attn, whatever the shape of the cache). */
int fkv_workspace_bytes(const fkv_config *cfg, size_t *bytes);

/*
 * init_cache(shapes, budget) - Section 3.1.  Carves the caller's device
 * workspace (dev, 256-byte aligned, `bytes` long) into the page pool, page
 * tables, lengths, scorer blocks and scratch, and clears it on `stream`.
 * The handle is host memory owned by the library until fkv_destroy.
 */
int fkv_init_cache(const fkv_config *cfg, void *dev_workspace, size_t bytes, void *stream, fkv_cache **out);
int fkv_destroy(fkv_cache *c);

/* Empty every segment and return all pages to the pool (scorers and budgets stay). */
int fkv_reset(fkv_cache *c, void *stream);

/*
 * Scorer of one (layer, KV head) - Appendix B.1:
 *   phi = sigma(x W1 + b1) W2 + b2,  x = Concat(k, v, a).
 * W1: host, [(2D+F)][H] row-major fp32, rows ordered k | v | a; b1, W2: host
 * [H].  The paper states no precision for the weights; they are taken as
 * fp32.  The 2D rows of W1 that multiply k and v are stored as TWO bf16 values
 * per weight, the rounding (to nearest even) of the weight and the rounding of
 * the remainder, and both are multiplied with the bf16 channels on the tensor
 * cores with fp32 accumulation: a weight enters with about 2^-17 relative
 * error instead of bf16's 2^-9.  The F feature rows, b1, W2, b2 stay fp32.
 * Copies to the device on `stream` from a staging buffer the handle owns
 * (syncs).
 */
int fkv_load_scorer(fkv_cache *c, int layer, int kv_head, const float *W1, const float *b1, const float *W2, float b2,
                    void *stream);

/*
 * Per-sequence budget B - Section 3.1 states the problem with one budget B per cache; the batched
 * configurations give every sequence its own (B = half its context), so the budget is a property of
 * the sequence.  Host value; takes effect for later fkv_evict calls.
 */
int fkv_set_budget(fkv_cache *c, int seq, int32_t budget, void *stream);

/*
 * Bulk-load one EMPTY (layer, sequence): n pairs per KV head - the cache as the prefill phase leaves
 * it (Section 3.1 starts from a cache that already holds the prompt; the one-shot compression mode of
 * Section 4.4 evicts right after this call).  The paper has no counterpart for the call itself.
 * k, v: dev [Hkv][n][D] bf16; feat: dev [Hkv][n][F] fp32 or NULL (zeros);
 * pos: dev [n] int32 (strictly increasing token positions) or NULL (0..n-1).
 */
int fkv_prefill(fkv_cache *c, int layer, int seq, const void *k, const void *v, const float *feat, const int32_t *pos,
                int32_t n, void *stream);

/*
 * append(k, v) - Section 3.1: one new pair per sequence and KV head of `layer`.
 * k, v: dev [max_batch][Hkv][D] bf16; pos: dev [max_batch] int32 token
 * positions, or NULL: the position after the last stored one (0 for an empty
 * segment).  The feature row of the new pair is zero.  seq_mask: host bit
 * array of the sequences that take part, (max_batch + 63) / 64 words, bit
 * s % 64 of word s / 64; NULL = all.  It is read before the call returns.
 */
int fkv_append(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const uint64_t *seq_mask,
               void *stream);

/*
 * Overwrite the attention features a_n (Appendix B.1: six per query head and pair) of one (layer,
 * sequence) with values computed elsewhere: feat dev [Hkv][n][F] fp32, n = current length.  For
 * callers that maintain the features themselves (feature_window = 0) and for checks; the paper has no
 * counterpart for the call itself.
 */
int fkv_set_features(fkv_cache *c, int layer, int seq, const float *feat, void *stream);

/*
 * evict(layer) - Section 3.1 with the deterministic Top-K action: for every
 * segment of `layer` (or of all layers, FKV_ALL_LAYERS) with n > B, score the
 * pairs, keep the R most recent and the B - R best-scoring of the others
 * (higher score first, then lower slot; -0 = +0, NaN lowest), and compact K, V,
 * features and positions of the kept pairs, in position order, into fresh
 * pages.  Afterwards n = B.  Segments with n <= B are left untouched.
 */
int fkv_evict(fkv_cache *c, int layer, void *stream);

/*
 * evict(layer) with the paper's SAMPLED action - Section 3.1, second equation,
 * and Appendix B.2: D = Multinomial_E(Softmax(Top_2E(-Phi))), s' = s \ D.  For
 * every segment with n > B, E = n - B pairs are evicted: the candidates are
 * the 2E competing pairs with the lowest scores (ties: the higher slot ranks
 * lower; all competing pairs if there are fewer than 2E), and E of them are
 * drawn without replacement with probabilities softmax(-score).  The draws use
 * the CALLER'S randomness: noise holds standard Gumbel values g = -log(-log u),
 * u uniform in (0, 1); the candidate of rank j in slot order uses g_j, and the
 * E candidates with the largest (-score + g_j), compared in fp32, are evicted
 * (Gumbel-top-k, which is sampling without replacement from the softmax; ties:
 * the higher slot is evicted).  Everything else is as in fkv_evict.  With all
 * g = 0 this is fkv_evict.
 *
 * noise: dev fp32 [layers of the call][max_batch][Hkv][noise_stride] (one
 * layer, or all layers in order for FKV_ALL_LAYERS); noise_stride must be at
 * least min(2E, n - R) for every segment that is evicted, else
 * FKV_ERR_INVALID_ARG.  The library draws no random numbers itself.
 */
int fkv_evict_sampled(fkv_cache *c, int layer, const float *noise, int32_t noise_stride, void *stream);

/*
 * evict(layer) with a BASELINE score in place of the learned scorer - Appendix E.2.  The score of a
 * pair is one column of its attention features, averaged over the g query heads of the KV head
 * (summed in head order, divided by g, fp32): column FKV_FEATURE_CUM_SUM is H2O (cumulative
 * attention), FKV_FEATURE_WINDOW8 is SnapKV as the paper uses it (attention of the final 8 tokens).
 * Selection, compaction and (with a feature window) the feature refresh are those of fkv_evict; no
 * scorer needs to be loaded.
 */
#define FKV_FEATURE_WINDOW8 0
#define FKV_FEATURE_WINDOW16 1
#define FKV_FEATURE_WINDOW32 2
#define FKV_FEATURE_WINDOW_CHUNK 3
#define FKV_FEATURE_CUM_SUM 4
#define FKV_FEATURE_CUM_DECAY 5
int fkv_evict_by_feature(fkv_cache *c, int layer, int32_t column, void *stream);

/*
 * evict(layer) with the R-KV baseline score - Appendix E.2: "R-KV also takes into account the redundancy among
 * tokens": the window attention score and a token-to-token similarity are weighed 0.1 and 0.9.  The paper gives
 * the weights and no formula; this library's reading:
 *     score_i = lambda_attn * a_i - lambda_sim * s_i
 *     a_i = the SnapKV score above (feature FKV_FEATURE_WINDOW8 averaged over the g query heads),
 *     s_i = the largest cosine between the stored key k_i and the key of ANOTHER pair of the same segment
 *           (0 if either key is the zero vector, or the segment has one pair),
 * so a pair with a near-duplicate elsewhere in the cache is evicted before an equally attended unique one.
 * No normalisation of either term.  Cost: the n x n products of a segment's keys, 2 n^2 D flops, on the tensor
 * cores.  Features must be finite.  Everything else is as in fkv_evict_by_feature.  FKV_RKV_LAMBDA_* are the
 * paper's weights.  fkv_score_rkv is the score alone (layout as fkv_score).
 * Errors beyond those of fkv_evict_by_feature: FKV_ERR_CUDA if the driver's tensor-map encoder cannot be reached or
 * refuses the page pool's geometry, or if the device cannot place clusters of two thread blocks (the contraction
 * runs on pairs of SMs); fkv_last_cuda_error has the text.  No pair is evicted or moved in that case.
 */
#define FKV_RKV_LAMBDA_ATTN 0.1f
#define FKV_RKV_LAMBDA_SIM 0.9f
int fkv_evict_rkv(fkv_cache *c, int layer, float lambda_attn, float lambda_sim, void *stream);
int fkv_score_rkv(fkv_cache *c, int layer, float lambda_attn, float lambda_sim, float *scores_out, void *stream);

/*
 * decode_attn(q) - Appendix A: out[s][h] = sum_i softmax_i(scale <q[s][h], k_i>) v_i
 * over all retained pairs i of the KV head that query head h belongs to
 * (h / g).  q, out: dev [max_batch][Hkv*g][D] bf16.  scale 0 means 1/sqrt(D).
 * Sequences with n = 0 get zeros.
 */
int fkv_decode_attn(fkv_cache *c, int layer, const void *q, void *out, float scale, void *stream);

/*
 * append(k, v) followed by decode_attn(q) on `layer`, as ONE kernel launch
 * (Section 3.1 + Appendix A): the new pair of every participating sequence is
 * stored at slot n and attended together with the n retained pairs.  Arguments
 * as in fkv_append and fkv_decode_attn; the result equals the two calls made
 * one after the other.
 */
int fkv_append_decode_attn(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos,
                           const uint64_t *seq_mask, const void *q, void *out, float scale, void *stream);

/*
 * One decode token through every layer, in layer order: for l = 0 .. L-1,
 * fkv_append_decode_attn(k[l], v[l], q[l]) -> out[l].  k, v: dev
 * [L][max_batch][Hkv][D] bf16; q, out: dev [L][max_batch][Hkv*g][D] bf16; pos:
 * dev [max_batch] or NULL (as fkv_append).  One launch per layer, issued from
 * native code.  Every layer's k, v and q must be complete when the call is
 * enqueued: the layers do not depend on one another here, so the launches of
 * layers 1 .. L-1 are allowed to run alongside the launch before them
 * (programmatic dependent launch), and out[l] is complete only when the whole
 * step is (the next work on the stream is ordered after all of it).  For
 * engines that have all layers' tensors at hand, and for benchmarks of the
 * attention side alone.
 *
 * Stream capture: fkv_append_decode_attn and fkv_decode_step only enqueue
 * kernels, so they may be recorded into a CUDA graph.  Every replay appends one
 * more pair per sequence from the recorded k / v / q buffers: the kernel reads
 * the lengths on the device, divides a segment's pages over the recorded number
 * of splits whatever its length has become, and skips an append past
 * max_tokens_per_head (FKV_DEV_CAPACITY).  The host's copy of the lengths does
 * not see replays: call fkv_sync_lengths after the last replay and before any
 * other call of this library.
 */
int fkv_decode_step(fkv_cache *c, const void *k, const void *v, const int32_t *pos, const void *q, void *out,
                    float scale, void *stream);

/*
 * ---- sliding windows and sinks ----
 * fkv_decode_attn / fkv_append_decode_attn of a layer whose queries see only part of the retained set: a query of
 * position p sees the pairs of positions (p - window, p] and those of positions below `sinks` (the first tokens, that
 * stay visible).  Positions are the stored ones, so a window means the same before and after an eviction.  window >= 1,
 * sinks >= 0, and k, v, q and out 16-byte aligned (else FKV_ERR_INVALID_ARG).  The rest is as in the calls without a
 * window, but that the query is NOT put on record for the attention features (those describe attention over the whole
 * retained set).  A windowed layer that wants features while it decodes takes its tokens as chunks of one: fkv_append_chunk_attn,
 * which gives the log-sum-exp, and fkv_chunk_features.
 *
 * Positions must not be negative and must grow from pair to pair of a segment, and k and v must be finite where some of the
 * queries of a call see a pair and others do not.
 *
 * fkv_decode_attn_window: q_pos dev [max_batch] int32 positions of the queries (pairs of later positions are not seen), or
 * NULL: the position of the last pair.  A query that sees no pair gets zeros.  fkv_append_decode_attn_window: the query's
 * position is the new pair's; a sequence outside seq_mask attends from its last pair.
 */
int fkv_decode_attn_window(fkv_cache *c, int layer, const void *q, const int32_t *q_pos, int32_t window, int32_t sinks,
                           void *out, float scale, void *stream);
int fkv_append_decode_attn_window(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos,
                                  const uint64_t *seq_mask, const void *q, int32_t window, int32_t sinks, void *out,
                                  float scale, void *stream);

/*
 * ---- chunks of new tokens (a prompt in pieces, the draft tokens of a speculative decoder) ----
 *
 * chunk_lens: host [max_batch], the number of tokens of every sequence in this call (0: it takes no part); at most 2^24 in
 * all.  Tensors over tokens are packed: the tokens of sequence 0, then those of sequence 1, ...; nothing is read or
 * written behind the last one.  k, v: dev [tokens][Hkv][D] bf16; q, out: dev [tokens][Hkv*g][D] bf16; all 16-byte
 * aligned (FKV_ERR_INVALID_ARG otherwise).  Host arrays are read before the call returns.
 *
 * fkv_append_chunk: stores the chunk behind the pairs that stay.  keep_lens: host [max_batch], the number of pairs that
 * stay of every sequence, at most its length (the pairs behind are dropped and their pages returned: rejected drafts; with
 * chunk_lens all 0 the call only rolls back, and k, v may be NULL), or NULL: all.  pos: dev [tokens] int32, or NULL: the
 * positions after the last pair that stays (from 0 for an empty segment).  The feature rows of the new pairs are zero.
 * Decode queries on record (feature_window) whose tokens are dropped leave the record; a record that has wrapped starts
 * over then.  FKV_ERR_CAPACITY if a sequence would exceed max_tokens_per_head.  Pages that the call returns serve the growth
 * of its other sequences; if these and the free ones are too few, the whole call, roll-backs included, does nothing
 * (FKV_DEV_POOL_EXHAUSTED; what fkv_append_chunk_attn writes to out and lse_out is then of no meaning).
 *
 * fkv_chunk_attn: attention of a chunk's queries, the chunk's pairs being the last chunk_lens[s] pairs of their segments:
 *     out[j] = sum_i softmax_i(scale <q_j, k_i>) v_i,   lse_out[j] = ln sum_i exp(scale <q_j, k_i>),
 * over the pairs i up to query j's own and, with window > 0, inside its window or among the sinks (as above; window = 0:
 * every pair).  lse_out: dev [tokens][Hkv*g] fp32 or NULL.  scale 0 means 1/sqrt(D); one outside [2^-100, 2^100] is
 * FKV_ERR_INVALID_ARG, as is a chunk longer than its segment.  Errors as fkv_evict_rkv for the tensor maps.
 * P is rounded to bf16 for the product with V (as V is); everything else is fp32.
 *
 * fkv_append_chunk_attn: the two calls in one.
 *
 * Stream capture: all three only enqueue kernels.  A replayed fkv_append_chunk appends once more from the recorded buffers
 * (with keep_lens: behind the same number of pairs again); the device's lengths count, a sequence that would pass its
 * capacity (FKV_DEV_CAPACITY) or is shorter than keep_lens or its chunk (FKV_DEV_BAD_INDEX) is skipped.  Call
 * fkv_sync_lengths after the last replay.  The calls of one cache share its workspace: graphs that hold them must not run
 * at the same time.
 */
int fkv_append_chunk(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const int32_t *keep_lens,
                     const int32_t *chunk_lens, void *stream);
int fkv_chunk_attn(fkv_cache *c, int layer, const void *q, const int32_t *chunk_lens, int32_t window, int32_t sinks,
                   float scale, void *out, float *lse_out, void *stream);
int fkv_append_chunk_attn(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos,
                          const int32_t *keep_lens, const int32_t *chunk_lens, const void *q, int32_t window,
                          int32_t sinks, float scale, void *out, float *lse_out, void *stream);

/*
 * The attention features of Appendix B.1 from the queries of a chunk, so that fkv_evict and fkv_evict_by_feature
 * (FKV_FEATURE_CUM_SUM: accumulated attention) can follow a prompt.  The chunk's pairs are the last chunk_lens[s] pairs of
 * their segments; q, window, sinks and scale are those of fkv_chunk_attn, lse what it wrote (dev [tokens][Hkv*g]).  With
 * P_ji = exp(scale <q_j, k_i> - lse_j) for the pairs that query j sees and 0 for the others, the features of EVERY pair of
 * the sequences with tokens become, per query head, the means of P over the chunk's last 8 / 16 / 32 queries (fewer queries
 * still divide by 8 / 16 / 32) and over the whole chunk, previous sum + the latter, 0.9 * previous decayed sum + the latter:
 * one chunk of the recurrence described at fkv_update_features.  A chunk counts as one whatever its length: the sums
 * grow by its MEAN, so a prompt in two chunks adds two means, and a chunk of a few drafts weighs as much as one of
 * thousands of tokens.  Needs no feature_window.  Decode queries that are on record (feature_window) for a sequence with
 * tokens came before the chunk: they are a chunk of their own, applied first, as fkv_update_features would, and leave the
 * record.  (A captured call takes the scale of the decode calls made before it was captured, and one captured before the first
 * of them leaves the record as it is.)  Errors as fkv_chunk_attn.
 */
int fkv_chunk_features(fkv_cache *c, int layer, const void *q, const float *lse, const int32_t *chunk_lens, int32_t window,
                       int32_t sinks, float scale, void *stream);

/*
 * ---- draft trees of a speculative decoder ----
 *
 * The drafts of a step as a tree: node 0 is its root, in general the token that the step before gave, whose pair is not stored yet;
 * every other node is a guess for the token after its parent.  A tree's nodes are packed like the tokens of a chunk (above), in any
 * order in which parents come before their children; tree_lens: host [max_batch], the nodes of every sequence's tree, at most
 * FKV_TREE_NODES each (0: the sequence takes no part).  One step:
 *     fkv_tree_masks(parents) -> masks
 *     for every layer:  fkv_append_tree_attn(k, v, q, masks) -> out, lse
 *     fkv_verify_tree(target's probabilities) -> path, path_len, tokens
 *     fkv_commit_tree(path, path_len)                 (all layers)
 * and the last one of `tokens` is the root of the next step's tree.  Everything only enqueues kernels and may be captured.
 *
 * fkv_tree_masks: parents dev [tokens] int32, a node's parent as an index inside its own tree (smaller than its own), or -1 for a root
 * (there may be several: children of the last stored pair).  masks: dev [tokens][FKV_TREE_WORDS] uint32, 16-byte aligned; bit i of
 * node j's mask (bit i % 32 of word i / 32) says that j sees node i: its ancestors and itself.  A parent that is not before its
 * node sets FKV_DEV_BAD_INDEX and counts as -1.
 *
 * fkv_append_tree: fkv_append_chunk for the nodes of trees.  pos NULL: a node's position is one more than its parent's, a root's the
 * one after the last pair that stays (with masks of another kind: as many further as the mask names nodes ahead of its own); given
 * positions must be behind that of the last pair that stays.
 * fkv_tree_attn: fkv_chunk_attn for the nodes of trees, which are the last tree_lens[s] pairs of their segments: a node sees the pairs
 * ahead of the tree as a chunk's token does (with window > 0 those inside the window of its own position, and the sinks), and the pairs
 * of the tree that its mask names up to its own (other masks than fkv_tree_masks writes are welcome; a node that sees nothing gets
 * zeros, and -infinity as its log-sum-exp).  A window must not be shorter than the longest tree, so that it holds every ancestor.
 * As in fkv_chunk_attn, P is rounded to bf16 for the product with V (as V is); everything else is fp32.
 * k and v of a tree must be finite.  A tree's own positions do not grow from pair to pair: commit it or roll it back (keep_lens) before
 * a call that goes by positions (windows, fkv_append without pos).  fkv_append_tree_attn: the two calls in one.  Errors and stream capture as for the chunk calls.
 *
 * fkv_verify_tree: which drafts stand, and the token after them, so that every token is distributed as the target says (speculative
 * sampling; siblings are tried in the order of their indices).  Per sequence, from a = node 0 with R = p = target[a]:
 *     for every child c of a, x = tokens[c]:
 *         accepted if u_accept[c] * draft[a][x] < R[x]:  go on at a = c with R = target[c];
 *         else R = max(R - draft[a], 0) / sum(max(R - draft[a], 0)),  or R = target[a] where that sum is 0;
 *     no child left: the next token is the first one whose running sum of R exceeds u_sample[s] times the whole sum.
 * draft NULL: the drafts are no samples but a choice (the likeliest tokens of a draft head): child c is accepted if u_accept[c] * m <
 * target[a][x], m = 1 less the probabilities of the siblings that were rejected; a rejection takes x out of R (a rejected token that
 * comes again has probability 0).
 * tokens, parents: dev [tokens] int32 (tokens[node 0] is not read; nodes that node 0 does not lead to are never reached; one whose token
 * is outside the vocabulary is passed over).  target, draft: dev [tokens][vocab] of dtype FKV_F32 or FKV_BF16, rows target_stride and
 * draft_stride elements apart (row a: the token after node a); taken as they are, not normalised, NaN and negative ones as 0.  A child
 * whose own draft[a][x] is NaN is rejected whatever its number: of a token that no known probability drew nothing can be said, and R, in
 * which the NaN counts as 0, gives the next one.  The draft's row of a node is read only where it has children.
 * u_accept: dev [tokens] fp32 (entry 0 of a tree is not read), u_sample: dev [max_batch] fp32, uniform in [0, 1): the library draws no
 * random numbers itself.  vocab at most 2^20.
 * path: dev [max_batch][path_stride] int32, the accepted nodes from node 0 down, -1 behind them; path_len: dev [max_batch] int32, their
 * number (at least 1, 0 without a tree); tokens_out: dev [max_batch][path_stride] int32, the path_len tokens that the step gives: those of
 * the accepted nodes behind node 0, then the next one (-1 if R is zero everywhere), -1 behind them.  path_stride is at least the longest tree.
 * Arithmetic in fp64.  Same inputs give same results, in any batch.
 * fkv_verify_tree_greedy: the same at temperature 0: choice dev [tokens] int32 is the target's own token after every node, a child is
 * accepted if it is that token (of several the first one), and the next token is the choice of the last accepted node.
 *
 * fkv_commit_tree: of every sequence's last tree_lens[s] pairs (its tree's) those of path[s][0 .. path_len[s]) move together behind the
 * pairs ahead of the tree, the others are dropped and their pages returned, in one layer or (FKV_ALL_LAYERS) in all.  path and path_len:
 * dev, as fkv_verify_tree writes them: ascending indices inside the tree; path_len[s] = 0 drops the whole tree.  A path that is not, or
 * a tree longer than its segment, sets FKV_DEV_BAD_INDEX and leaves the sequence as it is.  What a pair holds moves with it, so
 * fkv_chunk_features may follow with the path's queries and log-sum-exps (gathered, chunk_lens = path_len).  Decode queries on record that saw pairs of the tree leave the
 * record.  The new lengths are known to the device alone: call fkv_sync_lengths before any call that goes by the host's (until then the
 * host's are those with the whole trees; fkv_append_tree and fkv_append_chunk with keep_lens may follow at once).
 */
#define FKV_TREE_NODES 256
#define FKV_TREE_WORDS (FKV_TREE_NODES / 32)
enum { FKV_F32 = 0, FKV_BF16 = 1 };
int fkv_tree_masks(fkv_cache *c, const int32_t *parents, const int32_t *tree_lens, uint32_t *masks, void *stream);
int fkv_append_tree(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const int32_t *keep_lens,
                    const int32_t *tree_lens, const uint32_t *masks, void *stream);
int fkv_tree_attn(fkv_cache *c, int layer, const void *q, const int32_t *tree_lens, const uint32_t *masks, int32_t window,
                  int32_t sinks, float scale, void *out, float *lse_out, void *stream);
int fkv_append_tree_attn(fkv_cache *c, int layer, const void *k, const void *v, const int32_t *pos, const int32_t *keep_lens,
                         const int32_t *tree_lens, const uint32_t *masks, const void *q, int32_t window, int32_t sinks,
                         float scale, void *out, float *lse_out, void *stream);
int fkv_verify_tree(fkv_cache *c, const int32_t *tokens, const int32_t *parents, const int32_t *tree_lens, const void *target,
                    int64_t target_stride, const void *draft, int64_t draft_stride, int32_t dtype, int32_t vocab,
                    const float *u_accept, const float *u_sample, int32_t *path, int32_t *path_len, int32_t *tokens_out,
                    int32_t path_stride, void *stream);
int fkv_verify_tree_greedy(fkv_cache *c, const int32_t *tokens, const int32_t *parents, const int32_t *tree_lens,
                           const int32_t *choice, int32_t *path, int32_t *path_len, int32_t *tokens_out, int32_t path_stride,
                           void *stream);
int fkv_commit_tree(fkv_cache *c, int layer, const int32_t *tree_lens, const int32_t *path, const int32_t *path_len,
                    int32_t path_stride, void *stream);

/*
 * ---- sequences that are copied, change places or end ----
 * fkv_fork: every sequence s becomes, in all layers, what sequence from[s] was before the call (from[s] = s: it stays as it is; -1: it
 * is emptied and its pages are returned): a prompt for several samples, beams that change places, requests that end, in any mixture.
 * from: host [max_batch], read before the call returns; entries outside [-1, max_batch) are FKV_ERR_INVALID_ARG.  Everything a sequence
 * holds goes with it: pairs, features, positions, decode queries on record, its budget (an emptied place keeps its own).  Sequences never
 * share pages (each keeps features of its own in them): of a sequence that goes away while others become what it was, one takes the pages
 * over and the others get copies.  The pages of sequences that go away serve the copies; if these and the free ones are too few the
 * whole call does nothing (FKV_DEV_POOL_EXHAUSTED).  Only enqueues kernels; a replayed call does the same to what it finds.  The host's
 * lengths and budgets are those of a call that ran once and found its pages: call fkv_sync_lengths, which reads both, after the last
 * replay and after a call that did nothing.
 *
 * fkv_export_chunk: dense copy of the last chunk_lens[s] pairs of every sequence of a layer, packed, the inverse of fkv_append_chunk:
 * k, v dev [tokens][Hkv][D] bf16 (16-byte aligned), feat dev [tokens][Hkv][F] fp32 (8-byte aligned), pos dev [tokens][Hkv] int32 (after an eviction the
 * heads keep pairs of different positions); any may be NULL.  FKV_ERR_INVALID_ARG if a chunk is longer than its segment.
 */
int fkv_fork(fkv_cache *c, const int32_t *from, void *stream);
int fkv_export_chunk(fkv_cache *c, int layer, const int32_t *chunk_lens, void *k, void *v, float *feat, int32_t *pos, void *stream);

/* ---- staged entry points: one kernel each, for per-step checks ---- */

/*
 * The scorer alone - Appendix B.1: phi_n = sigma(Concat(k_n, v_n, a_n) W1 + b1) W2 + b2 for every pair
 * of `layer`, with the (layer, KV head)'s own weights (Section 3.1: one scoring model per layer and
 * attention group).  scores_out dev [max_batch][Hkv][cap] fp32, cap = fkv_score_stride.
 */
int fkv_score(fkv_cache *c, int layer, float *scores_out, void *stream);
/*
 * The selection alone - Section 3.1: the most recent R pairs stay, the others are pruned back to
 * B - R by score (the lowest scores are evicted; the Top-K row of the paper's sampling ablation, i.e.
 * the deterministic action; ties: higher score, then lower slot).  From given scores (dev, layout as
 * fkv_score writes them) writes for each segment the kept slots, ascending, to idx_out dev
 * [max_batch][Hkv][cap] int32 and their number min(B, n) to kept_count_out dev [max_batch][Hkv].
 */
int fkv_select(fkv_cache *c, int layer, const float *scores_in, int32_t *idx_out, int32_t *kept_count_out,
               void *stream);
/* Selection by the sampled action of fkv_evict_sampled from given scores; noise dev [max_batch][Hkv][noise_stride]. */
int fkv_select_sampled(fkv_cache *c, int layer, const float *scores_in, const float *noise, int32_t noise_stride,
                       int32_t *idx_out, int32_t *kept_count_out, void *stream);
/*
 * The compaction alone - Section 3.1's state update s' = s \ D: the kept pairs' K, V, feature and
 * position rows move, in order, into fresh pages and the segment's length becomes the kept count.
 * By given ascending slot lists (dev, layout as fkv_select writes them; every sequence must have the
 * same count on all its heads).  Syncs (reads the new lengths back).
 */
int fkv_compact(fkv_cache *c, int layer, const int32_t *idx, const int32_t *kept_count, void *stream);

/*
 * Attention features a_n of Appendix B.1, maintained by the library when feature_window > 0.
 * Every fkv_append_decode_attn / fkv_decode_step records the token's queries, their softmax
 * statistics and the number of pairs they saw (the last W tokens since the last eviction).
 * fkv_evict / fkv_evict_sampled then refresh the features of the segments they evict, before
 * scoring: per query head, in this order inside a_n,
 *   windows 8, 16, 32: (1/w) sum over the last w recorded queries of the softmax probability
 *                      the head gave the pair (0 for queries older than the pair),
 *   window = chunk:    the same mean over all recorded queries of the chunk (the chunk's score),
 *   direct sum:        previous value + chunk score,
 *   decayed sum:       0.9 * previous value + chunk score,
 * and start a new chunk.  With no query on record (e.g. right after fkv_prefill) the stored
 * features are used as they are.  The paper gives one sentence on these features; mean versus sum,
 * and what a chunk is, are this library's reading of it.
 * fkv_update_features does the refresh alone for `layer` (all its sequences), without closing the
 * chunk - a staged entry point for checks.  FKV_ERR_NOT_READY if feature_window is 0.
 */
int fkv_update_features(fkv_cache *c, int layer, void *stream);

/* Row stride, in elements, of the score and index arrays above. */
int fkv_score_stride(const fkv_cache *c, int32_t *cap);

/*
 * Dense copy of one segment: k, v dev [n][D] bf16, feat dev [n][F], pos dev [n]; any may be NULL.
 * The paper has no counterpart: a read-out for checks and for moving a cache elsewhere.
 */
int fkv_export_head(fkv_cache *c, int layer, int seq, int kv_head, void *k, void *v, float *feat, int32_t *pos,
                    void *stream);

/* Dense copy of the features of one (layer, sequence): feat dev [Hkv][n][F] fp32 (the layout fkv_set_features takes). */
int fkv_export_features(fkv_cache *c, int layer, int seq, float *feat, void *stream);

/* Current lengths of `layer`: host_out [max_batch] (host mirror, no device access). */
int fkv_get_lengths(const fkv_cache *c, int layer, int32_t *host_out);

/*
 * Reads the device status word and free-page count (syncs `stream`); clears the word.
 * When it returns FKV_ERR_DEVICE, a kernel has skipped work the host had already counted (an append, or
 * a whole eviction step), so the host's copy of the lengths may be ahead of the device: call
 * fkv_sync_lengths (or fkv_reset) before any other call on this handle.
 */
int fkv_device_status(fkv_cache *c, uint32_t *status_bits, int32_t *free_pages, void *stream);

/*
 * Re-read the lengths of every layer and the sequences' budgets from the device
 * into the host mirror (syncs).  After replays of captured calls, calls that
 * ended with an error bit, fkv_commit_tree, and for callers that restored a
 * saved copy of the workspace.
 */
int fkv_sync_lengths(fkv_cache *c, void *stream);

/*
 * Per-kernel timing of fkv_evict.  While on, fkv_evict records CUDA events on
 * the caller's stream around its kernels; fkv_get_evict_timing waits for the
 * last recorded set and returns milliseconds for
 * {plan, score, select (both passes of the sampled action), compact, commit, feature refresh}.
 */
int fkv_set_timing(fkv_cache *c, int on);
int fkv_get_evict_timing(fkv_cache *c, float ms_out[6]);

/* Number of kernel launches this handle has enqueued so far. */
int fkv_launch_count(const fkv_cache *c, uint64_t *launches);

/*
 * Decode attention without any allocation (the paper has no counterpart; this
 * is a service entry point of the library).
 *
 * For callers that may not allocate device memory: code running inside a
 * memory pool that was sized once and frozen, a serving process that accounts
 * for every byte of HBM itself, a plug-in that is handed tensors and nothing
 * else.  Such a caller cannot provide the workspace fkv_init_cache needs, so
 * this call takes dense tensors and keeps its split-K partials in a fixed
 * array inside the library image (about 1.1 MB of HBM on every GPU that loads
 * the library, held until the process exits).  It calls no cudaMalloc,
 * cudaFree or other allocating routine.
 *
 *   out[h] = sum_i softmax_i(scale <q[h], k[h / g][i]>) v[h / g][i],  i < n
 *
 * q, out: dev [num_kv_heads * group_size][head_dim] bf16; k, v: dev
 * [num_kv_heads][n][head_dim] bf16, dense row-major; scale 0 means
 * 1/sqrt(head_dim).  Same arithmetic as fkv_decode_attn (fp32 online softmax,
 * bf16 result), for one sequence.
 *
 * k and v must be 8-byte aligned (FKV_ERR_INVALID_ARG otherwise).  This is a
 * service path: it reads one row per warp and step and is far slower than
 * fkv_decode_attn for long sequences.
 *
 * Limits: head_dim 64 or 128 (else FKV_ERR_INVALID_ARG); 1 <= n <=
 * FKV_NOALLOC_MAX_PAIRS, num_kv_heads <= FKV_NOALLOC_MAX_KV_HEADS, group_size
 * <= 8 - beyond them the call does nothing and returns FKV_ERR_CAPACITY.
 *
 * The first call on a device looks up the array's device address (once per
 * device, with that device current); make that first call before any stream
 * capture begins.  All calls share the one array, which keeps the previous
 * call's partials (the call clears the only part that must start at zero):
 * two calls that overlap on the GPU - different streams, or different
 * threads without ordering - race on it.  Order them on one stream.
 */
#define FKV_NOALLOC_MAX_PAIRS (1 << 20)
#define FKV_NOALLOC_MAX_KV_HEADS 16
int fkv_decode_attn_dense_noalloc(const void *q, const void *k, const void *v, int32_t n, int32_t num_kv_heads,
                                  int32_t group_size, int32_t head_dim, float scale, void *out, void *stream);

/*
 * Golden Eviction labels - Section 3.2, Eq. 3-5: the supervision targets of the scorer, from the full
 * attention matrix of ONE attention group (no cache handle involved).
 *   attn: dev fp32 [g][T][T] attention probabilities of the group's g heads, row = query position,
 *         column = key position.
 * Query rows are cut into blocks of L starting at the first eviction position B + L (the last block
 * zero-padded): M = ceil((T - B) / L) - 1 blocks = eviction steps (fkv_golden_steps).  Block score =
 * average over the g heads and the block's L rows; future score alpha[t][i] = maximum of the block
 * scores of pair i over blocks t .. M; retained set of step t = the B - L pairs with the largest
 * alpha[t][.] among the B cached ones (those retained at step t - 1 plus the L tokens that just left
 * the recent window; [0, B) at step 1; ties: lower position).  The L newest tokens are kept by the
 * protocol and are not listed.
 *   alpha_out: dev fp32 [M][T] (row t - 1 = step t); kept_out: dev int32 [M][B - L], ascending.
 * B <= 8192 (FKV_ERR_CAPACITY beyond); M = 0 does nothing.  fkv_golden_select is the last step alone,
 * from given future scores.
 */
int fkv_golden_steps(int32_t T, int32_t B, int32_t L);
int fkv_golden_eviction(const float *attn, int32_t g, int32_t T, int32_t B, int32_t L, float *alpha_out,
                        int32_t *kept_out, void *stream);
int fkv_golden_select(const float *alpha, int32_t T, int32_t B, int32_t L, int32_t M, int32_t *kept_out, void *stream);

/* Text of the last CUDA error seen by this library on this thread ("" if none). */
const char *fkv_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FKV_H */
