/*
 * kafila_stage.h -- one pipeline stage of a decoder-only LLM on one MI355X (gfx950).
 *
 * In Kafila (arxiv 2609.34045) a model's contiguous chain of transformer blocks
 * is divided among the members of a ring; each member runs a *stage*: the
 * hidden state of every token passes through its block range, and the member
 * holding the *head* also embeds tokens before its blocks and unembeds and
 * samples after the model's last block (Section III and Fig. 1).  A stage's
 * decode cost is dominated by reading its weights once per token (Section V-A,
 * eq. (2)); the session reserves cache for a declared context and concurrency
 * and refuses a plan that would exhaust a device (Sections V-C, V-D).
 *
 * The block is a pre-norm decoder layer: RMSNorm, grouped-query attention with
 * rotate-half RoPE over a per-user KV cache, SwiGLU MLP, no biases.  The head is
 * an embedding gather, a final RMSNorm, the vocabulary projection and a greedy
 * argmax (lowest index on ties).
 *
 * Conventions
 *  - "_dev" pointers are device pointers on the stage's device; other pointers
 *    are host pointers.  The caller owns every I/O buffer.
 *  - bf16 tensors are passed as uint16_t bit patterns.  Matrices are row-major
 *    [out, in] (the layout of a linear layer's weight).
 *  - Compute calls only enqueue work on the stage's stream and return; argument
 *    checks run on the host before anything is enqueued, and a call that fails
 *    them changes no state.  Errors of enqueued work are sticky and surface from
 *    kf_stage_sync() or the next call as KF_EDEVICE.
 *  - A stage and its KV caches are not thread-safe; distinct stages are
 *    independent.  kf_last_error() returns a thread-local message for the last
 *    failure on the calling thread.
 *  - Requirements checked at init: head_dim in {64, 128}; n_q_heads a multiple
 *    of n_kv_heads with at most 8 query heads per KV head; hidden and ffn
 *    multiples of 64.  Anything else is KF_EUNSUPPORTED.  The query width
 *    n_q_heads * head_dim need not equal hidden.
 */
#ifndef KAFILA_STAGE_H
#define KAFILA_STAGE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KF_ABI_VERSION 5  /* 2: kf_model_config.qk_norm and the q/k norm tensor kinds;
                            3: paged KV caches, kf_stage_describe, kf_kv_describe;
                            4: kf_stage_set_flags / kf_stage_get_flags (KF_STAGE_ORDERED), range and
                               NaN-logit errors reported by kf_stage_sync, token -1 for a row of NaN logits,
                               kf_stage_prefill_noalloc; kf_ring_generate's hidden_out_dev (kafila_ring.h);
                               the kf_shard_* loader (kafila_shard.h);
                            5: a head stage's decode may keep its output rows (hidden_out_dev NULL)
                               for kf_head_logits / kf_head_argmax with hidden_dev NULL.
                            Calls added since leave the others as they are: kf_kv_create_typed,
                            kf_kv_format, kf_kv_copy, kf_kv_fork, kf_kv_attend,
                            kf_head_logprobs, kf_logits_logprobs, kf_kv_attend_tree,
                            kf_kv_accept, kf_kv_track, kf_kv_weigh, kf_kv_weights,
                            kf_kv_set_weights, kf_kv_evict, kf_kv_dropped, kf_kv_set_dropped */
#define KF_KV_PAGE 64     /* positions per KV cache page */
#define KF_MAX_BATCH 4

typedef struct kf_stage kf_stage;
typedef struct kf_kv kf_kv;

typedef enum {
  KF_OK = 0,
  KF_EINVAL = 1,       /* malformed argument (NULL, size mismatch, position gap, bad range) */
  KF_ENOMEM = 2,       /* a device or host allocation failed */
  KF_ERANGE = 3,       /* a position or length beyond the declared capacity */
  KF_ESTATE = 4,       /* call not allowed in this state (e.g. head call on a stage without the head) */
  KF_EDEVICE = 5,      /* a HIP error, including a sticky error from earlier enqueued work */
  KF_EUNSUPPORTED = 6  /* a model shape the kernels are not built for */
} kf_status;

typedef enum { KF_F32 = 0, KF_BF16 = 1, KF_F16 = 2 } kf_dtype; /* element types at the boundary */

typedef struct {
  int32_t n_layers;   /* layers in the whole model (the stage holds a sub-range) */
  int32_t hidden;     /* H */
  int32_t n_q_heads;  /* nq */
  int32_t n_kv_heads; /* nkv; query head h reads KV head h / (nq / nkv) */
  int32_t head_dim;   /* hd */
  int32_t ffn;        /* F */
  int32_t vocab;      /* V (used only with the head) */
  float rms_eps;      /* RMSNorm epsilon, added to mean(x^2) inside the square root */
  float rope_theta;   /* RoPE base: pair (i, i + hd/2) turns by pos * theta^(-2i/hd) */
  int32_t qk_norm;    /* 1: each q and k head vector is RMS-normalised (gains KF_W_Q_NORM / KF_W_K_NORM,
                         eps rms_eps) before RoPE, as in the Qwen3 models the paper serves; 0: no such norm */
} kf_model_config;

typedef enum {
  KF_W_ATTN_NORM = 0, /* [H]            gain of the attention RMSNorm */
  KF_W_Q = 1,         /* [nq*hd, H] */
  KF_W_K = 2,         /* [nkv*hd, H] */
  KF_W_V = 3,         /* [nkv*hd, H] */
  KF_W_O = 4,         /* [H, nq*hd] */
  KF_W_MLP_NORM = 5,  /* [H]            gain of the MLP RMSNorm */
  KF_W_GATE = 6,      /* [F, H] */
  KF_W_UP = 7,        /* [F, H] */
  KF_W_DOWN = 8,      /* [H, F] */
  KF_W_EMBED = 9,     /* [V, H]         head only */
  KF_W_FINAL_NORM = 10, /* [H]          head only */
  KF_W_LM_HEAD = 11,  /* [V, H]         head only (not tied to the embedding) */
  KF_W_Q_NORM = 12,   /* [hd]           gain of the per-head q norm (only when qk_norm) */
  KF_W_K_NORM = 13    /* [hd]           gain of the per-head k norm (only when qk_norm) */
} kf_tensor_kind;

typedef struct {
  int32_t layer;        /* global layer index in [layer_lo, layer_hi); -1 for head tensors */
  int32_t kind;         /* kf_tensor_kind */
  const uint16_t* bf16; /* host pointer to row-major bf16 bits */
  int64_t numel;        /* must equal the element count of the kind's shape */
} kf_tensor;

typedef struct {
  const kf_tensor* tensors;
  int32_t count;
} kf_weights;

/* ABI version of the loaded library (KF_ABI_VERSION at build time). */
int32_t kf_abi_version(void);

/* Thread-local message describing the last failed call on this thread ("" if none). */
const char* kf_last_error(void);

/*
 * Byte sizes behind the stage-cost model (Section V-A, eq. (2)) and the block
 * limit at a declared context and concurrency (Section V-C).
 *   beta_block : bytes of one decoder layer's weights (2 bytes per element as given in bf16 and as
 *                held: fp16 matrices, bf16 gains; both gains included)
 *   beta_head  : bytes of the head's weights (embedding + final gain + LM head), 0 without the head
 *   resident   : device bytes kf_stage_init + kf_kv_create(max_users, max_ctx) would hold for
 *                layers [lo, hi): weights, KV cache, RoPE table and decode workspaces (not the
 *                workspaces that a first prefill or many-row logits call allocates)
 * Host only; any output pointer may be NULL.  KF_EINVAL for an invalid config or range.
 */
kf_status kf_stage_bytes(const kf_model_config* cfg, int32_t layer_lo, int32_t layer_hi, int32_t has_head,
                         int32_t max_users, int32_t max_ctx, int64_t* beta_block, int64_t* beta_head,
                         int64_t* resident);

/*
 * Create a stage holding layers [layer_lo, layer_hi) of the model and, if has_head,
 * the head (Section III and Fig. 1: a member's contiguous block range, and the
 * head's embedding and unembedding on the member the rotation makes head;
 * Section V-C places it).  Weight tensors are copied to the current HIP device (the stage's
 * device) before the call returns, so the caller may free them afterwards.  Every
 * layer tensor of every held layer must be present exactly once (kinds 0..8, plus
 * KF_W_Q_NORM and KF_W_K_NORM when qk_norm), plus the three head tensors when
 * has_head; anything else is KF_EINVAL.  The weight matrices (kinds Q, K, V, O, GATE,
 * UP, DOWN, LM_HEAD) are stored in fp16, rounded to nearest even from the bf16
 * given: exact for 2^-17 <= |w| < 65504 and for 0, within 2^-25 below that.  A finite
 * weight that fp16 cannot hold (|w| >= 65520) is KF_EINVAL.  Gains and the
 * embedding table stay bf16.  hip_stream (a
 * hipStream_t, NULL for the default stream) is where all later work is enqueued.
 */
kf_status kf_stage_init(const kf_model_config* cfg, int32_t layer_lo, int32_t layer_hi, int32_t has_head,
                        const kf_weights* weights, void* hip_stream, kf_stage** out);

/* Waits for the stage's stream, then frees its device memory.  KV caches of the stage must be destroyed first. */
kf_status kf_stage_destroy(kf_stage* stage);

/* Replace the stream later work is enqueued on (the caller orders it after earlier work). */
kf_status kf_stage_set_stream(kf_stage* stage, void* hip_stream);

/*
 * Wait for all enqueued work; KF_EDEVICE (with the HIP error text) if any of it failed.
 * Then reports, and clears, the stage's sticky data errors raised by enqueued work:
 *   KF_EINVAL : a token id given to decode or prefill was outside [0, vocab); that row's
 *               hidden state was set to NaN (a target's log probability alike);
 *   KF_ERANGE : a value the stage holds in fp16 (keys and values in the cache, and the
 *               fp16 activations: from batch 2 the decode residual copy, SwiGLU output and
 *               merged attention output; in prefill the normalised rows, queries, attention
 *               output and SwiGLU output) reached 65520 in magnitude and was stored as
 *               infinity (in an MXFP4 cache as 49152, and a NaN as 0); or a logit was NaN (skipped by
 *               the argmax and the log probabilities; see kf_head_argmax and kf_head_logprobs);
 *   KF_ESTATE : two captured evictions in place of one cache were replayed at the same time, and pages
 *               of positions were left where they were (see kf_kv_evict).
 * The message (kf_last_error) names every condition that occurred.
 */
kf_status kf_stage_sync(kf_stage* stage);

/*
 * Behaviour flags of a stage (0 after kf_stage_init).
 *   KF_STAGE_ORDERED : batch-1 decode adds the query heads' output projections to each
 *                      residual row in a fixed order (a separate merge of the split-KV
 *                      partials, then a row-owning output GEMV), so that repeated runs are
 *                      bit-identical and a stage split anywhere composes to the same bits.
 *                      Without it, batch 1 fuses the merge into a head-split output
 *                      projection whose fp32 additions arrive in any order (one launch
 *                      fewer per layer; results vary run to run by fp32 reassociation).
 *                      Greedy decoding at a fixed seed (Section VI-A) reproduces exactly
 *                      only with this flag.  Batch 2-4 and prefill are always in fixed order.
 * kf_stage_set_flags: KF_EINVAL for unknown bits.  Host-only; affects later calls.
 */
#define KF_STAGE_ORDERED 1
kf_status kf_stage_set_flags(kf_stage* stage, int32_t flags);
kf_status kf_stage_get_flags(const kf_stage* stage, int32_t* flags);

/* What a stage holds: its config, layer range [layer_lo, layer_hi), whether it holds
 * the head, the stream it enqueues on (a hipStream_t) and its device ordinal.  Any
 * output pointer may be NULL.  Host-only. */
kf_status kf_stage_describe(const kf_stage* stage, kf_model_config* cfg, int32_t* layer_lo, int32_t* layer_hi,
                            int32_t* has_head, void** hip_stream, int32_t* device);

/*
 * Reserve a KV cache for max_users concurrent users of context up to max_ctx tokens
 * each, for every layer the stage holds (the declared concurrency x context of
 * Section V-C).  Layout on the device: fp16 K and V in pages of KF_KV_PAGE
 * positions, [layer][page][kv_head][KF_KV_PAGE][hd]; user u holds pages
 * u * P .. u * P + P - 1 with P = ceil(max_ctx / KF_KV_PAGE) (fp16 keeps 8x the
 * mantissa of bf16 in the same bytes; keys and values must stay below 65504 in
 * magnitude).
 * All user lengths start at 0.  KF_ENOMEM if the device cannot hold it.
 */
kf_status kf_kv_create(kf_stage* stage, int32_t max_users, int32_t max_ctx, kf_kv** out);

/*
 * A paged KV cache: the same users and context limits, but only n_pages pages
 * (>= 1) of KF_KV_PAGE positions for all users together, so that cache is held by
 * the prompts that arrive rather than reserved for every declared user (the
 * reservation the paper leaves as future work, Section VIII).  A user is lent
 * pages from the pool as its length grows (decode, prefill, kf_kv_write,
 * kf_kv_set_len) and gives back the pages past its new length when
 * kf_kv_set_len shortens it (0 frees them all).  A call that needs more pages
 * than are free fails with KF_ENOMEM before anything is enqueued.  A device
 * table [max_users][P] maps each user's page index to a pool page.
 */
kf_status kf_kv_create_paged(kf_stage* stage, int32_t max_users, int32_t max_ctx, int32_t n_pages, kf_kv** out);

/*
 * A cache of a given type: KF_KV_F16 as kf_kv_create (n_pages 0) and kf_kv_create_paged
 * (n_pages >= 1) make it, or KF_KV_MXFP4, reserved or paged alike, which takes 35/128 of the bytes.
 * An MXFP4 cache holds each head vector of a key or value in blocks of 32 consecutive
 * values: E2M1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign), rounded to
 * nearest even, times one power of two 2^e.  A value x is rounded to fp16 first; e is
 * the exponent of the block's largest |x|, rounded to one mantissa bit, less 2, in
 * [-23, 13], so that the largest rounds to 4 or 6 times 2^e; magnitudes past 6 2^13 = 49152
 * become that.  Every stored value is an fp16 number.  Infinities and what fp16 rounds
 * to one are stored as 49152, a NaN as 0, and all three raise the stage's range
 * error (KF_ERANGE from kf_stage_sync).
 * Every call takes caches of both types.  Decode attends to the new position as it is
 * stored.  Prefill attends through fp16 pages of one user and layer that an MXFP4 cache keeps
 * beside its own (max_ctx positions, or the pool's where those are fewer).  KF_EINVAL for a negative n_pages or an unknown type.
 */
typedef enum { KF_KV_F16 = 0, KF_KV_MXFP4 = 1 } kf_kv_type;
kf_status kf_kv_create_typed(kf_stage* stage, int32_t max_users, int32_t max_ctx, int32_t n_pages, kf_kv_type type,
                             kf_kv** out);

/* A cache's type and the device bytes it holds (pages, tables and workspaces).  Any output pointer may be NULL.  Host-only. */
kf_status kf_kv_format(const kf_kv* kv, kf_kv_type* type, int64_t* bytes);
kf_status kf_kv_destroy(kf_kv* kv);

/* Pages of the cache and, for a paged cache, how many are free (-1 for a reserved cache, whose users
 * hold all their pages from the start).  Host-only. */
kf_status kf_kv_pages(const kf_kv* kv, int32_t* total, int32_t* free_pages);

/* The stage a cache was created on, and its capacity.  Any output pointer may be NULL.  Host-only. */
kf_status kf_kv_describe(const kf_kv* kv, kf_stage** stage, int32_t* max_users, int32_t* max_ctx);

/* Number of cached positions of a user (a host-side value; no device sync). */
kf_status kf_kv_len(const kf_kv* kv, int32_t user, int32_t* len);

/* Set a user's length to any value in [0, max_ctx]: 0 resets the user; positions below
 * len are from then on taken as valid in every layer (e.g. after kf_kv_write).  In a
 * paged cache the user holds exactly the pages its length needs afterwards
 * (KF_ENOMEM, with nothing changed, if the pool cannot lend them). */
kf_status kf_kv_set_len(kf_kv* kv, int32_t user, int32_t len);

/*
 * Copy n positions of keys (already rotated) and values for one held layer and user,
 * from k_dev / v_dev laid out [n, nkv, hd] in dtype (KF_F16 or KF_BF16 bits, or KF_F32),
 * stored as fp16 rounded to nearest even, into positions [pos0, pos0 + n).  Does not
 * change lengths (a paged cache lends the pages up to pos0 + n; KF_ENOMEM if it cannot).
 * KF_ERANGE if pos0 + n > max_ctx.  Enqueued on the stage's stream.
 */
kf_status kf_kv_write(kf_kv* kv, int32_t layer, int32_t user, int32_t pos0, int32_t n, const void* k_dev,
                      const void* v_dev, kf_dtype dtype);

/* Copy positions [pos0, pos0 + n) of one layer and user out as fp32 (exact), [n, nkv, hd].
 * KF_ERANGE for positions on pages the user does not hold (paged caches). */
kf_status kf_kv_read(const kf_kv* kv, int32_t layer, int32_t user, int32_t pos0, int32_t n, float* k_dev,
                     float* v_dev);

/*
 * Copy positions [pos0, pos0 + n) of src_user, in every layer the stage holds, to the
 * same positions of dst_user in the same cache or another one of the stage (a user
 * handed from one cache to another, e.g. an idle one from fp16 into 4 bits).  Between
 * types the values are converted: to MXFP4 as kf_kv_write stores them, to fp16 exactly.
 * Does not change lengths (a paged destination lends the pages up to pos0 + n;
 * KF_ENOMEM if it cannot).  KF_ERANGE past either cache's max_ctx or for positions on
 * pages that src_user does not hold; KF_EINVAL for caches of different stages and for a
 * user copied onto itself.  Enqueued on the stage's stream.
 */
kf_status kf_kv_copy(kf_kv* dst, int32_t dst_user, const kf_kv* src, int32_t src_user, int32_t pos0, int32_t n);

/*
 * Give dst_user the first n positions of src_user (n at most its length) in place of
 * whatever it held, and the length n: several continuations of one prompt.  A reserved
 * cache copies the positions.  In a paged cache the two users share the pages, at no
 * cost in pages; a user that writes to a page others hold too (decode, prefill,
 * kf_kv_write, kf_kv_copy) first gets a copy of its own from the pool (KF_ENOMEM
 * if it has none), so that no user sees another's writes.  A shared page returns to the pool when
 * its last user gives it back.  KF_EINVAL for src_user == dst_user, KF_ERANGE for n
 * above src_user's length.
 * Which pages are shared is known when a call is made, not when a graph is replayed: under graph
 * capture a paged fork, and a call that would first copy a shared page, is KF_ESTATE.  Pages that a
 * captured call lends are their user's from that call on, replayed or not.  A replay uses the pages that the
 * users hold by then, and counts nothing: replay a graph while they hold the positions that it uses, and
 * capture anew what writes to pages that have been shared since.
 */
kf_status kf_kv_fork(kf_kv* kv, int32_t src_user, int32_t dst_user, int32_t n);

/*
 * Attention of given queries over cached positions of one held layer, as a decode step
 * attends: out[b][h] = softmax(q[b][h] . K^T / sqrt(hd)) V over positions [0, lens[b]) of
 * users[b], query head h reading KV head h / (nq / nkv).
 *   rows : 1..KF_MAX_BATCH; users may repeat (several queries of one user, or users
 *          that share pages); lens[b] 0 gives a row of zeros
 *   q_dev : [rows, nq, hd] rotated queries in io (KF_F32, KF_BF16 or KF_F16), 16-byte aligned
 *   out_dev : [rows, nq, hd] in io; may be q_dev
 * Over caches of both types the products take queries and probabilities in two fp16 parts each (22 bits),
 * whatever the queries' size, and fp32 sums.  (A decode step on an fp16 cache takes one part of each.)
 * A query head that holds a NaN or an infinity gives NaN.  KF_ERANGE for lens[b] beyond max_ctx or the pages the user holds.
 * Changes nothing in the cache.  Enqueued on the stage's stream.
 */
kf_status kf_kv_attend(kf_kv* kv, int32_t layer, int32_t rows, const int32_t* users, const int32_t* lens,
                       const void* q_dev, kf_dtype io, void* out_dev);

/*
 * Attention of drafted tokens, each with its own branch of a tree of continuations (one
 * step of speculative decoding, verified in one pass).  Tree b has nodes[b] tokens of users[b],
 * whose keys and values lie at positions lens[b] + i (kf_kv_write them there first); token i
 * attends to positions [0, lens[b]), to itself and to its ancestors.
 *   trees : 1..KF_MAX_BATCH; users may repeat; nodes[b] 0..KF_MAX_NODES (0: no rows)
 *   parents_dev int32 [sum of nodes] : the parent of each token within its tree, an earlier token;
 *           -1 where it follows position lens[b] - 1; -2 for a row that only pads the tree, which
 *           gives zeros and which no token sees (a token that names it as its parent sees itself and what lies
 *           before the tree).  Any other value counts as -1.
 *   q_dev, out_dev : [sum of nodes, nq, hd] in io, tree after tree; as for kf_kv_attend
 * Queries and probabilities keep 22 bits.  A position that a token does not see does not reach it, whatever it holds; an
 * infinite value that it sees shows in its place alone, and a key whose score is -inf counts for nothing.  KF_ERANGE for
 * positions beyond max_ctx or the pages the user holds.
 * The splits' partial results use the cache's own workspace, which kf_kv_attend and decode use too.
 * Changes nothing in the cache.  Enqueued on the stage's stream.
 */
#define KF_MAX_NODES 256
kf_status kf_kv_attend_tree(kf_kv* kv, int32_t layer, int32_t trees, const int32_t* users, const int32_t* lens,
                            const int32_t* nodes, const int32_t* parents_dev, const void* q_dev, kf_dtype io,
                            void* out_dev);

/*
 * The accepted tokens of a tree become context: position len + nodes[i] of the user moves to
 * len + i, for i < n, in every layer the stage holds, exactly as it is held; the user's length becomes len + n, and the pages
 * past it are given back.  nodes: host array, ascending, in [0, KF_MAX_NODES); n 0..KF_MAX_NODES (0: the
 * length alone).  KF_ERANGE for positions beyond max_ctx or the pages the user holds; a
 * page that other users hold too is copied first, as for any write (KF_ENOMEM; KF_ESTATE under graph capture).
 */
kf_status kf_kv_accept(kf_kv* kv, int32_t user, int32_t len, int32_t n, const int32_t* nodes);

/*
 * From now on the cache adds up the attention weight of every position: for each layer and KV head,
 * the sum of the probabilities that queries of its group's heads gave the position, in fp32.
 * Added are every row of a decode step, the last `window` (0..KF_MAX_WEIGH_ROWS) tokens of each prefill
 * chunk, and what kf_kv_weigh is given; not kf_kv_attend and kf_kv_attend_tree.  A head's probabilities add up to 1
 * within fp32 sums: queries keep 22 bits in maximum, sum and exponent alike (a prefill chunk's 11, as fp16 has
 * them), also of a step whose attention rounds them to 11.  A position that is written anew (decode, prefill, kf_kv_write)
 * starts at 0; kf_kv_copy and kf_kv_fork copy the weights (0 from an untracked cache), kf_kv_accept and
 * kf_kv_evict move them with their positions, and kf_kv_set_len leaves them.
 * The first call allocates 4 bytes per layer, KV head and position of max_ctx of every user, and a
 * little more than once more of one user (KF_ENOMEM; KF_ESTATE under graph capture), and the weights
 * start at 0; later calls set the window alone.
 */
#define KF_MAX_WEIGH_ROWS 32
kf_status kf_kv_track(kf_kv* kv, int32_t window);

/*
 * Add the attention weights of given queries in one held layer of a tracked cache (else KF_ESTATE):
 * row b attends to positions [0, lens[b]) of users[b], as for kf_kv_attend; users may repeat (a
 * prompt's last queries, say, each over one position more).  rows 1..KF_MAX_WEIGH_ROWS; lens[b] 0 adds nothing.
 * A query head whose softmax is not finite (a NaN or an infinity among its query or the keys it sees) adds nothing.
 * The order of all additions is fixed.  Uses the cache's own workspace, as kf_kv_attend does.  Enqueued on the stage's stream.
 */
kf_status kf_kv_weigh(kf_kv* kv, int32_t layer, int32_t rows, const int32_t* users, const int32_t* lens, const void* q_dev,
                      kf_dtype io);

/* Copy the weights of positions [pos0, pos0 + n) of one layer and user out, [nkv, n], or in (a user that was saved, or
 * weights of the caller's own).  KF_ESTATE for an untracked cache, KF_ERANGE past max_ctx.  Enqueued on the stage's stream. */
kf_status kf_kv_weights(const kf_kv* kv, int32_t layer, int32_t user, int32_t pos0, int32_t n, float* weights_dev);
kf_status kf_kv_set_weights(kf_kv* kv, int32_t layer, int32_t user, int32_t pos0, int32_t n, const float* weights_dev);

/*
 * Give dst_user `keep` positions of src_user (at most its length, else KF_ERANGE) in place of whatever it
 * held, and the length keep: in each layer and KV head the first `first`, the last `last` (first + last <= keep)
 * and, of those between, the ones of the largest weights, the lower position of two equal ones and a NaN
 * below every number.  They keep their order, their exact values and their weights.  The keys keep the rotation of
 * the positions they came from, and the tokens that follow (kf_stage_decode, kf_stage_prefill) are rotated as the
 * source's would have been: to their slot plus what was dropped (kf_kv_dropped).  dst_user may be src_user (in
 * place); else src_user is left as it is.
 *   kept_dev : int32 [layers held, nkv, keep], the positions kept, ascending; may be NULL
 * Tracked caches only (else KF_ESTATE).  In a paged cache dst_user gives its pages back and is lent what keep
 * positions need; in place, other pages take the place of those that other users hold too (KF_ENOMEM, with nothing
 * changed, if the pool cannot lend them), and a call under graph capture is KF_ESTATE.  Uses the cache's own workspace:
 * captured evictions of one cache are not replayed at the same time (KF_ESTATE from kf_stage_sync, with what the users hold
 * lost, where that is seen).  Enqueued on the stage's stream.
 */
kf_status kf_kv_evict(kf_kv* kv, int32_t src_user, int32_t dst_user, int32_t keep, int32_t first, int32_t last,
                      int32_t* kept_dev);

/*
 * How many positions evictions have dropped before a user's next token: the token at slot p is rotated to position
 * p + dropped, and callers that rotate their own queries and keys do the same.  Evictions add to it; kf_kv_fork, and a
 * kf_kv_copy from position 0, take it along; an empty user (length 0) has none.  Setting it (0 .. INT32_MAX - max_ctx, else
 * KF_ERANGE) is for users that were saved and written back.  The cache's table of rotations grows with it, to the farthest
 * position that a user can reach: 8 bytes for each position and pair of a head and up to a quarter more, beside which the new
 * table is made (KF_ENOMEM, with nothing changed); tables that captured steps read are kept while the cache is.  A call that cannot allocate, under graph capture or
 * kf_stage_prefill_noalloc, and that lacks rows is KF_ESTATE: an eviction outside a capture makes those that its user can need.
 */
kf_status kf_kv_dropped(const kf_kv* kv, int32_t user, int32_t* dropped);
kf_status kf_kv_set_dropped(kf_kv* kv, int32_t user, int32_t dropped);

/*
 * Forward one token for each of `batch` (1..KF_MAX_BATCH) users (decode): the
 * stage's part of one decode step, hidden state in, hidden state out (Section III:
 * the token's hidden state passes through each member's block range around the
 * ring; the head member embeds it first).  Its cost is one read of every held
 * weight plus each user's cache (Section V-A, eq. (2)); batch > 1 serves several
 * users' requests in one pass over the weights (Sections III and VII-C).
 *   users[b], positions[b] : host arrays; users distinct and < max_users;
 *                            positions[b] must equal the user's current length
 *                            (append-only; else KF_EINVAL) and be < max_ctx (else KF_ERANGE).
 *   tokens_dev  : int32 [batch] token ids (stage with the head only), or NULL
 *   hidden_in_dev : [batch, H] in `io`, or NULL; exactly one of tokens_dev / hidden_in_dev
 *   hidden_out_dev : [batch, H] in `io`; may alias hidden_in_dev.  NULL (a stage
 *                    that holds the head only, else KF_EINVAL): the output rows stay
 *                    in the stage for the head (kf_head_logits / kf_head_argmax with
 *                    hidden_dev NULL), as when the member that holds the model's
 *                    last blocks also holds the head and samples the next token.
 *                    At batch 2-4 they are kept in fp16 (the rounding every layer's
 *                    input of this stage already takes), which halves the LM head's
 *                    input traffic; at batch 1 in fp32.
 * Row b's token is at positions[b]: its key and value are written at that slot of
 * the user's cache in every held layer, and it attends slots 0..positions[b].
 * On success every user's length advances by one.  A paged cache lends a page to
 * each user whose position starts one (KF_ENOMEM, nothing enqueued, if the pool
 * is short for the batch).
 */
kf_status kf_stage_decode(kf_stage* stage, kf_kv* kv, int32_t batch, const int32_t* users,
                          const int32_t* positions, const int32_t* tokens_dev, const void* hidden_in_dev,
                          void* hidden_out_dev, kf_dtype io);

/*
 * Forward a chunk of n_tokens consecutive tokens of one user starting at pos0 (prefill:
 * the prompt phase of a request, which the paper separates from decode in its
 * time-to-first-token accounting, Section VI; the per-user cache it fills is the
 * reservation of Section V-C).  pos0 must equal the user's length and pos0 + n_tokens <= max_ctx.  Token i attends
 * slots 0..pos0+i.  tokens_dev int32 [n] or hidden_in_dev [n, H]; hidden_out_dev [n, H].
 * A paged cache lends the pages up to pos0 + n (KF_ENOMEM if it cannot).
 * Dense products run on the matrix cores with fp16 operands (the stage's fp16 weights)
 * and fp32 accumulation.  The stage's workspace grows to the longest chunk; where the device has not
 * the memory for all the partial sums that would be fastest, the sums are split less (the last
 * bits of the results may differ), and KF_ENOMEM only where the chunk does not fit at all.
 * On success the user's length advances by n_tokens.
 */
kf_status kf_stage_prefill(kf_stage* stage, kf_kv* kv, int32_t user, int32_t pos0, int32_t n_tokens,
                           const int32_t* tokens_dev, const void* hidden_in_dev, void* hidden_out_dev,
                           kf_dtype io);

/*
 * kf_stage_prefill without any device allocation, for callers that cannot allocate:
 * code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, checks, results and state changes as
 * kf_stage_prefill; the chunk's workspace (residual rows, normalised rows,
 * split-K partial sums, queries, attention output, SwiGLU output) lives in a static
 * per-device scratch array of KF_PREFILL_SCRATCH_BYTES instead of the stage's own
 * grown buffer.  A chunk whose workspace exceeds it is KF_ERANGE (nothing enqueued);
 * a 512-token chunk of every shape used here fits (the largest, hidden 8192 with
 * ffn 28672, needs 132 MiB).  All no-allocation prefills on one device share the
 * array: calls on one device whose work overlaps (other streams, other stages, other
 * threads) race, so the caller orders them.  No per-kernel timing is recorded.
 */
#define KF_PREFILL_SCRATCH_BYTES (144LL << 20)
kf_status kf_stage_prefill_noalloc(kf_stage* stage, kf_kv* kv, int32_t user, int32_t pos0, int32_t n_tokens,
                                   const int32_t* tokens_dev, const void* hidden_in_dev, void* hidden_out_dev,
                                   kf_dtype io);

/*
 * The head's unembedding (Section III and Fig. 1: the head member holds the
 * embedding and unembedding and samples after the model's last block):
 * logits_dev fp32 [rows, V] = RMSNorm(hidden; final gain) x LM_head^T, for hidden_dev
 * [rows, H] in dtype (KF_F32 or KF_BF16), any rows >= 1.  Head stages only (else KF_ESTATE).
 * Equal LM-head rows give exactly equal logits.  Up to four rows and more rows sum in
 * different orders (the last bits of a row's logits may differ between the two); among
 * calls of more than four, a row's logits have the same bits whatever the count.  These
 * use a workspace of 6 KB and 1 KB per hidden value, allocated at a stage's first such call and kept;
 * where it cannot be had (no device memory left, or that call is under HIP graph capture)
 * the rows go four at a time, in the order and at the cost of such calls.
 * A row whose values two fp16 parts do not hold (more than an eighth of them far below its
 * largest, or an infinity) is taken in fp32 all the same; such rows cost a pass over the LM head per four.
 * hidden_dev NULL: the rows the stage's last kf_stage_decode kept (its hidden_out_dev
 * was NULL); rows must equal that decode's batch and dtype is ignored (else KF_ESTATE,
 * also when the last decode returned its rows or failed).
 */
kf_status kf_head_logits(kf_stage* stage, int32_t rows, const void* hidden_dev, kf_dtype dtype, float* logits_dev);

/*
 * The head's sampler: greedy decoding (Section VI-A decodes greedily at a fixed
 * seed).  token_dev int32 [rows] = argmax over the vocabulary of the logits of
 * kf_head_logits, the lowest index winning exact ties; max_logit_dev fp32 [rows]
 * (may be NULL) receives the winning logit.  A NaN logit is skipped and raises the
 * stage's NaN-logit error (KF_ERANGE from kf_stage_sync); a row whose logits are all
 * NaN gives token -1 and max logit NaN.  rows in [1, KF_MAX_BATCH] (else KF_EINVAL).
 * Head stages only (else KF_ESTATE).  hidden_dev NULL: the kept rows, as for kf_head_logits.
 */
kf_status kf_head_argmax(kf_stage* stage, int32_t rows, const void* hidden_dev, kf_dtype dtype,
                         int32_t* token_dev, float* max_logit_dev);

/*
 * Log probabilities instead of logits or an argmax: what scoring a prompt, sampling with
 * alternatives or a beam search takes from the head.  rows, hidden_dev and dtype as
 * for kf_head_logits (any rows; hidden_dev NULL: the kept rows).
 *   targets_dev int32 [rows], logprob_dev fp32 [rows] : both or neither.  logprob =
 *       z_t - ln sum e^z of the row's logits z; a target of -1 (padding) gives 0, any
 *       other id outside [0, vocab) NaN and the stage's token error
 *   entropy_dev fp32 [rows] or NULL : -sum p ln p, in nats
 *   n_top in [0, KF_MAX_TOP], top_ids_dev int32 and top_logprobs_dev fp32 [rows, n_top] :
 *       the most probable tokens, largest first, the lower id first among equal logits
 * A logit of -inf is masked: probability 0 and never an alternative; where a row has
 * fewer than n_top others the rest are -1 with -inf.  A row with nothing left gives
 * -inf for its target and entropy 0.  A NaN or +inf logit is left out and raises
 * the NaN-logit error (a target there gives NaN).
 * The logits of up to 256 rows stay in a workspace of the stage (4 rows for calls of up
 * to 4, 64 up to 64), allocated by the first call that needs it and kept; KF_ENOMEM
 * where not even 4 rows can be had, which includes a first call under graph capture.
 * More than four bf16 rows (where the matrix holds the gain) take logits of plain fp32 sums, off by some
 * 4e-7 of their size; kf_head_logits' own are off by 1e-7.
 * Vocabularies up to 2^20 (else KF_EUNSUPPORTED).  Head stages only (else KF_ESTATE).
 */
#define KF_MAX_TOP 32
kf_status kf_head_logprobs(kf_stage* stage, int32_t rows, const void* hidden_dev, kf_dtype dtype,
                           const int32_t* targets_dev, float* logprob_dev, float* entropy_dev, int32_t n_top,
                           int32_t* top_ids_dev, float* top_logprobs_dev);

/*
 * The same of logits that the caller holds (after masking or a temperature of its own):
 * logits_dev fp32 [rows] rows of `vocab` values, `stride` values apart.  Any stage;
 * the logits may be of another vocabulary than the stage's.
 * Rows that more than one workgroup takes (longer than 8192 values) have partial results in a workspace
 * of the stage, 280 KB to 18 MB, allocated by the first calls that need it and kept; KF_ENOMEM where not even
 * 280 KB can be had, which includes a first call under graph capture.  After any such call every other
 * one can be captured: where the workspace is small, in more launches, to the same bits.
 */
kf_status kf_logits_logprobs(kf_stage* stage, int32_t rows, int32_t vocab, int64_t stride, const float* logits_dev,
                             const int32_t* targets_dev, float* logprob_dev, float* entropy_dev, int32_t n_top,
                             int32_t* top_ids_dev, float* top_logprobs_dev);

/*
 * Per-kernel timing (instrumentation).  The paper's sessions record predicted and
 * measured cost per stage (Section VI); this records, per kernel class, the HIP-event
 * time of every launch the stage enqueues while recording is on.
 *   kf_stage_profile(stage, mask) clears the records and starts recording the classes
 *   whose bit (1 << class) is set in mask; kf_stage_profile(stage, 0) stops recording
 *   (records are kept).  KF_K_ALL records every class.
 *   kf_stage_profile_read waits for the stage's stream, then returns the number of
 *   recorded launches of a class and their summed duration in milliseconds.
 * Each recorded launch is bracketed by two hipEventRecord calls on the stage's
 * stream, which adds a few microseconds per launch to the stream's timeline.
 */
typedef enum {
  KF_K_PREP = 0,       /* kept for numbering: the first layer's launches read the stage input; nothing records here */
  KF_K_QKV = 1,        /* decode: RMSNorm + QKV GEMV + RoPE + KV append */
  KF_K_ATTN = 2,       /* decode: split-KV attention (partials per split) */
  KF_K_OPROJ = 3,      /* decode: merge of the partials + O GEMV + residual */
  KF_K_GATEUP = 4,     /* decode: RMSNorm + gate/up GEMV + SwiGLU */
  KF_K_DOWN = 5,       /* decode: down GEMV + residual */
  KF_K_LMHEAD = 6,     /* head: final RMSNorm + LM-head GEMV + partial argmax */
  KF_K_ARGMAX = 7,     /* head: final argmax reduction */
  KF_K_PF_NORM = 8,    /* prefill: row RMSNorm to fp16 */
  KF_K_PF_QKV = 9,     /* prefill: QKV GEMM (matrix cores) */
  KF_K_PF_ROPE = 10,   /* prefill: RoPE + KV append */
  KF_K_PF_ATTN = 11,   /* prefill: causal flash attention (matrix cores) */
  KF_K_PF_OPROJ = 12,  /* prefill: O GEMM + residual */
  KF_K_PF_GATEUP = 13, /* prefill: gate/up GEMM + SwiGLU */
  KF_K_PF_DOWN = 14,   /* prefill: down GEMM + residual */
  KF_K_PF_STORE = 15,  /* prefill: hidden output store */
  KF_K_QKNORM = 16,    /* kept for numbering: the decode per-head q/k RMSNorm + RoPE of qk_norm blocks
                          now runs inside the attention launch (KF_K_ATTN); nothing records here */
  KF_K_LOGPROB = 17,   /* head: log probabilities of logits */
  KF_K_COUNT = 18
} kf_kernel_class;
#define KF_K_ALL 0x3ffff

kf_status kf_stage_profile(kf_stage* stage, int32_t mask);
kf_status kf_stage_profile_read(kf_stage* stage, int32_t kernel_class, int64_t* launches, double* total_ms);

#ifdef __cplusplus
}
#endif
#endif /* KAFILA_STAGE_H */
