/*
 * flashmesh.h -- C ABI of the speculative decode step of an hourglass mesh transformer
 * (FlashMesh, arXiv 2511.15618), hand-written CUDA for sm_100a, one GPU.
 *
 * The paper states the problem as: given a condition c and the accepted prefix, every
 * forward pass of the backbone yields one main token and the draft modules yield D draft
 * tokens (Sec. 3.1); the drafts may be edited before they are fed back (Sec. 3.2); one
 * forward pass with causal masking verifies main + drafts (Sec. 3.3); the main token and
 * the drafts up to the first mismatch are accepted and decoding continues from the
 * backbone's output at the last accepted token (Sec. 3.3).  The calls below are those
 * stages.  The model is the hourglass of the supplement ("Hourglass Transformer": three
 * coordinates form a vertex, three vertices a face; shortening and upsampling layers with
 * residuals between levels) with a KV cache at each level.
 *
 * Where the paper is silent the model is read as follows: pre-norm RMSNorm blocks, FFN =
 * W2 gelu_erf(W1 x) without biases, rotate-half rotary embedding on the level-local index,
 * conditioning as per-layer prefix keys/values (every layer projects rms(c) with its own K/V
 * matrices; un-rotated, visible to every query, sharing the softmax with the causal keys),
 * shortening = linear on the concatenation of hiddens 3v-2, 3v-1, 3v (zeros below 0), upsampling
 * = linear d -> 3d whose slot r is added to the pre-shorten hidden of position 3v+r,
 * longest-matching-prefix acceptance, masked argmax with ties to the lowest id.
 *
 * Conventions
 *   - Every call returns FM_OK (0) or a negative FM_ERR_* code; nothing throws.  On an error
 *     return no decoding state has been changed, except after FM_ERR_CUDA or FM_ERR_TIMEOUT:
 *     then nothing more is enqueued and the sequences must be started again with fm_prefill
 *     (or the context destroyed).
 *   - Pointers are marked HOST or DEV.  DEV pointers are caller-owned device memory that must
 *     stay valid until the work enqueued by the call has finished on the context's stream.
 *   - fm_draft and fm_verify launch their kernels one by one the first time they see a set of
 *     pointer arguments, capture them into a CUDA graph when the same pointers come again, and
 *     replay that graph afterwards: a host that drives the loop call by call should pass the same
 *     buffers every pass.  (A stream that cannot be captured keeps the plain launches.)
 *   - All calls except fm_create / fm_destroy / fm_generate only enqueue work on the
 *     context's stream and return; fm_generate polls a completion flag and returns when every
 *     sequence has finished.
 *   - The library allocates no device memory: the caller hands a workspace of
 *     fm_workspace_bytes() bytes to fm_create, which carves weights (bfloat16), KV caches and
 *     scratch out of it.  (fm_create allocates a few hundred bytes of pinned host memory.)
 *   - Indexing: inputs u_0 = BOS, u_i = t_{i-1}; the row at position i predicts mesh token
 *     t_i.  L = inputs consumed so far; the pending main token is t_{L-1}.  A verify pass
 *     feeds positions L..L+D; accepting a tokens moves L to L+a.
 *   - Lossless by construction (Sec. 3.3): within one context the logits of a position do not
 *     depend on the row of the pass it is fed in, on the other rows or sequences of the pass,
 *     nor on the accept lengths of the passes before it, to the last bit (reduction orders are
 *     fixed by slot and column index; every value that can be produced at two places of the code
 *     is rounded explicitly), so the tokens a speculative run emits are those of one-token-per-
 *     pass decoding with the same context, whatever the drafts were.  Two contexts (another
 *     batch size, draft count or capacity) may group reductions differently.
 *   - This is a statement about passes behind one prefill.  A prefill packs all prompts of the call
 *     into launches whose forms and tiles follow the prompt lengths of all sequences: the same call
 *     leaves the same bits, but a sequence prefilled in other company, or a prompt and the same
 *     tokens decoded in passes, agree to rounding only (tokens may then differ where two are all but
 *     tied).  To continue a run to the bit, repeat its prefill and feed the tokens it had emitted as
 *     drafts (fm_generate with a teacher, or cand of fm_verify) instead of a longer prompt.
 *   - Token ids: [0, n_bins) coordinate bins, BOS = n_bins, EOS = n_bins+1, PAD = n_bins+2.
 *     Emitted ids are always coordinate bins, or EOS at a face boundary when allow_eos != 0;
 *     ties in an argmax go to the lowest id.
 */
#ifndef FLASHMESH_H
#define FLASHMESH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FM_OK                0
#define FM_ERR_INVALID_ARG  -1   /* null pointer, size out of range, inconsistent config      */
#define FM_ERR_BAD_STATE    -2   /* call out of order (e.g. fm_verify before fm_prefill)       */
#define FM_ERR_CAPACITY     -3   /* batch > max_batch, prompt or run longer than max_tokens    */
#define FM_ERR_CUDA         -4   /* a CUDA runtime call failed                                 */
#define FM_ERR_TIMEOUT      -5   /* a bounded device-side wait gave up (see fm_device_status)  */
#define FM_ERR_UNSUPPORTED  -6   /* shape outside what the kernels were built for              */

#define FM_MAX_FACE_HEADS 4
#define FM_MAX_DRAFT      27

typedef struct fm_ctx fm_ctx;    /* opaque; owns nothing but pinned host flags */

/* Model and capacity description (the hourglass of the supplement, read as stated above). */
typedef struct fm_config {
  int32_t d_model, n_heads, n_kv_heads, head_dim, d_ff;
  int32_t layers[5];          /* coord_down, vertex_down, face, vertex_up, coord_up          */
  int32_t n_bins;             /* vocabulary = n_bins + 3                                     */
  int32_t n_prefix;           /* P conditioning vectors, held as prefix keys/values          */
  int32_t window[3];          /* attention window per level (coordinate, vertex, face); 0 = full */
  int32_t draft_len;          /* D, 0..FM_MAX_DRAFT                                          */
  int32_t max_batch;
  int32_t max_tokens;         /* capacity per sequence in coordinate positions (inputs)      */
  float   rope_theta;         /* 0 = no positional encoding                                  */
  float   norm_eps;
  int32_t allow_eos;          /* 0: EOS is masked everywhere (fixed-length runs)             */
  /* draft modules (Sec. 3.1; supplement "Three-Level Speculative Decoding") */
  int32_t draft_heads;        /* FM_HEADS_REDUCED: SP = h + A rms(h), HF = the upsample matrices alone;
                                 FM_HEADS_FULL: SP-Blocks with attention (Eq. 1), an HF-Block after
                                 every upsample (Eq. 2-5)                                     */
  int32_t draft_levels;       /* FM_LEVELS_THREE: 2 coordinate heads + point level + face level;
                                 FM_LEVELS_COORD: D coordinate heads, no point / face level (the
                                 supplement's ablation on multi-level decoding)               */
  int32_t hf_ff;              /* hidden width of the HF-Blocks' feed-forward networks (0 = d_model;
                                 a multiple of 64)                                            */
  int32_t avg_levels;         /* 1: where several levels predict a position their softmax
                                 distributions are averaged (supplement, "Integrating the three
                                 levels"); 0: one source per position ("Optimizations")       */
} fm_config;
#define FM_HEADS_REDUCED 0
#define FM_HEADS_FULL    1
#define FM_LEVELS_THREE  0
#define FM_LEVELS_COORD  1

/* HOST pointers to float32 matrices, row-major [out, in]; values are rounded to bfloat16
 * (nearest-even) when fm_create copies them.  Gains stay float32. */
typedef struct fm_layer_weights {
  const float* g1;            /* [d]                          RMSNorm gain before attention   */
  const float* Wqkv;          /* [(H + 2*Hkv)*dh, d]          rows: Q heads, K heads, V heads */
  const float* Wo;            /* [d, H*dh]                                                    */
  const float* g2;            /* [d]                          RMSNorm gain before the FFN     */
  const float* W1;            /* [d_ff, d]                                                    */
  const float* W2;            /* [d, d_ff]                                                    */
} fm_layer_weights;

/* One SP-Block head (Eq. 1).  Reduced: y = h + A rms(h, g).  Full: the attention of the block reads
 * the cache of the backbone's last layer at the head's level (keys / values of the split-node hiddens;
 * conditioning as the prefix entries of the same softmax) with the head's own query and output
 * matrices: u = h + Wo Attn(Wq rms(h, ga)), y = h + A rms(u, g).  ga / Wq / Wo are read only with
 * FM_HEADS_FULL. */
typedef struct fm_sp_weights {
  const float* g;  const float* A;        /* [d], [d, d]                                       */
  const float* ga; const float* Wq; const float* Wo;   /* [d], [H*dh, d], [d, H*dh]            */
} fm_sp_weights;

/* One HF-Block (Eq. 3-5) for one offset: x + W2 gelu(W1 Attn(Wq rms(x, g), K, V)) with K, V the cache
 * of the backbone's last layer at the block's level, entries up to the last accepted position. */
typedef struct fm_hf_weights {
  const float* g; const float* Wq; const float* W1; const float* W2;   /* [d], [H*dh, d], [hf, H*dh], [d, hf] */
} fm_hf_weights;

typedef struct fm_weights {
  const float* E;                         /* [V, d] token embedding                          */
  const fm_layer_weights* stack[5];       /* stack[s][l], l < layers[s]                      */
  const float* S_cv;                      /* [d, 3d] shorten coordinate -> vertex            */
  const float* S_vf;                      /* [d, 3d] shorten vertex -> face                  */
  const float* U_fv;                      /* [3d, d] upsample face -> 3 vertices             */
  const float* U_vc;                      /* [3d, d] upsample vertex -> 3 coordinates        */
  const float* g_out;                     /* [d]                                              */
  const float* W_out;                     /* [V, d]                                           */
  /* Draft modules.  heads_c: coordinate heads (2, or D with FM_LEVELS_COORD); heads_v: 2 point-level
   * heads (vertex v*+1, v*+2); heads_f: face-level heads, head e (1-based) drafts the face e-1 after
   * the one that holds the pending token; D < 7 uses 1 head, otherwise (D+8)/9 + 1.  heads_v,
   * heads_f and the HF-Blocks are not read with FM_LEVELS_COORD. */
  const fm_sp_weights* heads_c;
  const fm_sp_weights* heads_v;
  const fm_sp_weights* heads_f;
  /* HF-Blocks (FM_HEADS_FULL only): hf_vc[6] refine the point level's coordinate features (offset
   * 3..8 from the vertex row), hf_fv[3*Ef] the face level's vertex features, hf_fc[9*Ef] the face
   * level's coordinate features. */
  const fm_hf_weights* hf_vc;
  const fm_hf_weights* hf_fv;
  const fm_hf_weights* hf_fc;
  /* label head of the correction stage (Sec. 3.2): gain [d] and matrix [3, d]; may be NULL (then
   * fm_draft produces no labels) */
  const float* label_g;
  const float* label_W;
} fm_weights;

/* Optional device-side draft editor for fm_generate: the place where the paper's Correct
 * stage sits (Sec. 3.2 edits drafts only, never the main token).  Used by the benchmark to
 * pin the true acceptance length: draft j (1..keep) is replaced by the known continuation,
 * draft keep+1 by a deliberately different coordinate id. */
typedef struct fm_teacher {
  const int32_t* truth;       /* DEV [batch, truth_stride]: mesh tokens t_0.. (prompt included) */
  int32_t truth_stride;
  const int32_t* keep;        /* DEV [n_sched, batch]: correct drafts wanted per step, 0..D  */
  int32_t n_sched;            /* the schedule wraps around                                   */
} fm_teacher;

typedef struct fm_stats {
  int64_t steps;                          /* passes of the loop: exactly max_steps, or, without it,
                                             counted in groups of eight, the last one whole (its
                                             passes behind the end are not run)              */
  int64_t emitted;                        /* mesh tokens emitted, all sequences              */
  int64_t accept_hist[FM_MAX_DRAFT + 2];  /* accept_hist[a] = passes in which a running sequence
                                             accepted a tokens, all sequences: the mean accept
                                             length is emitted / sum(accept_hist)            */
  float   ms;                             /* device time of the decode loop (CUDA events)    */
} fm_stats;

/* Bytes of device workspace fm_create needs for this configuration (0 if it is invalid). */
size_t fm_workspace_bytes(const fm_config* cfg /*HOST*/);

/* Build a context inside `dev_workspace` (DEV, 256-byte aligned, >= fm_workspace_bytes):
 * copies and rounds the weights, zeroes state.  `cuda_stream` is a cudaStream_t (NULL = the
 * default stream); all later work of this context runs on it.  Synchronous.
 * Errors: INVALID_ARG (null, bad config), CAPACITY (workspace too small), UNSUPPORTED
 * (d_model or d_ff not a multiple of 64, n_heads*head_dim not a multiple of 128, head_dim not
 * 64/128, a stack without layers, D > FM_MAX_DRAFT, hf_ff not a multiple of 64), CUDA. */
int fm_create(const fm_config* cfg /*HOST*/, const fm_weights* w /*HOST*/, void* dev_workspace /*DEV*/,
              size_t workspace_bytes, void* cuda_stream, fm_ctx** out /*HOST*/);
int fm_destroy(fm_ctx* ctx);

/* Start `batch` sequences.  cond: DEV float32 [batch, P, d] conditioning vectors, projected by
 * every layer's own K/V matrices into prefix cache slots.  prompt: DEV int32, the sequences'
 * mesh tokens concatenated; prompt_off: HOST int32 [batch+1] offsets into it (lengths must be
 * multiples of 9).  Runs BOS + prompt of all sequences as one packed multi-row forward, in chunks
 * of up to 8192 rows.
 * Afterwards L[b] = 1 + prompt_len[b] and the first main token is pending.
 * Errors: INVALID_ARG, CAPACITY. */
int fm_prefill(fm_ctx* ctx, int32_t batch, const float* cond /*DEV*/, const int32_t* prompt /*DEV*/,
               const int32_t* prompt_off /*HOST*/);

/* Per-sequence limit: sequence b stops once 9*max_faces[b] tokens have been emitted after
 * its prompt (or at EOS).  HOST int32 [batch].  Default: the cache capacity. */
int fm_set_max_faces(fm_ctx* ctx, const int32_t* max_faces /*HOST*/);

/* Predict (Sec. 3.1, supplement "Three-Level Speculative Decoding"): run the draft modules
 * (reduced heads, or the full SP-Blocks and HF-Blocks; fm_config.draft_heads / draft_levels) on
 * the split-node hiddens stashed at the last accepted position; with a label head, also the
 * labels of the drafted points (fm_draft_labels).  cand: DEV int32 out
 * [batch, D+1] = pending main token, then D drafts (PAD for finished sequences).
 * draft_logits: DEV float32 out [batch, D, V] or NULL.  draft_margin: DEV float32 out
 * [batch, D] (top-1 minus top-2 of the masked draft logits) or NULL. */
int fm_draft(fm_ctx* ctx, int32_t* cand /*DEV*/, float* draft_logits /*DEV*/, float* draft_margin /*DEV*/);

/* Correct (Sec. 3.2 "Correction Mechanism"): edit the drafts of a candidate row in place, between
 * fm_draft and fm_verify.  A point is a vertex whose three coordinate tokens (z, y, x) are all
 * drafts of this pass (slot s of sequence b holds mesh token L[b] - 1 + s; slot 0 is the main
 * token and is never touched; vertices that are only partly in the row, or that hold a token that
 * is not a coordinate bin, are left alone).  labels: DEV int32 [batch, D+1]; labels[b][s] is the
 * label of the point that starts at slot s: FM_LABEL_HISTORICAL, FM_LABEL_NEW or FM_LABEL_INTRA
 * (other slots are not read; fm_draft_labels gives the labels of the library's own label head).
 * In sequence order, every FM_LABEL_INTRA point that has no identical point in the row is
 * replaced by the nearest (squared distance between bin indices, ties to the earliest) earlier
 * FM_LABEL_NEW point of another face, if there is one; then the points of every face are sorted
 * ascending by (z, y, x) among the slots they occupy.  Only rows the next pass feeds
 * (the first nrow slots of an unfinished sequence) are considered.
 * cand: DEV int32 in/out [batch, D+1].  Errors: INVALID_ARG (null pointer), BAD_STATE (before
 * fm_prefill), UNSUPPORTED (more than 48 slots per row; cannot happen while FM_MAX_DRAFT is 27). */
#define FM_LABEL_HISTORICAL 0
#define FM_LABEL_NEW 1
#define FM_LABEL_INTRA 2
int fm_correct(fm_ctx* ctx, int32_t* cand /*DEV*/, const int32_t* labels /*DEV*/);

/* Labels of the drafted points (Sec. 3.2: a label head, a linear layer, on every point-level
 * feature), as computed by the last fm_draft: labels[b][s] in {FM_LABEL_HISTORICAL, FM_LABEL_NEW,
 * FM_LABEL_INTRA} where a vertex made of drafts only starts at slot s, -1 elsewhere; the label is
 * the argmax (ties to the lowest) of label_W rms(f, label_g) over the point-level feature f in the
 * pipeline of the head that drafts the point's last coordinate.  margin: top-1 minus top-2, or NULL.
 * DEV out [batch, D+1].  Errors: UNSUPPORTED without a label head or with FM_LEVELS_COORD. */
int fm_draft_labels(fm_ctx* ctx, int32_t* labels /*DEV*/, float* margin /*DEV*/);

/* fm_correct with two options: labels == NULL takes the label head's labels of the last fm_draft;
 * use_history != 0 also enforces the historical label against the accepted tokens: a point labelled
 * FM_LABEL_HISTORICAL that equals no complete accepted vertex of the face that holds the pending
 * token or of the face before it is replaced by the nearest of them (same distance, ties to the
 * earliest); historical points are handled first, in sequence order. */
int fm_correct_ex(fm_ctx* ctx, int32_t* cand /*DEV*/, const int32_t* labels /*DEV or NULL*/, int32_t use_history);

/* Verify (Sec. 3.3): one forward pass over main + D candidates, causal among themselves,
 * through all five level stacks.  cand: DEV int32 in [batch, D+1]; cand[b][0] must be the
 * pending main token.  Rows fed per sequence = min(D+1, tokens left).  argmax: DEV int32 out
 * [batch, D+1] (masked argmax per row, -1 for rows not fed) or NULL; logits: DEV float32 out
 * [batch, D+1, V] or NULL; margin: DEV float32 out [batch, D+1] or NULL.
 * Writes keys/values beyond L (invisible until accepted); does not move L; calling it twice
 * is legal and gives the same result. */
int fm_verify(fm_ctx* ctx, const int32_t* cand /*DEV*/, int32_t* argmax /*DEV*/, float* logits /*DEV*/,
              float* margin /*DEV*/);

/* fm_verify for callers that cannot provide scratch memory of their own (no counterpart in the
 * paper).  Some hosts of this library carve the workspace of fm_create out of an arena that is
 * sized and committed once at start-up -- a serving process with a fixed memory plan, a plug-in that
 * is forbidden to call cudaMalloc because an allocation would synchronise the device under its
 * real-time loop -- and want the attention kernel's split-KV scratch (per-group partial results) kept
 * out of that arena.  This call does what fm_verify
 * does, same arguments, same results, but points the attention kernel at a fixed array of
 * FM_STATIC_SCRATCH_BYTES bytes that is part of the library image: every GPU that loads the library
 * holds that many bytes until the process exits.  It allocates nothing (no cudaMalloc, no
 * cudaFree, no allocating library routine); inputs and outputs are still the caller's.
 *   - Limit: the scratch one pass needs (it grows with max_batch * n_kv_heads and with the cache
 *     capacity) must fit in FM_STATIC_SCRATCH_BYTES, else FM_ERR_CAPACITY is returned and nothing
 *     is enqueued.
 *   - Every GPU has its own copy of the array: the device the context was created on must be the
 *     current device at every call (FM_ERR_BAD_STATE otherwise).  The first call on a device looks
 *     up the array's device address; make that first call before any stream capture is begun.
 *   - All contexts and all calls share the one array.  Two calls whose kernels overlap on
 *     the GPU -- different streams, different contexts -- race on it: serialise them. */
#define FM_STATIC_SCRATCH_BYTES (4 * 1024 * 1024)
int fm_verify_static_scratch(fm_ctx* ctx, const int32_t* cand /*DEV*/, int32_t* argmax /*DEV*/, float* logits /*DEV*/,
                             float* margin /*DEV*/);

/* Accept (Sec. 3.3) and roll back: a = 1 + number of leading drafts that equal the backbone's
 * argmax at the previous row; clipped to the rows fed and at an accepted EOS; L += a; the next
 * main token is the argmax at row a-1.  force_tok: DEV int32 [batch, D+1] or NULL, replaces the
 * stored argmax; force_len: DEV int32 [batch] or NULL, replaces a (values 1..D+1).
 * n_acc: DEV int32 out [batch]; emitted: DEV int32 out [batch, D+1] (accepted ids, then -1);
 * kv_len: DEV int32 out [batch, 3] = (L, ceil(L/3), ceil(L/9)).  Any output may be NULL.
 * Errors: BAD_STATE if no fm_verify preceded it. */
int fm_accept(fm_ctx* ctx, const int32_t* force_len /*DEV*/, const int32_t* force_tok /*DEV*/,
              int32_t* n_acc /*DEV*/, int32_t* emitted /*DEV*/, int32_t* kv_len /*DEV*/);

/* Verify a tree of candidates instead of one chain: several alternatives per position, for instance the top
 * alternatives of the draft distributions (fm_logprobs on fm_draft's logits).  tokens, parent: DEV
 * int32 [batch, nodes], nodes <= D+1.  Node 0 of a sequence is the pending main token (parent -1); another node continues
 * the earlier node of its sequence that parent names; a node whose parent is none, or deeper than the rows a pass
 * would feed, is not in use.  A node at depth k stands for position L + k and sees the accepted positions and its
 * ancestors, through all level stacks (fm_tree_attention over the context's caches).  predicted: DEV
 * int32 out [batch, nodes] (masked argmax, -1 where not in use) or NULL; logits: DEV float32 out
 * [batch, nodes, V] or NULL; margin: DEV float32 out [batch, nodes] or NULL.  Changes no cache entry and
 * does not move L; calling it twice is legal.  Its projections run in the tiled form, as a prefill's: a chain verified as a tree
 * agrees with fm_verify to rounding, not to the bit (see the statement on lossless decoding above).
 * Errors: INVALID_ARG, BAD_STATE (before fm_prefill), CAPACITY (nodes > D+1, batch > FM_MAX_TREES, or more rows than a prefill chunk's faces). */
int fm_verify_tree(fm_ctx* ctx, const int32_t* tokens /*DEV*/, const int32_t* parent /*DEV*/, int32_t nodes, int32_t* predicted /*DEV*/,
                   float* logits /*DEV*/, float* margin /*DEV*/);

/* Accept the longest confirmed path of the tree (fm_tree_accept on the predictions; it ends at an accepted EOS) and move its keys,
 * values and carried hiddens into the caches; L += its length; the next main token is the prediction at its last node.
 * force_pred: DEV int32 [batch, nodes] or NULL, replaces the stored predictions.  path: DEV int32 out
 * [batch, nodes], node indices, then -1; emitted: DEV int32 out [batch, nodes], their tokens, then -1; n_acc, kv_len as
 * in fm_accept.  Any output may be NULL.  Errors: BAD_STATE if no fm_verify_tree preceded it. */
int fm_accept_tree(fm_ctx* ctx, const int32_t* force_pred /*DEV*/, int32_t* path /*DEV*/, int32_t* n_acc /*DEV*/, int32_t* emitted /*DEV*/,
                   int32_t* kv_len /*DEV*/);

/* One pass of the loop for a host that sits in it (Sec. 3: predict, edit, verify, accept), with HOST
 * buffers: runs the draft modules; copies `cand` in (HOST int32 [batch, D+1], pinned memory makes
 * the copy asynchronous; an entry >= 0 replaces the draft modules' candidate at that slot, an entry
 * < 0 keeps it, slot 0 always stays the pending main token; NULL keeps all); verifies; accepts;
 * copies n_acc [batch], emitted [batch, D+1] (may be NULL) and kv_len [batch, 3] (may be NULL) back to
 * HOST memory and waits for the stream.  Equivalent to fm_draft, fm_verify, fm_accept with the
 * copies in between, in one call.  Errors as those calls. */
int fm_step_host(fm_ctx* ctx, const int32_t* cand /*HOST*/, int32_t* n_acc /*HOST*/, int32_t* emitted /*HOST*/,
                 int32_t* kv_len /*HOST*/);

/* The whole loop (Sec. 3): draft -> (optional teacher edit) -> verify -> accept, until every
 * sequence has emitted 9*max_faces tokens or EOS, or, when max_steps > 0, for exactly max_steps
 * passes (a later call continues where this one stopped).  out_tok: DEV int32 [batch, out_stride]
 * receives the emitted tokens (prompt not included), out_len: DEV int32 [batch], zeroed by the
 * first call after fm_prefill and advanced by every call; both may be NULL.  teacher and stats may
 * be NULL.  plain != 0 accepts only the main token every pass (the one-token-at-a-time baseline
 * on the same kernels).  max_faces == -1 keeps the per-sequence limits set with fm_set_max_faces
 * (tokens beyond out_stride are then not stored).  Synchronous (returns after the last pass).
 * Errors: BAD_STATE, CAPACITY (prompt + 9*max_faces + D + 2 > max_tokens, or out_stride too small). */
int fm_generate(fm_ctx* ctx, int32_t max_faces, int32_t* out_tok /*DEV*/, int32_t out_stride,
                int32_t* out_len /*DEV*/, const fm_teacher* teacher /*HOST struct, DEV arrays*/,
                int32_t plain, int64_t max_steps, fm_stats* stats /*HOST*/);

/* Algorithmic bytes one verify pass must move for the given per-sequence lengths (weights of
 * the stacks that have rows, shorten/upsample, output matrix, K and V entries visible to the
 * rows); kv_len HOST int32 [batch,3] as returned by fm_accept.  For roofline reports. */
double fm_verify_bytes(const fm_ctx* ctx, int32_t batch, const int32_t* kv_len /*HOST*/);

/* Per-kernel-class device timing for roofline reports (no counterpart in the paper).  Between
 * fm_profile_begin and fm_profile_end every weight-streaming GEMM launch and every attention
 * launch is bracketed by a CUDA event pair on the context's stream; fm_profile_end synchronises
 * and sums them.  gemm_bytes counts each launch's weight matrix once (2*M*K bytes). */
typedef struct fm_profile {
  double gemm_ms, gemm_bytes; int64_t gemm_launches;
  double attn_ms; int64_t attn_launches;
} fm_profile;
int fm_profile_begin(fm_ctx* ctx);
/* One kernel class timed alone (no counterpart in the paper): the launches of that class of one
 * verify pass over the current candidates and lengths (cls 0: the weight-streaming GEMMs, 1: the
 * attention launches; same kernels, arguments and data as in the pass) are captured as a CUDA graph
 * and replayed `reps` times after 3 warm-up replays, between two events.  out->gemm_ms /
 * out->attn_ms = milliseconds per replay, *_launches = launches per replay, gemm_bytes = weight bytes
 * per replay (2*M*K per launch).  Synchronous.  The
 * replays overwrite activations and the tentative cache rows of the pass: call fm_prefill (or
 * fm_verify) again before decoding on. */
int fm_profile_class(fm_ctx* ctx, int32_t cls, int32_t reps, fm_profile* out /*HOST*/);
int fm_profile_end(fm_ctx* ctx, fm_profile* out /*HOST*/);

/* How the attention kernel cuts a level's cache (no counterpart in the paper; for reports and
 * tests): slots per chunk, chunks per group (one CTA streams one group; fixed when the context is
 * created) and the number of groups the full cache has.  Chunk c belongs to group c mod groups, so a
 * (sequence, kv-head) whose cache holds n slots, prefix included, is read by
 * min(ceil(n / chunk), groups) CTAs, whose partial results go through the scratch buffer when there
 * is more than one.  level: 0 coordinate, 1 vertex, 2 face.  HOST out pointers, any may be NULL. */
int fm_attention_layout(const fm_ctx* ctx, int32_t level, int32_t* chunk_slots, int32_t* chunks_per_group,
                        int32_t* max_groups);

/* The form in which a projection of the model runs on `rows` rows of a level (no counterpart in the paper; for reports and
 * tests): FM_FORM_* for an FM_PROJ_* of the backbone, decided as the library does on a device of 148 SMs without the
 * environment switches.  (The QKV projection of a layer whose inputs the draft heads read, the last one of an up-stack or of the
 * face stack, takes the split-K form where the others are tiled, in decode passes.)  HOST only, needs no device.  Negative: error. */
#define FM_PROJ_QKV 0
#define FM_PROJ_OUT 1
#define FM_PROJ_FFN1 2
#define FM_PROJ_FFN2 3
#define FM_PROJ_LOGITS 4
#define FM_PROJ_CONDITIONING 5     /* keys and values of the prefix, all layers in one launch; rows: conditioning vectors of all sequences */
#define FM_FORM_FEW_ROWS 0
#define FM_FORM_SPLIT_K 1
#define FM_FORM_TILED 2
#define FM_FORM_TILED_PAIRS 3
int fm_projection_form(const fm_config* cfg, int32_t projection, int32_t rows);

/* Number of kernels launched by this context since creation (for launch accounting). */
int64_t fm_launch_count(const fm_ctx* ctx);

/* Self-check of the give-up path of the device-side waits (no counterpart in the paper).  Every
 * wait inside the kernels (on a shared-memory barrier that a copy, a tensor-core commit or a peer
 * CTA completes) polls for a bounded number of clock cycles, then records FM_ERR_TIMEOUT in the
 * device status word and lets the kernel finish without touching the data.  This call enqueues one
 * thread that runs the same wait, limited to `limit_cycles` (1 .. 1e8), on a barrier that nothing
 * completes: afterwards fm_device_status returns FM_ERR_TIMEOUT, and fm_prefill clears it.  The
 * kernel always ends by itself. */
int fm_selftest_wait_timeout(fm_ctx* ctx, int64_t limit_cycles);

const char* fm_strerror(int code);
/* Device status word: 0, or FM_ERR_TIMEOUT if a bounded wait inside a kernel gave up, or
 * FM_ERR_INVALID_ARG if a kernel met an out-of-range token id (it then used PAD).  The word is
 * cleared by fm_prefill.  Synchronises the stream. */
int fm_device_status(fm_ctx* ctx);

/* ------------------------------------------------------------------------------------------
 * Trees of drafts over a paged cache
 *
 * The stages above verify one chain of candidates over caches that a context owns.  The calls below
 * serve hosts that verify a tree of alternatives instead (several drafts per position, taken from
 * the top alternatives of the draft distributions) and share cached prefixes between sequences: they
 * work on the caller's own buffers and need no context.
 *   fm_logprobs          log probabilities of given tokens, entropy, rank, top alternatives
 *   fm_tree_attention    attention of a tree's nodes over a paged cache and their ancestors
 *   fm_tree_accept       the longest path of the tree that the predictions confirm
 *   fm_pages_*           pages for new positions, appended rows, forks, roll-back, compaction
 *
 * Conventions beside those at the top
 *   - All of them only enqueue work on `stream` (a cudaStream_t; NULL = the default stream), allocate
 *     nothing, never wait and can be captured into a graph.  The device that holds the buffers has to
 *     be the current one.  What the host can check is checked before anything is enqueued; an error
 *     return has enqueued nothing.
 *   - What only the device sees (an id out of range, an exhausted pool) never leads to an access out
 *     of bounds: the entry concerned is left as it was and, where a call has a status word, the error
 *     is recorded there (DEV int32, 0 = none; of several the lowest code stays; the caller clears it).
 *     Row offsets (row_off) ascend and stay inside the rows that the caller has.  Where a call is told how
 *     many those are (n_rows; the Python calls always tell), an entry whose offsets do not is one without rows, INVALID_ARG where
 *     there is a status word; where not, they are taken at their word, like the sizes of buffers.
 *   - A kernel enqueued behind these calls with programmatic stream serialization (its blocks may start
 *     before they end) has to wait for them with griddepcontrol.wait before it touches their buffers.
 *   - A call may be enqueued while earlier ones on the same buffers run on the same stream.  Calls on
 *     the same fm_pages, or with the same workspace, from two streams (or two graphs that may run at
 *     the same time) have to be ordered by the caller.
 *   - These are forms for serving: there is no backward pass.
 *   - Results depend on the arguments alone, to the last bit: the same call gives the same bits.  The
 *     attention of a sequence in other company agrees to rounding (the split of the work follows all lengths).
 * ------------------------------------------------------------------------------------------ */
#define FM_BF16 0
#define FM_FP16 1
#define FM_FP32 2

#define FM_MAX_TOP 32               /* alternatives per row of fm_logprobs                          */
#define FM_MAX_TREE_NODES 256       /* nodes of one tree                                            */
#define FM_MAX_SEQS 4096            /* sequences of one fm_pages, entries of one of its calls (of fm_pages_reserve and fm_pages_append
                                     * as many as it has sequences: INVALID_ARG beyond) */
#define FM_MAX_TREES 512            /* trees of one fm_tree_attention                               */
#define FM_FILL_OUT 1
#define FM_FILL_LSE 2

/* A pool of cache pages: element i of the key of position `slot` of page `page`, head h, layer l is
 * k[l*layer_stride + page*page_stride + h*head_stride + slot*slot_stride + i]; values alike.  Strides
 * in elements, multiples of 8; k and v 16-byte aligned.  The same page ids serve every layer.  Errors of all calls: INVALID_ARG (size,
 * stride, alignment), UNSUPPORTED (dtype), CAPACITY (more than 32766 layers, or than 2^30 pieces of 16 bytes in a page of a layer). */
typedef struct fm_cache {
  void* k; void* v;                 /* DEV                                                          */
  int64_t layer_stride, page_stride, head_stride, slot_stride;
  int32_t n_layers, n_pages, page_slots, n_kv_heads, head_dim;
  int32_t dtype;                    /* FM_BF16 or FM_FP16                                           */
} fm_cache;

/* Which pages belong to which sequence.  All arrays DEV int32, owned by the caller; the calls keep
 * refs[p] = number of table entries that hold page p.  The entries of a sequence are filled from the
 * front; positions 0 .. lens-1 hold keys and values, entries behind them may be reserved already. */
typedef struct fm_pages {
  int32_t n_pages, page_slots, max_seqs, max_pages;
  int32_t* table;                   /* [max_seqs, max_pages] page ids, -1 = none                    */
  int32_t* lens;                    /* [max_seqs]                                                   */
  int32_t* refs;                    /* [n_pages] holders of every page, 0 = free                    */
  int32_t* status;                  /* [1]                                                          */
  int32_t* work;                    /* [fm_pages_work_ints()] scratch, zeroed once (fm_pages_reset) */
} fm_pages;
size_t fm_pages_work_ints(int32_t n_pages, int32_t max_seqs);      /* 0 if a size is out of range */

/* All pages free, all lengths zero; clears status and work. */
int fm_pages_reset(const fm_pages* pages, void* stream);

/* dst[i] becomes a copy of src[i], i < n: it gives up its own pages and holds those of src[i] that
 * have positions, shared (pages reserved ahead are not shared).  Nothing is copied until one of them grows
 * (fm_pages_reserve).  Entries with a negative src or dst are skipped.  INVALID_ARG in the status
 * word, and the entry skipped: an id >= max_seqs, a dst that an earlier entry has too, a src that is
 * a dst of the same call. */
int fm_pages_fork(const fm_pages* pages, const int32_t* src /*DEV*/, const int32_t* dst /*DEV*/, int32_t n, void* stream);

/* Pages for grow[i] more positions of sequence seqs[i]: afterwards the table covers lens + grow
 * positions, and the page of the next position is the sequence's own: when it is partly filled and shared, its filled
 * part is copied to a fresh page, in every layer (the last of several holders in one call keeps it).
 * Free pages are handed out lowest id first, in the order of the entries, inside an entry in the
 * order of the positions.  An entry that cannot have all its pages (too few free, or behind
 * max_pages) gets none: CAPACITY in the status word; those behind it are still served.  Negative
 * seqs are skipped; an id >= max_seqs or listed before: INVALID_ARG, skipped.  Copied pages are read whole up to the length. */
int fm_pages_reserve(const fm_pages* pages, const fm_cache* cache, const int32_t* seqs /*DEV*/, const int32_t* grow /*DEV*/, int32_t n,
                     void* stream);

/* Write new keys and values behind the cache of the listed sequences and advance their lengths.
 * Sequence seqs[i] owns the rows row_off[i] .. row_off[i+1]-1 of k_new / v_new (element j of head h
 * of row r, layer l: k_new[l*new_layer_stride + r*new_row_stride + h*new_head_stride + j]; strides multiples of 8, 16-byte aligned).
 * path == NULL: all its rows, in order.  Otherwise rows path[i*path_stride + 0 .. n_acc[i]-1],
 * counted from row_off[i] (an accepted path of a tree).  max_rows: bound on the rows one sequence
 * appends (HOST; beyond 2^30 pieces of 16 bytes in a layer it is lowered to that).  An entry whose pages are not all there, or are shared (no fm_pages_reserve), with a
 * row outside its own or the n_rows that there are, or more rows than max_rows is skipped: BAD_STATE or INVALID_ARG in the status
 * word; its length stays.  Ids as in fm_pages_reserve. */
typedef struct fm_new_rows {
  const void* k; const void* v;     /* DEV, the type of the cache                                   */
  int64_t layer_stride, row_stride, head_stride;
  int32_t n_rows;                   /* rows of k and v, or 0: not said                              */
} fm_new_rows;
int fm_pages_append(const fm_pages* pages, const fm_cache* cache, const fm_new_rows* rows, const int32_t* seqs /*DEV*/,
                    const int32_t* row_off /*DEV [n+1]*/, const int32_t* path /*DEV or NULL*/, int32_t path_stride,
                    const int32_t* n_acc /*DEV [n], with path*/, int32_t n, int32_t max_rows, void* stream);

/* Cut sequence seqs[i] to min(lens, max(new_lens[i], 0)) positions and give back every page behind them, those
 * reserved ahead included (0: the sequence is empty).  Ids as in fm_pages_reserve. */
int fm_pages_truncate(const fm_pages* pages, const int32_t* seqs /*DEV*/, const int32_t* new_lens /*DEV*/, int32_t n, void* stream);

/* Move the pages in use to the front of the pool: with U pages in use the k-th lowest used page with an id
 * >= U moves to the k-th lowest free id, in every layer; table and refs follow.  used: DEV out [1] U, or NULL. */
int fm_pages_compact(const fm_pages* pages, const fm_cache* cache, int32_t* used /*DEV*/, void* stream);

/* Attention of trees of drafted tokens (one node: a single token).  The nodes of sequence i are rows
 * row_off[i] .. row_off[i+1]-1 of q, k_new and v_new, with parent[row] the node it continues, counted
 * from row_off[i]: an earlier node, or -1 for a node that continues the cached positions.  With
 * len = lens[seq], depth(i) the number of a node's ancestors and position len + depth(i):
 *   a node sees itself and its ancestors, and the cached positions s < len;
 *   window > 0: of both only what lies less than `window` positions before it, and always the
 *   positions s < n_prefix (conditioning).
 * out = sum p v, p = softmax(scale q k), sums and softmax in 32 bits (p is rounded to the cache's type for its
 * product with v; in half precision what is below 2^-34 of the row's largest p rounds to nothing there); lse = log sum exp(scale q k).
 * A parent that is no earlier node and not -1 takes its node and every node below it out of use:
 * out 0, lse -inf; nobody sees them.  Values of positions and nodes that a row does not see have no
 * effect on it, whatever they hold.  Positions behind the table or max_len are not seen.  A tree of more
 * than max_nodes nodes: CAPACITY in the status word, and the nodes behind take no part.  Offsets that are not inside the n_rows
 * rows: INVALID_ARG there.  Rows of such nodes, and those in front of row_off[0] and
 * behind row_off[n], are left as they were, or get what `fill` says.
 * Nothing is appended to the cache.  out may be q; it shares no memory with k_new, v_new or the cache.  max_nodes and max_len also
 * choose between two kernels, for passes of few rows and of many: both are right at any size, bounds far above the
 * sizes cost time.  Errors: INVALID_ARG (null pointer, size, stride or alignment),
 * UNSUPPORTED (head_dim not 64 / 128, dtype), CAPACITY (workspace, batch > FM_MAX_TREES, max_nodes > FM_MAX_TREE_NODES). */
typedef struct fm_tree_args {
  const void* q;                    /* DEV [rows, n_heads, head_dim], rows q_row_stride apart        */
  const void* k_new; const void* v_new;   /* DEV [rows, n_kv_heads, head_dim], rows new_row_stride apart */
  void* out;                        /* DEV [rows, n_heads, head_dim], rows out_row_stride apart      */
  float* lse;                       /* DEV [rows, n_heads] or NULL                                   */
  int64_t q_row_stride, new_row_stride, out_row_stride;   /* elements, multiples of 8; buffers 16-byte aligned */
  const int32_t* table;             /* DEV [.., max_pages] as in fm_pages                            */
  const int32_t* lens;              /* DEV                                                           */
  const int32_t* seqs;              /* DEV [batch] rows of table and lens, NULL: 0 .. batch-1; a negative one has no positions */
  const int32_t* row_off;           /* DEV [batch+1]                                                 */
  const int32_t* parent;            /* DEV [rows]                                                    */
  int32_t* status;                  /* DEV [1] or NULL: CAPACITY (above), INVALID_ARG (above; a page id that is none, for a position
                                     * that is seen: its key and value count as zeros), TIMEOUT if a bounded wait gave up */
  int32_t max_pages, max_seqs, batch, n_heads, max_nodes, max_len, window, n_prefix;
  float scale;                      /* above 0                                                       */
  int32_t n_rows;                   /* rows of q, k_new, v_new, out and lse, or 0: not said          */
  int32_t fill;                     /* rows of no tree (with n_rows): FM_FILL_OUT out 0, FM_FILL_LSE lse -inf */
} fm_tree_args;
size_t fm_tree_attention_bytes(const fm_cache* cache, const fm_tree_args* args);   /* workspace; 0 if the arguments are invalid */
int fm_tree_attention(const fm_cache* cache, int32_t layer, const fm_tree_args* args, void* workspace /*DEV, 256-byte aligned*/,
                      size_t workspace_bytes, void* stream);

/* The longest confirmed path of every tree: from node 0 (the token already accepted, parent -1) on to the lowest
 * child whose token is the prediction at the node, as long as there is one.  path: DEV out
 * [batch, path_stride], node indices counted from row_off[i], then -1; n_acc: DEV out [batch]; next_tok:
 * DEV out [batch], the prediction at the last node of the path.  A sequence without rows, or whose
 * node 0 has a parent: n_acc 0, next_tok -1.  Nodes behind path_stride or FM_MAX_TREE_NODES are not followed.
 * fm_tree_accept_rows: the same, told how many rows there are; a sequence whose offsets are not inside them is one without rows. */
int fm_tree_accept(const int32_t* tokens /*DEV [rows]*/, const int32_t* parent /*DEV*/, const int32_t* row_off /*DEV*/,
                   const int32_t* predicted /*DEV [rows]*/, int32_t batch, int32_t* path, int32_t path_stride, int32_t* n_acc, int32_t* next_tok,
                   void* stream);
int fm_tree_accept_rows(const int32_t* tokens, const int32_t* parent, const int32_t* row_off, const int32_t* predicted, int32_t rows, int32_t batch,
                        int32_t* path, int32_t path_stride, int32_t* n_acc, int32_t* next_tok, void* stream);

/* Scores of logits rows x (FM_FP32 / FM_BF16 / FM_FP16, `row_stride` elements apart; e.g. those of
 * fm_verify or fm_draft), one pass over the data:
 *   logprob[r] = x_t - log sum exp x, t = tokens[r];  rank[r] = number of entries above x_t
 *   entropy[r] = -sum p log p (natural logarithm; an entry of -inf counts 0)
 *   top_ids / top_logprobs [rows, top]: the largest entries, equal ones lowest id first
 * in 32 bits.  tokens NULL, or a token outside [0, vocab): logprob -inf, rank -1.  An output may be
 * NULL.  A row of -inf alone: logprob -inf, entropy 0, top_logprobs -inf.  A NaN or +inf in a row makes logprob, entropy
 * and top_logprobs NaN; a NaN ranks below -inf.  Errors: INVALID_ARG (null logits, rows < 0, vocab < 1, stride < vocab, top < 0 or > vocab, dtype),
 * CAPACITY (top > FM_MAX_TOP). */
int fm_logprobs(const void* logits /*DEV*/, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride, const int32_t* tokens /*DEV or NULL*/,
                float* logprob, float* entropy, int32_t* rank, int32_t top, int32_t* top_ids, float* top_logprobs, void* stream);


#ifdef __cplusplus
}
#endif
#endif /* FLASHMESH_H */
