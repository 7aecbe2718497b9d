/*
 * esp.h -- C ABI of the ESP (Embedding-Space Probing) speculate-and-verify decode step
 * for MI355X (gfx950).  Plain pointers and sizes only; no C++ or framework types.
 *
 * One decode step (paper Sec. 3.3, Fig. 1 right) is four calls on one stream:
 *
 *   esp_tree_forward      forward of [last accepted token | draft-tree tokens | mask tokens]
 *                         against the KV cache under the tree attention mask, LM head and
 *                         argmax at the tree rows                       (Sec. 2, Sec. 3.3, App. C/E)
 *   esp_verify_accept     lossless longest-accepted-path check, bonus token, KV commit
 *                                                                       (Sec. 2 Eq. 3, Sec. 3.3, Sec. 4)
 *   esp_mask_topk         LM head + vocabulary softmax + Top-K' at the mask rows aligned to the
 *                         accepted position                             (Sec. 2 Eq. 2, Sec. 3.3)
 *   esp_build_prune_tree  pruning rule and dynamic tree construction -> next block
 *                                                                       (Sec. 3.4 Alg. 1, Sec. 3.5, App. C)
 *
 * Conventions
 *  - "device" = pointer into GPU memory owned by the caller; "host" = ordinary host memory.
 *    The library never allocates or frees device memory and never keeps a caller pointer
 *    beyond the call, except the weight pointers handed to esp_create (kept until esp_destroy)
 *    and the workspace.
 *  - Every call enqueues its kernels on the ctx stream and returns without synchronising,
 *    except where stated.  The return value reports what the host can check (null pointers,
 *    shapes, capacities known on the host).  Conditions only the device can see (a sequence
 *    whose length exceeds the host's bound or its capacity, a malformed tree) set a sticky
 *    device status word, read with esp_last_device_status(); the offending work is skipped,
 *    never executed out of bounds.
 *  - No entry point throws or aborts.
 *  - Matrices are row-major [out_features, in_features] in the model dtype.
 *  - Rows: a block holds `batch` sequences, sequence b owning rows
 *    [b*rows_per_seq, b*rows_per_seq + n_rows[b]).  Within a sequence rows 0..n_nodes-1 are
 *    tree nodes in (depth, creation) order, row 0 the last accepted token; mask rows follow
 *    (Fig. 3).  ESP_LAYOUT_PER_NODE: node a owns mask rows n_nodes + a*k + (j-1), j = 1..k,
 *    so n_rows = (k+1) n_nodes (block complexity, Sec. 3.3).  ESP_LAYOUT_ROOT_CHAIN: only the
 *    root owns a chain, n_rows = n_nodes + k.
 */
#ifndef ESP_H_
#define ESP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct esp_ctx esp_ctx; /* opaque; host object, owns nothing on the device */

typedef enum {
  ESP_OK = 0,
  ESP_EINVAL = 1,    /* null pointer or value out of range */
  ESP_ESHAPE = 2,    /* shape the kernels do not support */
  ESP_ECAPACITY = 3, /* rows / batch / length beyond what ctx or workspace was created for */
  ESP_EDTYPE = 4,
  ESP_EDEVICE = 5,   /* a HIP call failed */
  ESP_ESTATE = 6
} esp_status;

typedef enum { ESP_F32 = 0, ESP_BF16 = 1 } esp_dtype;

enum { ESP_LAYOUT_PER_NODE = 0, ESP_LAYOUT_ROOT_CHAIN = 1 };

enum {
  ESP_MAX_MASKS = 8,         /* k */
  ESP_MAX_ROWS_PER_SEQ = 1024,
  ESP_MAX_TOPK = 32,         /* K' */
  ESP_MAX_TREE_NODES = 256,  /* B */
  ESP_KV_BLOCK = 64          /* V-cache slot blocking, see esp_kv */
};

/* bits of the device status word */
enum {
  ESP_DEV_LEN_OVER_BOUND = 1,  /* kv.len[b] + n_rows[b] exceeds kv.len_bound or seq capacity */
  ESP_DEV_BAD_TREE = 2,        /* parent not before child, n_nodes/n_rows out of range, list */
                               /* entries above 1 that keep a node without its parent        */
  ESP_DEV_BAD_TOKEN = 4,       /* token id outside the vocabulary                            */
  ESP_DEV_BAD_ROWS = 8,        /* esp_chunk.row0 descends, or a sequence has more rows than   */
                               /* max_rows or rows past total_rows                            */
  ESP_DEV_BAD_PAGE = 16,       /* a page that is needed lies outside the pool                 */
  ESP_DEV_BAD_PATH = 32        /* an accepted path that is none (esp_paged_commit)            */
};

typedef struct {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ff, vocab;
  float rope_theta; /* rotary base; pairs (i, i + head_dim/2) turn by pos * theta^(-2i/head_dim) */
  float rms_eps;
  int32_t qk_norm;  /* 1: per-head RMSNorm over head_dim on q and k before the rotation */
  int32_t dtype;    /* esp_dtype of weights, KV cache, mask embeddings and hidden_out */
} esp_model_desc;

/* Weights: the arrays of per-layer pointers are HOST arrays of n_layers DEVICE pointers. */
typedef struct {
  const void *embed;             /* [vocab, d_model]                                   */
  const void *lm_head;           /* [vocab, d_model] (untied)                          */
                                 /* bf16 models: every matrix below and lm_head in the */
                                 /* layout of esp_pack_weight; embed stays row-major   */
  const void *final_norm;        /* [d_model]                                          */
  const void *const *wqkv;       /* [(n_q + 2 n_kv) * head_dim, d_model]: q, k, v rows */
  const void *const *wo;         /* [d_model, n_q * head_dim]                          */
  const void *const *w_gate_up;  /* [2 d_ff, d_model].  ESP_F32: all gate rows, then all up rows.
                                  * ESP_BF16: blocks of 32 rows alternate (gate rows 0..31, up rows
                                  * 0..31, gate rows 32..63, ...) before esp_pack_weight, so that the
                                  * projection can apply the SwiGLU in its epilogue */
  const void *const *w_down;     /* [d_model, d_ff]                                    */
  const void *const *norm_attn;  /* [d_model]                                          */
  const void *const *norm_mlp;   /* [d_model]                                          */
  const void *const *q_norm;     /* [head_dim], NULL unless qk_norm                    */
  const void *const *k_norm;     /* [head_dim], NULL unless qk_norm                    */
} esp_weights;

/* KV cache pool (device, model dtype), shared by the sequences of a batch.  k and v each hold
 * [n_layers][n_kv_heads] planes of capacity * head_dim elements.  A plane is a sequence of blocks
 * of 32 slots; inside a block the elements sit in the order the matrix cores consume them
 * (64 lanes x 8 elements per fragment), head_dim a multiple of 32:
 *   k block: [head_dim/16][64][8]     element (slot, d) at ((d/16)*64 + ((d/8)%2)*32 + slot%32)*8 + d%8
 *   v block: [head_dim/32][2][64][8]  element (slot, d), key = slot%32, at
 *            (((d/32)*2 + key/16)*64 + ((key/4)%2)*32 + d%32)*8 + 4*((key/8)%2) + key%4
 * Callers never index the pool themselves: esp_kv_store / esp_kv_load convert from and to plain
 * [slots][head_dim] rows.
 * Sequence b owns slots [base[b], base[b] + seq_cap[b]); base[b] is a multiple of 64.
 * Slots [0, len[b]) of a sequence hold committed tokens; a forward writes the block's rows at
 * len[b] + row (scratch until committed). */
typedef struct {
  void *k, *v;             /* device */
  int32_t *len;            /* device [batch]; advanced by esp_verify_accept                   */
  const int32_t *base;     /* device [batch]                                                  */
  const int32_t *seq_cap;  /* device [batch]                                                  */
  int64_t capacity;        /* host: slots per (layer, kv head) in the pool, multiple of 64    */
  int32_t len_bound;       /* host: upper bound of len[b] over the batch for this call; sizes */
                           /* the attention launch (the kernels read the true len on device)  */
} esp_kv;

/* One forward block.  Scalars are host values; arrays are device memory sized for
 * batch * rows_per_seq rows, written by esp_build_prune_tree / esp_block_from_tree. */
typedef struct {
  int32_t batch;
  int32_t rows_per_seq; /* row stride of a sequence, <= ESP_MAX_ROWS_PER_SEQ               */
  int32_t k_masks;      /* k, 0..ESP_MAX_MASKS                                              */
  int32_t layout;
  int32_t anc_words;    /* 64-bit words per ancestor bitset = ceil(rows_per_seq / 64)       */
  int32_t *n_rows;      /* [batch]                                                          */
  int32_t *n_nodes;     /* [batch]                                                          */
  int32_t *tok;         /* [rows] token id of node rows, -1 on mask rows                    */
  int32_t *parent;      /* [rows] tree parent row (in-sequence index), -1 for the root;     */
                        /*        mask rows: the row before them in their chain             */
  int32_t *depth;       /* [rows] position of a row = len[b] + depth (App. E)               */
  int32_t *mask_j;      /* [rows] 0 for node rows, 1..k for mask rows                       */
  int32_t *attach;      /* [rows] node row a mask row hangs on (node rows: themselves)      */
  uint64_t *anc;        /* [rows][anc_words] bit c set: row may attend to block row c       */
} esp_block;

/* Parameters of the tree builder (Alg. 1; Sec. 3.5). */
typedef struct {
  int32_t B;            /* node budget including the root, <= ESP_MAX_TREE_NODES             */
  int32_t k;            /* mask tokens = maximum depth                                       */
  int32_t K;            /* cap on children per expanded node (children = min(K, B - i))      */
  int32_t expand_width; /* nodes expanded per depth: 1 = Top-1 expansion (App. C), <=0 = all */
  int32_t prune_parent; /* drop a candidate equal to its parent's token (Sec. 3.5)           */
  int32_t prune_last;   /* also drop the last generated token at depths >= 2                 */
  int32_t layout;       /* layout of the block to write                                      */
  int32_t static_widths[ESP_MAX_MASKS]; /* [K_1..K_k] fixed tree, no selection; all 0 = dynamic */
} esp_tree_params;

const char *esp_status_str(esp_status s);

/* Workspace (device scratch for activations, split-K partials, attention partials, logits of
 * the mask rows).  max_rows_per_seq and max_batch bound every later block; max_kv_len bounds
 * kv.len_bound + rows_per_seq. */
size_t esp_workspace_bytes(const esp_model_desc *m, int32_t max_batch, int32_t max_rows_per_seq,
                           int64_t max_kv_len);

/* Creates the host context.  `workspace` is device memory of at least esp_workspace_bytes(),
 * 256-byte aligned, owned by the caller and used by every call until esp_destroy.  `stream` is a
 * hipStream_t (NULL = the default stream).  Calls on one ctx must not overlap.
 * Errors: EINVAL (null / non-positive sizes), ESHAPE (head_dim not in {64,128} for bf16 models,
 * d_model or d_ff not a multiple of 64 for bf16, n_q_heads not a multiple of n_kv_heads, ...),
 * ECAPACITY (workspace too small), EDTYPE. */
esp_status esp_create(const esp_model_desc *m, const esp_weights *w, int32_t max_batch,
                      int32_t max_rows_per_seq, int64_t max_kv_len, void *workspace,
                      size_t workspace_bytes, void *stream, esp_ctx **out);
esp_status esp_destroy(esp_ctx *ctx);

/* Synchronises the stream and returns (and clears) the sticky device status bits. */
esp_status esp_last_device_status(esp_ctx *ctx, int32_t *host_out);

/* ---- the four calls of a step ------------------------------------------------------------ */

/* Sample matching (the paper's temperature-1 mode, Sec. 4 / appendix on sampling): when enabled,
 * node_argmax[r] of esp_tree_forward is not the arg-max but a temperature-1 draw of the token that
 * follows row r, taken as arg-max over the vocabulary of logit + Gumbel noise.  The noise is a
 * counter-based function of (seed, absolute position of the drawn token, token id), so the draw at a
 * position is the same whether that position is reached by one-token-at-a-time decoding or inside a
 * tree, and esp_verify_accept (exact match against the draws) stays lossless with respect to
 * sampling with the same seed.  Disabled (greedy) after esp_create.  Host state only; applies to
 * later esp_tree_forward calls on this context. */
esp_status esp_set_sampling(esp_ctx *ctx, int32_t enabled, uint32_t seed);

/* Forward of all rows of `blk` (Sec. 3.3): h0 = embed[tok] on node rows, mask_embed[j-1] on mask
 * rows (Sec. 3.1); per layer RMSNorm, QKV, optional QK-norm, rotary at position len[b]+depth,
 * K/V of the rows written to cache slots len[b]+row, tree-masked grouped-query attention over
 * cache slots [0,len[b]) plus the block rows in the row's ancestor bitset (App. C), output
 * projection, SwiGLU MLP; final RMSNorm.
 *   mask_embed  device [k_masks, d_model], model dtype ([batch, k_masks, d_model] after esp_set_mask_batch)
 *   hidden_out  device [batch*rows_per_seq, d_model], model dtype: final-norm hidden states
 *   node_argmax device [batch*rows_per_seq] int32: argmax over the vocabulary of the LM head at
 *               node rows (lowest id on ties); entries of mask rows are left untouched
 *   logits_dbg  NULL, or device [batch*rows_per_seq, vocab] fp32 receiving the LM-head logits of
 *               every row (parity tests)
 * Errors: EINVAL, ECAPACITY (batch/rows beyond ctx, len_bound + rows_per_seq > max_kv_len; bf16 with node_argmax and without
 * logits_dbg, as esp_mask_topk: hidden states of 4 GiB and more). */
esp_status esp_tree_forward(esp_ctx *ctx, const esp_block *blk, const void *mask_embed,
                            const esp_kv *kv, void *hidden_out, int32_t *node_argmax,
                            float *logits_dbg);

/* Greedy verification (Sec. 2 Eq. 3): starting at the root, a child is accepted iff its token
 * equals node_argmax of its parent; the walk ends at the first miss at node n*; node_argmax[n*]
 * is the bonus token (Sec. 4: tau counts accepted + bonus).  Then the K/V of the accepted rows are
 * moved to slots len+1.. in path order (the root already sits at len) and len[b] += n_emit[b].
 * Outputs (device): n_emit [batch]; emit_tok, accepted_row [batch][ESP_MAX_MASKS+1]
 * (accepted_row[b][0] = 0, the root, then the accepted rows); star_row [batch] = n*. */
esp_status esp_verify_accept(esp_ctx *ctx, const esp_block *blk, const int32_t *node_argmax,
                             const esp_kv *kv, int32_t *n_emit, int32_t *emit_tok,
                             int32_t *accepted_row, int32_t *star_row);

/* Proposal (Sec. 2 Eq. 2; Sec. 3.3): LM head on the mask rows aligned to the accepted position,
 * softmax over the full vocabulary in fp32, the Kp most probable tokens per row ordered by
 * (probability descending, id ascending).  PER_NODE: rows mask(n*, i), i = 1..k.  ROOT_CHAIN:
 * rows mask(root, a+i), i = 1..k-a, with a = n_emit-1 accepted tokens.
 *   hidden   device: hidden_out of esp_tree_forward, unchanged since that call.  For blocks of at
 *            most 128 rows (bf16) the forward has already taken all rows through the LM head and
 *            left the logits in the workspace; this call then reads its rows there instead of
 *            streaming the LM-head matrix a second time (recognised by the same `hidden` pointer
 *            and row count; any other esp_tree_forward in between invalidates it)
 *   topk_id  device [batch][k_masks][Kp] int32;  topk_p same shape fp32
 *   n_lists  device [batch] int32: number of valid lists (depths the next tree may have)
 *   logits_out NULL or device [batch][k_masks][vocab] fp32 (parity tests)
 * Errors: EINVAL (Kp < 1 or > ESP_MAX_TOPK or > vocab). */
esp_status esp_mask_topk(esp_ctx *ctx, const esp_block *blk, const int32_t *star_row,
                         const int32_t *n_emit, const void *hidden, int32_t Kp, int32_t *topk_id,
                         float *topk_p, int32_t *n_lists, float *logits_out);

/* Pruning + dynamic tree (Alg. 1, Sec. 3.5): root = last emitted token with P = 1; for depth
 * i = 1..n_lists the expanded nodes of depth i-1 (all of the current node set, or its
 * expand_width most probable) take their first min(K, B-i) candidates of list i that survive the
 * pruning rule, P(child) = P(parent) * p as one fp32 product; between depths the node set is the
 * B-i most probable not-yet-used candidates; the tree is the root plus the B-1 most probable of
 * all candidates (ties: earlier created first).  Writes every array of `next` for each sequence.
 * Fixed trees (static_widths set; Sec. 4.3): root, K_1 children, K_i children under the first node
 * of depth i-1.  Their rows do not depend on the lists, so they are built once per block: the
 * context remembers which blocks (by the address of `tok`) hold the rows of which fixed tree, and a
 * later call with the same parameters writes only the tokens (per sequence the kernel still checks
 * that the block holds a tree of that size and that no list runs out, and builds in full if not).
 * A caller that writes the structure arrays of such a block itself must pass the block through
 * esp_block_from_tree before the next esp_build_prune_tree.
 * topk_p: probabilities, 0 <= p <= 1, which is what esp_mask_topk and esp_softmax_topk hand out; a child is
 * then never more probable than its parent, so the chosen nodes form a tree.  Entries above 1 are taken as
 * they are (the build is then slower: nothing can be dropped early), NaN ranks above all, negative entries count
 * as 0.  Where the nodes chosen are no tree (a child kept, its parent cut) the sequence gets n_rows = n_nodes = 0
 * and ESP_DEV_BAD_TREE.
 * Errors: EINVAL (B, k, K, Kp out of range; k != next->k_masks), ECAPACITY (rows of the tree
 * exceed next->rows_per_seq). */
esp_status esp_build_prune_tree(esp_ctx *ctx, const esp_tree_params *p, const int32_t *topk_id,
                                const float *topk_p, int32_t Kp, const int32_t *n_lists,
                                const int32_t *n_emit, const int32_t *emit_tok, esp_block *next);

/* ---- stage-level and auxiliary entry points ----------------------------------------------- */

/* Fills depth, mask rows, attach, mask_j, parent of mask rows, n_rows and the ancestor bitsets
 * from blk->tok / blk->parent / blk->n_nodes of the node rows (already on the device). */
esp_status esp_block_from_tree(esp_ctx *ctx, esp_block *blk);

/* Mask vectors (Sec. 3.1): Eq. 4, m_i = mean of embed[prompt tokens] (fp32 accumulation), and
 * Eq. 5, m <- m + lambda (embed[last emitted token of sequence 0] - m).  mask_embed: device
 * [k, d_model] model dtype.  tokens: device int32. */
esp_status esp_mask_mean(esp_ctx *ctx, const int32_t *tokens, int32_t n_tokens, int32_t k,
                         void *mask_embed);
esp_status esp_mask_ema(esp_ctx *ctx, const int32_t *n_emit, const int32_t *emit_tok, float lambda,
                        int32_t k, void *mask_embed);

/* Mask vectors per sequence (Eq. 4 and Eq. 5 are stated per generation).  esp_set_mask_batch with
 * per_sequence != 0 makes esp_tree_forward read the mask rows of sequence b from
 * mask_embed + b * k_masks * d_model, i.e. mask_embed is device [batch, k_masks, d_model]; 0 (the state a
 * new context is in) is the shared [k_masks, d_model] form.  Host-side state only: takes effect for the calls
 * enqueued after it.  esp_mask_ema_batch is Eq. 5 for that form: the vectors of sequence b move towards
 * the embedding of b's own last emitted token (n_emit[b], emit_tok[b][.]); sequences that emitted nothing
 * keep theirs.  The initialisers above write one [k, d_model] slice per call: pass mask_embed + b * k * d_model. */
esp_status esp_set_mask_batch(esp_ctx *ctx, int32_t per_sequence);
esp_status esp_mask_ema_batch(esp_ctx *ctx, int32_t batch, const int32_t *n_emit, const int32_t *emit_tok,
                              float lambda, int32_t k, void *mask_embed);

/* The two other initialisations of the mask-design ablation (Sec. 4) and the out-of-distribution
 * rows of the appendix table on mask initialisation.
 * esp_mask_last_k: hard initialisation, mask i (0-based) = embed[tokens[n_tokens - k + i]], the last
 *   k prompt tokens in prompt order (the index printed in the paper would skip exactly those
 *   tokens; its words are followed).  EINVAL if n_tokens < k.
 * esp_mask_gaussian: m_i = mu + (shift + z_i) sigma with the Gaussian fit of the embedding table:
 *   mu[d_model] the mean over the vocabulary per dimension, sigma one scalar, the root mean square
 *   deviation of all entries from their dimension's mean (two passes over the table, fp32 slab
 *   sums added in fp64).  z: device fp32 [k, d_model], the caller's standard normal draws (the
 *   library draws nothing), or NULL for z = 0; shift 0 gives the paper's "Sample" variant, z NULL
 *   with shift 5 or 10 its mu + 5 sigma and mu + 10 sigma rows.  Uses the context's logits buffer
 *   as scratch (logits kept for esp_mask_topk by the last esp_tree_forward are dropped).
 * mask_embed: device [k, d_model] model dtype. */
esp_status esp_mask_last_k(esp_ctx *ctx, const int32_t *tokens, int32_t n_tokens, int32_t k,
                           void *mask_embed);
esp_status esp_mask_gaussian(esp_ctx *ctx, const float *z, float shift, int32_t k, void *mask_embed);

/* Copies plain K/V rows [n_slots][n_kv_heads][head_dim] (model dtype, device) of one layer into /
 * out of the cache layout at slots base + first_slot .. */
esp_status esp_kv_store(esp_ctx *ctx, const esp_kv *kv, int32_t layer, int32_t seq_base,
                        int32_t first_slot, int32_t n_slots, const void *k_rows, const void *v_rows);
esp_status esp_kv_load(esp_ctx *ctx, const esp_kv *kv, int32_t layer, int32_t seq_base,
                       int32_t first_slot, int32_t n_slots, void *k_rows, void *v_rows);

/* Rewrites a row-major bf16 matrix W[N,K] (device) into the streaming layout the bf16 GEMMs read:
 * tiles of 32 output rows x 64 inputs, each 4 KB contiguous in MFMA operand order, tiles ordered
 * [K/64][N/32].  dst: device, N*K bf16, must not alias src.  Needs N % 32 == 0, K % 64 == 0.
 * Every bf16 matrix handed to esp_create (wqkv, wo, w_gate_up, w_down, lm_head) must be in this
 * layout; embed and the norm gains stay plain.  fp32 models use plain row-major matrices. */
esp_status esp_pack_weight(void *stream, const void *src, void *dst, int32_t N, int32_t K);

/* C[M,N] (fp32, device) = A[M,K] * W[N,K]^T, A and W in `dtype` (device), on `stream`.
 * bf16 needs N % 32 == 0 and K % 64 == 0; w_packed != 0: W is in the streaming layout.
 * `partials` is device scratch of esp_gemm_scratch_bytes(M,N,K) bytes (split-K partial sums;
 * reduced in a fixed order). */
size_t esp_gemm_scratch_bytes(int32_t M, int32_t N, int32_t K);
esp_status esp_gemm(void *stream, int32_t dtype, const void *A, const void *W, int32_t w_packed,
                    float *C, int32_t M, int32_t N, int32_t K, void *partials, size_t partial_bytes);

/* LM head with the greedy choice of Sec. 2 Eq. 3 taken in the GEMM's epilogue (the path
 * esp_tree_forward uses at the tree rows): argmax[m] = arg-max over n of A[m,:] . W[n,:], lowest n on
 * ties, for bf16 A[M,K] and W[N,K] in the streaming layout (both device).  The [M,N] logits are never
 * written.  `scratch`: device, esp_gemm_argmax_scratch_bytes(M,N) bytes (per-tile (value, index)
 * pairs).  ESP_ESHAPE if N % 32 or K % 64. */
size_t esp_gemm_argmax_scratch_bytes(int32_t M, int32_t N);
esp_status esp_gemm_argmax(void *stream, const void *A, const void *W, int32_t M, int32_t N, int32_t K,
                           void *scratch, size_t scratch_bytes, int32_t *argmax);

/* Tree-masked grouped-query attention of one layer (the kernel esp_tree_forward uses):
 * q device [batch*rows_per_seq, n_q_heads, head_dim] model dtype, already rotated; K/V of the
 * block rows already in the cache at len[b]+row; out same shape as q. */
esp_status esp_attn_tree(esp_ctx *ctx, const esp_block *blk, const esp_kv *kv, int32_t layer,
                         const void *q, void *out);

/* Fused softmax + Top-K over `rows` fp32 logit rows of `vocab` entries (device): ids/probs
 * [rows][Kp], ordered by (probability descending, id ascending).  `scratch`: device memory of
 * esp_softmax_topk_scratch_bytes() bytes (per-chunk statistics and candidates). */
size_t esp_softmax_topk_scratch_bytes(int32_t rows, int32_t vocab, int32_t Kp);
esp_status esp_softmax_topk(void *stream, const float *logits, int32_t rows, int32_t vocab,
                            int32_t Kp, int32_t *ids, float *probs, void *scratch,
                            size_t scratch_bytes);

/* esp_softmax_topk for callers that cannot allocate or bring a workspace (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the per-segment records live in a
 * device array that is part of the library image (2.06 MiB per GPU, held until the process ends)
 * instead of `scratch`.  Same kernels, same results as esp_softmax_topk.  The call allocates
 * nothing and synchronises nothing; the device that is current at the call must be the stream's.
 * Limit: rows * min(64, ceil(vocab / 2048)) * (2 + 2 Kp) <= 128 * 64 * 66 floats, i.e. up to 128
 * rows at any vocabulary and Kp (more rows for smaller vocabularies or Kp); beyond that
 * ESP_ECAPACITY and nothing is launched.  All calls on one GPU share the one array: calls that
 * overlap in time on the same GPU (different streams or threads) race; successive calls on one
 * stream do not (every record a call reads it has written itself).
 * Errors: EINVAL as esp_softmax_topk, ECAPACITY, EDEVICE (symbol lookup or launch failed). */
esp_status esp_softmax_topk_static(void *stream, const float *logits, int32_t rows, int32_t vocab,
                                   int32_t Kp, int32_t *ids, float *probs);

/* The next token of every row from its logits, each row with limits of its own.  In order of their logits (equal ones by id) the tokens weigh
 * w = exp((logit - largest) / temperature).  Kept are the first top_k; of those, W their weights' sum, each before which less than top_p W lies;
 * of those, what weighs min_p or more; the first of all in any case.  The token is the lowest id at which the kept weights, added up over the ids to
 * it, are above u times their sum.  temperature 0: the first of the order.
 *   logits      device [rows][vocab], fp32 or bf16, rows row_stride elements apart (any alignment of the type)
 *   temperature, top_p, min_p  device fp32 [rows]; top_k device int32 [rows]; NULL: 1, 1, 0 and none.  top_k below 1, top_p of 1 and more and
 *               min_p of 0 and less are no limit; top_p below 0 is 0, min_p above 1 is 1
 *   u           device fp32 [rows], uniform in [0, 1): below (and NaN) 0, above the largest below 1
 *   ids         device int32 [rows]; probs NULL or device fp32 [rows]: the token's share of the kept weights (temperature 0: 1)
 * Minus infinity and NaN are tokens that cannot be chosen, plus infinity is as the largest finite fp32 value.  A row without any other, and a row
 * whose temperature is negative or not finite or whose top_p or min_p is NaN, gets -1 and 0.
 * Temperatures between 0 and 1e-20 are as 1e-20, above 1e20 as 1e20.  Weights are taken in fp64 (1.1e-12 of themselves) and added up in units of 2^-S of
 * the largest, S = min(45, 62 - ceil log2 vocab); tokens of less than half a unit are not chosen, and count in W unless there is a top_k.  A border among n
 * tokens that weigh W of the largest may lie 2 (3e-12 + n 2^-(S+1) / W) of all off: 4e-9 at 128256 tokens and W = 1.  The same call chooses the same tokens.
 *   scratch     device, 16-byte aligned, esp_sample_scratch_bytes(): what is enough for so many rows and for fewer (of a row of 128256 up to 329 KB for 32 rows,
 *               181 KB where there are more; of up to 4096 tokens 16 bytes; of up to 1024 rows: more are done in lots; the same with limits and without).  Calls that overlap in time need one
 *               each.  Results do not depend on what it held
 * Errors: EINVAL (null pointers, rows < 0, vocab < 1), ESHAPE (row_stride < vocab), EDTYPE, ECAPACITY (scratch; vocab above 2^22). */
size_t esp_sample_scratch_bytes(int32_t rows, int32_t vocab);
esp_status esp_sample(void* stream, int32_t dtype, const void* logits, int64_t row_stride, int32_t rows, int32_t vocab, const float* temperature,
                      const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* ids, float* probs, void* scratch,
                      size_t scratch_bytes);

/* ---- paged KV cache ------------------------------------------------------------------------
 * A cache whose sequences own pages anywhere in a pool, the rotation and the norms that come before it, and the
 * attention that reads it.  The calls take a stream and no context; the device that is current at the call must
 * be the stream's.  They allocate nothing, synchronise nothing and can be captured into a graph. */

/* Rotary positions of a head: the first rot_dim features turn in pairs, (i, i + rot_dim/2) or, interleaved,
 * (2i, 2i+1); the others pass.  Pair i turns by position * turns[i] revolutions, and the turned features are
 * multiplied by `amplitude`.  Filled by esp_rope_make (host only); `turns` may hold any other finite speeds. */
typedef struct {
  int32_t head_dim;     /* 64 or 128                                     */
  int32_t rot_dim;      /* multiple of 16, 16 .. head_dim                */
  int32_t interleaved;
  float amplitude;
  double turns[64];     /* [rot_dim/2] revolutions per position          */
} esp_rope;

/* f_i = theta^(-2i/rot_dim) radians a position.  factor > 1 stretches the positions for contexts longer than the
 * model was trained on: n_i = orig_len f_i / 2 pi is how often pair i turns in the trained context, keep_i =
 * clamp((n_i - low_turns) / (high_turns - low_turns), 0, 1), and the pair's speed is f_i (keep_i + (1 - keep_i) /
 * factor): what turns often keeps its speed, what turns seldom is slowed down.  orig_len 0: all are slowed down
 * (positions divided by factor).
 * Errors: EINVAL (out null, theta or factor not positive and finite, orig_len < 0, low_turns >= high_turns with orig_len > 0,
 * amplitude not finite, or a speed that comes out of them), ESHAPE (head_dim, rot_dim); *out is then as it was. */
esp_status esp_rope_make(int32_t head_dim, int32_t rot_dim, int32_t interleaved, double theta, double factor,
                         int32_t orig_len, double low_turns, double high_turns, double amplitude, esp_rope *out);

/* Rotary positions on rows of queries and keys, with the RMS norm of every head (over head_dim, gain [head_dim] in
 * `dtype`) before it where a gain is given.  q [rows][n_q_heads][head_dim], k [rows][n_kv_heads][head_dim]: heads lie
 * side by side, rows *_stride elements apart (parts of one projection's rows are taken as they are).  The outputs
 * have strides of their own; an output may be its input with the same stride, and otherwise must not overlap any input.
 * positions device [rows].  Either of q and k may be NULL with its output (its head count is then not looked at).  The
 * arithmetic is fp32 (the angle fp64), rounded once; the squares of a head that is normed have to fit it (features up to 1e18).
 * Errors: EINVAL (null pointers, rows < 0, n_* < 1, eps negative or not finite), ESHAPE (strides below heads * head_dim), EDTYPE,
 * ECAPACITY (more than 2^26 - 4 rows, or than 2^31 - 1 rows x heads, or 2^22 - 1 heads). */
esp_status esp_rope_qk(void *stream, int32_t dtype, const esp_rope *rope, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads,
                       const void *q, int64_t q_stride, const void *k, int64_t k_stride, const int32_t *positions,
                       const void *q_gain, const void *k_gain, float eps, void *q_out, int64_t q_out_stride, void *k_out,
                       int64_t k_out_stride);

/* The pool.  k and v each hold [n_layers][n_pages][n_kv_heads] planes of page_size * head_dim elements in the block order
 * of esp_kv (blocks of 32 slots); 16-byte aligned.  Slot s of sequence b lies in page page_table[b][s / page_size], at slot
 * s % page_size; entries of pages that hold no token of the sequence are never used.  Two sequences may share pages that
 * nobody writes.  Slots [0, len[b]) hold committed tokens.
 * ECAPACITY: table_stride * page_size or n_pages * n_kv_heads * page_size / 32 of 2^31 and more, n_layers * n_kv_heads of 2^24 and
 * more, n_layers or batch above 65535. */
typedef struct {
  void *k, *v;                /* device                                                                          */
  const int32_t *page_table;  /* device [batch][table_stride]                                                    */
  const int32_t *len;         /* device [batch]                                                                  */
  int32_t *status;            /* device, one word that collects ESP_DEV_ bits (the caller clears it), or NULL    */
  int32_t dtype, n_layers, n_kv_heads;
  int32_t head_dim;           /* 64 or 128                                                                       */
  int32_t page_size;          /* slots of a page, multiple of 32                                                 */
  int32_t n_pages;            /* of the pool                                                                     */
  int32_t batch;
  int32_t table_stride;       /* entries of the page table per sequence: it holds table_stride * page_size slots */
  int32_t len_bound;          /* host: upper bound of len[b] for this call                                       */
} esp_paged_kv;

/* New rows of the sequences, packed: sequence b has rows row0[b] .. row0[b+1] - 1 (none, one or many), in the order of
 * its slots: row r of it belongs into slot len[b] + r.  Rows from row0[batch] on are not touched. */
typedef struct {
  const int32_t *row0;        /* device [batch + 1], ascending                                                   */
  int32_t total_rows;         /* host: rows that the buffers hold, at least row0[batch]                          */
  int32_t max_rows;           /* host: upper bound of a sequence's rows                                          */
} esp_chunk;

/* What only the device can see -- len[b] negative, above len_bound or with its rows past the table, row0 or pages out of
 * range -- sets bits in *status.  Of a sequence with bad lengths or rows nothing is read or written; a slot in
 * a page outside the pool is not written (append, commit), and not seen (attention).  Where row0 descends, a row may be among those of
 * several sequences that are each in order: which of them get it, and whose output it holds, is not defined. */

/* Writes K and V of the chunk's rows into their slots of `layer`, K normed and rotated on the way, and the rows' queries,
 * normed and rotated, to q_out [total_rows][n_q_heads][head_dim] (rows q_out_stride elements apart).  rope NULL: no rotation.
 * positions device [total_rows], or NULL: a row's position is its slot (a tree's rows have len + depth).  q and q_out may
 * both be NULL, and q_out may be q with the same stride.  len is not advanced.
 * Errors: as esp_rope_qk (heads of q, k and v); EINVAL also for a malformed esp_paged_kv or esp_chunk or a layer outside it; ESHAPE for head_dim other than the
 * rope's. */
esp_status esp_paged_append(void *stream, const esp_paged_kv *kv, int32_t layer, const esp_chunk *rows, const esp_rope *rope,
                            const int32_t *positions, int32_t n_q_heads, const void *q, int64_t q_stride, const void *k,
                            int64_t k_stride, const void *v, int64_t v_stride, const void *q_gain, const void *k_gain, float eps,
                            void *q_out, int64_t q_out_stride);

/* Grouped-query attention of the chunk's rows, whose K and V are in their slots already: row r of sequence b sees slots
 * [0, len[b]) and, of the chunk, rows 0..r (anc NULL) or the rows c whose bit is set in its ancestor bitset anc
 * [total_rows][anc_words] (as esp_block).  out = softmax(scale q k) v; a row that sees nothing gets zeros.  What a row does
 * not see does not reach it, whatever it holds.  q as in esp_paged_append; out device [total_rows][n_q_heads][head_dim],
 * contiguous, no overlap with q.
 * Scores, sums and the outputs until they are written are fp32; in bf16 the probabilities are rounded to it for the product with V (their
 * sum is of the unrounded ones), by 2^-8 of each at most: outputs are 2.3e-3 of their size off in the mean, where the rounding of the output
 * alone makes 1.7e-3.  Scores (scale q k) may be as large as 5e8 and values 1e24; beyond that outputs may be infinite, NaN or zero.
 * A key with a score of minus infinity is as one that is not seen; a score of infinity or NaN makes the row NaN.  An infinity in V makes the
 * output of the rows that see it that infinity, or NaN where its probability rounds to nothing; NaN in V, and infinities of both signs,
 * make it NaN.
 * scratch: device, 16-byte aligned, esp_paged_attn_scratch_bytes() bytes (0: it may be NULL), which depend on the host's values
 * alone, len_bound among them; calls that overlap in time need one each.  Results do not depend on what it held.
 * Errors: EINVAL (null pointers, scale below 1e-20 or not finite, ...), ESHAPE (n_q_heads not a multiple of n_kv_heads, anc_words * 64
 * < max_rows, q_stride), EDTYPE, ECAPACITY (scratch; more work than a launch can have, 2^24 workgroups). */
size_t esp_paged_attn_scratch_bytes(const esp_paged_kv *kv, const esp_chunk *rows, int32_t n_q_heads);
esp_status esp_paged_attn(void *stream, const esp_paged_kv *kv, int32_t layer, const esp_chunk *rows, int32_t n_q_heads,
                          const void *q, int64_t q_stride, float scale, const uint64_t *anc, int32_t anc_words, void *out,
                          void *scratch, size_t scratch_bytes);

/* After a verified block whose rows were appended: moves K and V of the accepted rows, in every layer, from slots len[b] +
 * accepted_row[b][i] to len[b] + i, i = 1 .. n_emit[b] - 1 (accepted_row[b][0], the root, sits at len[b] already), and writes
 * len_out[b] = len[b] + n_emit[b]; len_out may be kv->len.  accepted_row [batch][ESP_MAX_MASKS + 1] and n_emit [batch] are
 * laid out as esp_verify_accept's, which itself walks and moves in the contiguous cache only: over pages the caller finds the path,
 * from the root to each next row whose token is the choice made at the one before.  A path is ascending rows from 1 on, n_emit[b]
 * 0 .. ESP_MAX_MASKS + 1; of a sequence with another one nothing moves, len_out[b] = len[b], and ESP_DEV_BAD_PATH is set.
 * Errors: EINVAL. */
esp_status esp_paged_commit(void *stream, const esp_paged_kv *kv, const int32_t *n_emit, const int32_t *accepted_row,
                            int32_t *len_out);

/* How much attention the chunk's rows give to each token of their sequences, for esp_paged_evict: with p the softmax of esp_paged_attn (causal; K of
 * the rows is in its slots already), mass[t] = before[t] + the sum of p_rt over the sequence's counted rows r and the kv head's query heads, for
 * t < len[b]; the chunk's own tokens get the sum alone, whatever was there.  Slots from len[b] + rows on, and sequences without rows, are not touched.
 * After a verified tree: esp_paged_commit with a len_out of its own, then this with the accepted rows alone, packed, and len as it was before them; then len is
 * advanced.
 *   last_rows   0: all rows count; otherwise only the last so many of each sequence's
 *   before, mass device fp32 [n_layers][batch][n_kv_heads][mass_slots]; before NULL: zeros; it may be mass itself, and otherwise must not overlap it
 *   scratch     device, 16-byte aligned, esp_paged_weigh_scratch_bytes(), which depend on the host's values alone; calls that overlap in time need
 *               one each.  Up to 32 counted (row, query head) pairs a kv head it holds their scores, 4 bytes a pair (in fours), kv head and token of
 *               len_bound: a call with more rows can want less
 * Scores, probabilities and sums are fp32, tokens' sums always in the same order.  Scores may be as large as 5e8.  A row with a score of plus infinity or NaN makes all
 * tokens it sees NaN, in another row a score of minus infinity weighs nothing; a token in a page outside the pool is not seen (its mass is `before`).  A sequence
 * with len + rows above mass_slots is as one that is over its bound.
 * Errors: as esp_paged_attn; EINVAL also for last_rows < 0 and mass_slots < 1; ECAPACITY also for more than 65535 kv heads. */
size_t esp_paged_weigh_scratch_bytes(const esp_paged_kv* kv, const esp_chunk* rows, int32_t n_q_heads, int32_t last_rows);
esp_status esp_paged_weigh(void* stream, const esp_paged_kv* kv, int32_t layer, const esp_chunk* rows, int32_t n_q_heads, const void* q,
                           int64_t q_stride, float scale, int32_t last_rows, const float* before, float* mass, int32_t mass_slots, void* scratch,
                           size_t scratch_bytes);

/* Bounds what sequences keep: of one with len[b] > keep tokens the first `first`, the last `recent` and of the others those of greatest mass (equal ones: the
 * earlier; NaN is least) stay, `keep` in all, chosen for every layer and kv head by itself.  They move to slots 0 .. keep - 1 in their order, and
 * their masses with them; len_out[b] = keep.  Of the other sequences nothing is chosen, and len_out[b] = len[b].  Positions are in the rotated K already and
 * stay; a row that is appended next has its own position, no longer its slot.
 *   table_out   device [batch][table_out_stride]: pages that take the kept tokens.  A sequence's entry is either that of kv's page_table in the same place
 *               (then the block's tokens are moved within the page; page_table itself: all in place) or a page that no sequence reads in this call, for
 *               instance because the old one is shared.  Pages that are written must belong to one sequence
 *   mass_out    device fp32 [n_layers][batch][n_kv_heads][mass_out_slots], mass itself with the same mass_slots, or no overlap.  Slots from len_out on
 *               are left as they were
 *   len_out     device [batch], may be kv->len
 *   kept        device int32 [n_layers][batch][n_kv_heads][keep]: the old slots of the tokens, ascending, then -1
 * A kept token whose old page is outside the pool becomes zeros, one whose new page is is not written; both set ESP_DEV_BAD_PAGE.  A sequence with a length
 * that is negative, above len_bound, mass_slots or its table is left out: its kept are -1, its len_out its len.
 * Errors: EINVAL (null pointers, keep < 1, first or recent negative or together above keep, mass_out or table_out the input with other strides), ECAPACITY
 * (table_out or mass_out too small for keep, more than 4194303 layers x sequences x kv heads, keep or len_bound above 2^31 - 65537). */
esp_status esp_paged_evict(void* stream, const esp_paged_kv* kv, const float* mass, int32_t mass_slots, int32_t keep, int32_t first, int32_t recent,
                           const int32_t* table_out, int32_t table_out_stride, float* mass_out, int32_t mass_out_slots, int32_t* len_out,
                           int32_t* kept);

/* Copies slots first_slot .. of sequence seq, one layer, out of the pool to plain rows [n_slots][n_kv_heads][head_dim].
 * Slots of a page outside the pool come back as zeros.
 * Errors: EINVAL, ECAPACITY (slots past the table). */
esp_status esp_paged_load(void *stream, const esp_paged_kv *kv, int32_t layer, int32_t seq, int32_t first_slot, int32_t n_slots,
                          void *k_rows, void *v_rows);

/* Optional timing of launch sites with HIP events recorded on the ctx stream (benchmarks).
 * esp_profile_enable: bit s of site_mask turns site s on (0 = off, the default; events are host
 * objects, no device memory is allocated).  esp_profile_read: synchronises the stream, adds the
 * finished spans to per-site totals and returns, then clears, the totals of `site`. */
enum {
  ESP_SITE_GEMM_LAYER = 0, /* QKV, O, gate/up and down projections          */
  ESP_SITE_ATTN = 1,       /* tree attention main kernel                    */
  ESP_SITE_ATTN_MERGE = 2,
  ESP_SITE_LM_HEAD = 3,    /* LM-head GEMMs (tree rows and mask rows)       */
  ESP_SITE_TOPK = 4,       /* softmax + Top-K (both passes)                 */
  ESP_SITE_TREE = 5,       /* verify/commit, row lists, tree build          */
  ESP_SITE_GLUE = 6,       /* embed, norms, rotary/KV append, SwiGLU, argmax */
  ESP_SITE_COUNT = 7
};
esp_status esp_profile_enable(esp_ctx *ctx, uint32_t site_mask);
esp_status esp_profile_read(esp_ctx *ctx, int32_t site, int64_t *launches, double *total_ms);

#ifdef __cplusplus
}
#endif
#endif /* ESP_H_ */
