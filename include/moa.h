/*
 * moa.h -- C ABI of the Mixture-of-Attentions drafter hot path for one NVIDIA B200 (sm_100a).
 *
 * The library computes the drafter's forward step of "Mixture of Attentions for
 * Speculative Decoding" (arXiv 2410.03804): Layer Self-Attention over each token's
 * stack of per-layer LLM activations followed by a mean over layers (Section 3.1.1),
 * causal / tree-masked self-attention over token embeddings and cross-attention into
 * keys and values derived from the LSA output (Section 3.1.2, Algorithm 1), the LM head
 * with log-softmax and the B most probable tokens (Eq. 1), and the EAGLE-2-style dynamic
 * draft tree with its ancestor mask (Section 2.2). Target Layer Inference (Section 3.2)
 * is off after moa_create (TLI = 0: the drafter predicts the last decoder layer's
 * activation); moa_tli_configure turns it on for the last N <= MOA_MAX_TLI decoder layers.
 *
 * Conventions
 *  - Every pointer is DEVICE memory owned by the caller unless its name ends in _host or
 *    the comment says "host". The library allocates and frees no device memory.
 *  - Matrices are row-major [out, in]; there are no biases. "T" below is the storage type
 *    selected by moa_config.dtype (float or bfloat16); accumulation is always fp32.
 *  - Every call enqueues work on `stream` (a cudaStream_t passed as void*) and returns
 *    without synchronising. Results are valid once the caller has synchronised the stream.
 *  - Arguments are validated on the host before anything is launched; on error a status is
 *    returned and nothing is enqueued. No call throws, aborts or exits.
 *  - All device base pointers must be 16-byte aligned.
 *  - One moa_ctx may be used by one host thread at a time.
 */
#ifndef MOA_H_
#define MOA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MOA_MAX_BATCH 64      /* sequences per call */
#define MOA_MAX_TOPK 16       /* tree breadth B */
#define MOA_MAX_DEPTH 16      /* tree depth D */
#define MOA_MAX_TLI 4         /* LLM decoder layers run by the drafter (Target Layer Inference) */

typedef struct moa_ctx moa_ctx; /* opaque, host side */

typedef enum {
  MOA_OK = 0,
  MOA_ERR_NULL = 1,       /* a required pointer is NULL */
  MOA_ERR_SHAPE = 2,      /* a dimension is out of range or inconsistent */
  MOA_ERR_DTYPE = 3,
  MOA_ERR_ALIGN = 4,      /* a device pointer is not 16-byte aligned */
  MOA_ERR_WORKSPACE = 5,  /* workspace smaller than moa_state_bytes() reports */
  MOA_ERR_CAPACITY = 6,   /* a cache or the node pool would overflow */
  MOA_ERR_STATE = 7,      /* calls out of order (e.g. draft step before moa_tree_begin) */
  MOA_ERR_ARCH = 8,       /* the current device is not compute capability 10.x */
  MOA_ERR_CUDA = 9,       /* a CUDA runtime call failed; see moa_last_cuda_error() */
  MOA_ERR_TIMEOUT = 10,   /* a bounded device-side wait expired */
  MOA_ERR_NONFINITE = 11  /* moa_state_status only: a tree expansion met a log-probability that is not a number (it
                             ranked that candidate last); the drafted tree of that cycle is not to be trusted */
} moa_status;

typedef enum { MOA_F32 = 0, MOA_BF16 = 1 } moa_dtype;

typedef struct {
  int32_t d_model;   /* E: token embedding width = SA and CA width                         */
  int32_t n_stack;   /* S: activations stacked per token (the LLM's layers) fed to LSA     */
  int32_t d_stack;   /* D_in: width of one stacked activation = LSA width                  */
  int32_t vocab;     /* V                                                                  */
  int32_t head_dim;  /* dh, 64 or 128, shared by the three attentions                      */
  int32_t lsa_hq, lsa_hkv, lsa_mlp; /* heads (query / key-value) and MLP width, LSA block  */
  int32_t sa_hq, sa_hkv, sa_mlp;    /* ... self-attention block                            */
  int32_t ca_hq, ca_hkv, ca_mlp;    /* ... cross-attention block                           */
  int32_t max_batch; /* <= MOA_MAX_BATCH                                                   */
  int32_t max_ctx;   /* capacity of the caches, in positions per sequence                  */
  int32_t tree_topk; /* B <= MOA_MAX_TOPK                                                  */
  int32_t tree_depth;/* D <= MOA_MAX_DEPTH: number of drafter forwards per tree            */
  int32_t tree_keep; /* m: nodes kept for verification (the root is one more)              */
  float rms_eps;       /* RMSNorm epsilon, added to the mean square                        */
  float sa_rope_theta; /* rotary base of the self-attention; 0 disables the rotation       */
  int32_t dtype;       /* moa_dtype of weights, activations and caches                     */
} moa_config;

typedef struct { /* device pointers of type T */
  const void *embed, *lm_head, *final_norm;                 /* [V,E] [V,E] [E] */
  const void *lsa_norm1, *lsa_wq, *lsa_wk, *lsa_wv, *lsa_wo; /* [D_in] [Hq*dh,D_in] [Hkv*dh,D_in] x2 [D_in,Hq*dh] */
  const void *lsa_norm2, *lsa_wgate, *lsa_wup, *lsa_wdown;  /* [D_in] [F,D_in] [F,D_in] [D_in,F] */
  const void *sa_norm1, *sa_wq, *sa_wk, *sa_wv, *sa_wo;     /* as above with E in place of D_in */
  const void *sa_norm2, *sa_wgate, *sa_wup, *sa_wdown;
  const void *ca_normq, *ca_normkv;                         /* [E] [D_in] */
  const void *ca_wq, *ca_wk, *ca_wv, *ca_wo;                /* [Hq*dh,E] [Hkv*dh,D_in] x2 [E,Hq*dh] */
  const void *ca_norm2, *ca_wgate, *ca_wup, *ca_wdown;
} moa_weights;

typedef struct {
  void *ca_k, *ca_v;        /* T [max_batch, max_ctx, ca_hkv, head_dim]: cross-attention keys / values   */
  void *sa_k, *sa_v;        /* T [max_batch, max_ctx, sa_hkv, head_dim]: rotated self-attention prefix   */
  int32_t *ca_len, *sa_len; /* device int32 [max_batch]: valid positions; written only by the library    */
  void *tree;               /* device blob of moa_state_bytes().tree_bytes: node pool, frontier, tree K/V, barrier
                               words of the fused kernels. ZERO IT ONCE after allocating it (and again after a call
                               reported MOA_ERR_TIMEOUT through moa_state_status) */
  int32_t *ca_len_host, *sa_len_host; /* HOST int32 [max_batch]: mirrors kept by the library             */
  int32_t step;             /* HOST: draft steps done since moa_tree_begin, -1 before it; library-owned  */
} moa_state;

/* Creates a context for the CURRENT device. Copies config and weight pointers (not the weights).
 * MOA_ERR_ARCH if the device is not compute capability 10.x: there is no fallback path. */
moa_status moa_create(const moa_config *cfg, const moa_weights *w, moa_ctx **out);
void moa_destroy(moa_ctx *ctx);

/* Target Layer Inference (Section 3.2; Algorithm 1, the loop over the last N decoder layers): with TLI = N > 0
 * the drafter's CA block predicts the input of LLM layer L+1-N, and moa_draft_step then runs the N last
 * (frozen) LLM decoder layers on the drafted rows before the LM head. Layer l attends over the LLM's own
 * key/value cache of that layer for the positions already decoded (0 .. sa_len[b]-1, the same positions as the
 * drafter's self-attention prefix) and over the keys/values of the row's drafted ancestors and itself, which
 * the library keeps in moa_state.tree for the duration of one tree and drops afterwards.
 * A layer is a Llama decoder layer: RMSNorm(norm1) -> q,k,v projections -> rotary embedding (half-split
 * pairing, base rope_theta) at the row's position -> grouped-query attention -> W_o, residual ->
 * RMSNorm(norm2) -> SwiGLU MLP, residual. Width E = d_model, head size = moa_config.head_dim.
 *   layers  HOST array [n_layers], layers[0] = the earliest of the N (LLM layer L+1-N); device pointers of T:
 *           norm1 [E], wq [hq*dh,E], wk, wv [hkv*dh,E], wo [E,hq*dh], norm2 [E], wgate, wup [mlp,E], wdown [E,mlp]
 *   k, v    device T [max_batch, max_ctx, hkv, head_dim] per layer: the LLM's cache of that layer (keys already
 *           rotated), owned and filled by the caller, never written by the library
 * Call it before moa_state_bytes: both sizes grow. n_layers = 0 (layers and caches may be NULL) turns it off
 * again.
 * MOA_ERR_SHAPE for n_layers > MOA_MAX_TLI, hq % hkv != 0, mlp % 16 != 0. */
typedef struct {
  int32_t n_layers;  /* N = TLI, 0 .. MOA_MAX_TLI */
  int32_t hq, hkv;   /* query / key-value heads of an LLM layer */
  int32_t mlp;       /* its MLP width */
  float rope_theta;  /* its rotary base; 0 disables the rotation */
} moa_tli_config;
typedef struct {
  const void *norm1, *wq, *wk, *wv, *wo, *norm2, *wgate, *wup, *wdown;
} moa_tli_layer;
typedef struct {
  const void *k[MOA_MAX_TLI], *v[MOA_MAX_TLI];
} moa_tli_caches;
moa_status moa_tli_configure(moa_ctx *ctx, const moa_tli_config *cfg, const moa_tli_layer *layers_host,
                             const moa_tli_caches *caches);

/* Sizes in bytes of moa_state.tree and of the workspace every compute call needs.
 * lsa_chunk_tokens (>= 1) is the number of tokens moa_lsa_forward processes per internal
 * pass; a larger value needs a larger workspace. */
moa_status moa_state_bytes(const moa_ctx *ctx, int32_t lsa_chunk_tokens, size_t *tree_bytes, size_t *workspace_bytes);

const char *moa_status_str(moa_status s);
const char *moa_last_cuda_error(void); /* text of the last CUDA error seen by this thread's calls */

/* Sets the valid length of the caches of sequences 0..batch-1 (device and host copies), e.g. after
 * the caller filled a cache itself or dropped rejected positions. which: 0 = ca, 1 = sa. */
moa_status moa_state_set_len(moa_ctx *ctx, moa_state *st, int32_t which, const int32_t *len_host, int32_t batch, void *stream);

/* Layer Self-Attention with mean, then the cross-attention key/value projection
 * (Section 3.1.1; Algorithm 1: kv <- LSA_layer_with_mean(h), kv <- (kv, kv')).
 *   h_stack    T [sum n_tok, S, D_in], sequences back to back
 *   n_tok_host HOST int32 [batch], tokens of each sequence (may be 0)
 *   kv_out     T [sum n_tok, D_in] or NULL: the LSA output rows
 * Appends n_tok[b] rows W_k n(kv), W_v n(kv) to ca_k / ca_v of sequence b at position ca_len[b]
 * and advances ca_len. MOA_ERR_CAPACITY if ca_len[b] + n_tok[b] > max_ctx. */
moa_status moa_lsa_forward(moa_ctx *ctx, moa_state *st, const void *h_stack, const int32_t *n_tok_host, int32_t batch,
                           void *kv_out, void *ws, size_t ws_bytes, void *stream);

/* Self-attention prefix for prompt / accepted tokens (Section 3.1.2 "Self-Attention"): embeds the
 * tokens, projects keys and values, rotates keys at positions sa_len[b], sa_len[b]+1, ... and
 * appends them to sa_k / sa_v.   tok: device int32 [sum n], n_host: HOST int32 [batch]. */
moa_status moa_sa_append(moa_ctx *ctx, moa_state *st, const int32_t *tok, const int32_t *n_host, int32_t batch,
                         void *ws, size_t ws_bytes, void *stream);

/* The drafter over whole token sequences in one pass (Section 3.1.2: self-attention with its causal mask over
 * prompt + response, cross-attention into the cached LSA keys / values; the parallel pass the paper trains the
 * drafter with, and a way to score many positions at once). Token i of sequence b sits at position sa_len[b] + i:
 * it sees the prefix and tokens 0..i in self-attention; in cross-attention it sees the first ca_limit[row] cached
 * positions (the K-step-bounded mask of the mask figure: the LLM activations available when that token is drafted),
 * or all ca_len[b] of them when ca_limit is NULL (the generation-time setting).
 *   tok        device int32 [sum n], sequences back to back;  n_host  HOST int32 [batch]
 *   ca_limit   device int32 [sum n] or NULL; values in 0 .. ca_len[b], non-decreasing within a sequence
 *   hidden_out T [sum n, E]: the drafter's output activation of every position (the LM head's input)
 * Appends the tokens' self-attention keys / values to sa_k / sa_v and advances sa_len, as moa_sa_append does.
 * Target Layer Inference and the LM head are not applied here. MOA_ERR_CAPACITY if the prefix would overflow. */
moa_status moa_drafter_prefill(moa_ctx *ctx, moa_state *st, const int32_t *tok, const int32_t *n_host, int32_t batch,
                               const int32_t *ca_limit, void *hidden_out, void *ws, size_t ws_bytes, void *stream);

/* The same operation as moa_sa_append for callers that cannot provide a workspace because they cannot
 * allocate device memory at that point: code running between other components that have already handed
 * all device memory to their own pools, or a serving loop in which a cudaMalloc (a device-wide
 * synchronisation) is not allowed. The paper has no counterpart; this is a convenience of the library.
 * Its scratch is a fixed array inside the library (4.5 MiB of device memory, held by every GPU on which
 * the library is loaded, until the process exits), so the call allocates and frees nothing. Inputs and
 * outputs are still the caller's: tok, the caches in st.
 *   Limits: sum(n_host) <= MOA_SA_STATIC_MAX_TOKENS, rows * d_model * sizeof(T) <= 512 KiB (rows = sum(n_host),
 *   on bf16 plus that count rounded up to 16, 32, 64 or 128 for the low-order terms of the activations) and
 *   sum(n_host) * 2 * sa_hkv * head_dim * 4 <= 4 MiB; beyond them MOA_ERR_WORKSPACE is returned, nothing
 *   is launched, and moa_last_cuda_error() holds the limits in words.
 *   The first call on a device looks up the array's device address (a CUDA runtime query made with that
 *   device current); make that first call outside any stream capture.
 *   All calls on one device share the array. It keeps the previous call's contents; nothing in it has
 *   to start at zero, because every element a call reads was written earlier in the same call. Two calls
 *   whose kernels can overlap on the GPU (different streams) race on it: serialise them. */
#define MOA_SA_STATIC_MAX_TOKENS 32
moa_status moa_sa_append_static(moa_ctx *ctx, moa_state *st, const int32_t *tok, const int32_t *n_host, int32_t batch,
                                void *stream);

/* Starts a draft tree per sequence (Section 2.2). root_tok: device int32 [batch], the last verified
 * token; it sits at position sa_len[b]. Sets st->step = 0. */
moa_status moa_tree_begin(moa_ctx *ctx, moa_state *st, const int32_t *root_tok, int32_t batch, void *stream);

/* One drafter forward for the current frontier (Algorithm 1, the SA_layer, CA_layer and LM_head
 * steps of the inner loop; Eq. 1): R = batch rows at step 0 (the roots), batch*B afterwards, row
 * b*B + r = r-th frontier node of sequence b. A row at depth d sits at position sa_len[b] + d and
 * sees the prefix, its ancestors and itself.
 *   topk_id    int32 [R, B]  token ids, by (log-probability descending, id ascending)
 *   topk_logp  float [R, B]  their log-probabilities (logit - logsumexp over the vocabulary)
 *   hidden_out T [R, E] or NULL: the drafter's output activation (input of the LM head; with Target Layer
 *              Inference on, the output of the last LLM decoder layer) */
moa_status moa_draft_step(moa_ctx *ctx, moa_state *st, int32_t batch, int32_t *topk_id, float *topk_logp,
                          void *hidden_out, void *ws, size_t ws_bytes, void *stream);

/* Expands the tree with the rows' top-B lists (Section 2.2): child score = parent score + logp
 * (fp32), children appended in (row, rank) order, next frontier = top B children by (score
 * descending, pool index ascending). Advances st->step. After the D-th expansion it also selects
 * the m best pool nodes (same order), lists them by pool index behind the root (slot 0) and, if the
 * out_* pointers are non-NULL, writes int32 / float [batch, m+1] arrays (parent = slot number,
 * root's parent = -1; unused tail slots hold -1 / 0) and out_n [batch] = 1 + nodes kept. */
moa_status moa_tree_expand(moa_ctx *ctx, moa_state *st, int32_t batch, const int32_t *topk_id, const float *topk_logp,
                           int32_t *out_tok, int32_t *out_parent, int32_t *out_depth, float *out_score, int32_t *out_n,
                           void *stream);

/* Tree Attention mask (Section 2.2, verification with Tree Attention): mask[b][i][j] = 1 iff j == i or
 * j is an ancestor of i. parent: device int32 [batch, n] with parent[0] = -1 and parent[i] < i; an
 * entry < 0 at i > 0 marks an unused slot (its row is zero).
 * packed = 0: uint8 [batch, n, n]; packed = 1: uint64 [batch, n, ceil(n/64)], bit j%64 of word j/64. */
moa_status moa_tree_attn_mask(const int32_t *parent, int32_t batch, int32_t n, void *mask_out, int32_t packed, void *stream);

/* Greedy verification of the kept tree (Section 2.2, step 2: exact matching, everything after the first mismatch
 * is discarded; Algorithm 1, the step that identifies the K' verified tokens and the LLM's next token y').
 * The LLM itself is not part of the library: the caller runs it once over the kept tree with the mask of
 * moa_tree_attn_mask and passes its logits.
 *   tok, parent    device int32 [batch, n]: the kept tree as moa_tree_expand wrote it (slot 0 = root, parent[0] = -1,
 *                  parent[i] < i, parent[i] < 0 at i > 0 = unused slot)
 *   target_logits  device [batch, n, vocab] of logits_dtype (moa_dtype): row (b, i) scores the token FOLLOWING slot i
 *   choice         device int32 [batch, n] out: arg-max of every row, ties to the smallest id (the row of an
 *                  unused slot is read like any other)
 *   acc_slot, acc_tok  device int32 [batch, cap] out: slots and tokens of the accepted path, root first, -1 behind it
 *   acc_len        device int32 [batch] out: 1 + K' (root included), at most cap
 *   next_tok       device int32 [batch] out: the LLM's choice at the last accepted slot = the next cycle's root
 * cap >= 1 bounds the path length (tree_depth + 1 covers every tree of this library). batch * n <= 65535. To carry the accepted
 * tokens into the drafter's self-attention prefix, pass acc_tok's first acc_len entries to moa_sa_append. */
moa_status moa_verify_greedy(const int32_t *tok, const int32_t *parent, int32_t batch, int32_t n, const void *target_logits,
                             int32_t logits_dtype, int32_t vocab, int32_t cap, int32_t *choice, int32_t *acc_slot,
                             int32_t *acc_tok, int32_t *acc_len, int32_t *next_tok, void *stream);

/* Client-server message codec (Section 4.2 "Client-Server" and the message-size table of the appendix).
 * moa_pack_tree: every node of the kept tree as 4 bytes -- the token id in 3 bytes, little endian, and 1 byte for
 * its position in the tree, here the parent's slot number -- so a tree of M nodes is a 4M-byte message. A negative
 * token id is written as ff ff ff, a negative parent (the root, an unused slot) as 255; token ids must be below
 * 2^24 - 1 and slots below 255 (larger values are truncated to their low bits).
 *   tok, parent  device int32 [count]      msg  device bytes [count, 4], 4-byte aligned
 * moa_unpack_tree is the inverse. */
moa_status moa_pack_tree(const int32_t *tok, const int32_t *parent, int64_t count, void *msg, void *stream);
moa_status moa_unpack_tree(const void *msg, int64_t count, int32_t *tok, int32_t *parent, void *stream);
/* 8-bit quantisation of activation rows (the E / E_kv tensors the server sends, Section 4.2). The paper names no
 * scheme; this one is symmetric with one fp32 scale per row: scale = max|x| / 127, code = round-half-even(x * r)
 * in [-127, 127] with r = 127 / max|x| (one fp32 reciprocal per row, one fp32 product per element), decided in fp32; an all-zero row has scale 0 and codes 0. moa_dequantize_rows writes
 * code * scale in `dtype`.
 *   x / out  device [rows, width] of dtype (moa_dtype)    codes  device int8 [rows, width]    scales  device float [rows] */
moa_status moa_quantize_rows(const void *x, int32_t dtype, int64_t rows, int32_t width, int8_t *codes, float *scales,
                             void *stream);
moa_status moa_dequantize_rows(const int8_t *codes, const float *scales, int64_t rows, int32_t width, void *out,
                               int32_t dtype, void *stream);

/* ---------------------------------------------------------------------------------------------------------------
 * Serving operators around the drafter: a paged key / value cache with the attention of new rows over it, its eviction,
 * and the rules between the LLM's logits and their verification. One cycle with a kept tree:
 *   per LLM layer  moa_paged_attention (appends the tree's rows and attends), later moa_paged_commit (keeps the accepted path)
 *   per cycle      moa_verify_greedy_rules on the logits, moa_token_record on the accepted tokens
 *   now and then   moa_paged_evict
 * and without drafting the same calls with one row per sequence. None of them needs a moa_ctx. They run on the current
 * device, and `stream` has to belong to it. Lengths, tables and penalties are read on the device when a call's kernels run,
 * so a captured call can be replayed while they change. Two calls that may overlap (different streams, two captured graphs)
 * need workspaces of their own.
 *
 * A cache of one attention layer. Slot j of sequence b lies on page page_table[b][j / page_size], row j % page_size. Keys are
 * stored as they enter the scores (already rotated). Slots 0 .. len[b]-1 are committed; len[b] < 0 marks a sequence that is
 * not in use: no call reads, writes or advances anything of it, its rows of an output stay as they were. len and seen may be
 * shared by the layers of a model; the calls take the new rows to lie behind len, and only moa_paged_commit with advance
 * and moa_paged_evict with len_out move it. Positions on a page whose table entry is outside 0 .. n_pages-1 are left out,
 * as are those behind the last slot, max_pages * page_size. The pages of a sequence must not be shared with another one
 * where they are written. */
typedef struct {
  void *k, *v;               /* T [n_pages, page_size, hkv, head_dim]; page p starts page_stride * p elements in */
  int64_t page_stride;       /* elements, >= page_size * hkv * head_dim, a multiple of 16 bytes (k and v may share blocks) */
  const int32_t *page_table; /* device int32 [batch, max_pages] */
  int32_t *len;              /* device int32 [batch] */
  float *weight;             /* device [batch, hkv, max_pages * page_size]: accumulated attention weights, or NULL */
  int32_t *pos;              /* device, the same shape: position that each slot's token had; NULL, or with weight and seen */
  int32_t *seen;             /* device int32 [batch]: positions appended so far = the next row's position; or NULL */
  int32_t batch;             /* <= MOA_MAX_BATCH */
  int32_t max_pages, n_pages;
  int32_t page_size;         /* a power of two <= 1024; max_pages * page_size <= 2^30 */
  int32_t hkv, head_dim;     /* head_dim 64 or 128 */
  int32_t dtype;             /* moa_dtype of k, v and of the rows */
} moa_paged_cache;

#define MOA_PAGED_MAX_ROWS 64 /* new rows per sequence: the slots that one packed mask word of moa_tree_attn_mask holds */

/* Writes rows i < n_new[b] (all n when n_new is NULL; device int32 [batch]) of k_new, v_new T [batch, n, hkv, head_dim] to
 * slots len[b] + i, without changing len. Rows lie row_stride elements apart (>= hkv * head_dim, a multiple of 16 bytes), so
 * that they may be a part of a fused projection. With pos, the slots get positions seen[b] + i and weight 0. n is not
 * bounded: a whole prompt may be appended. */
moa_status moa_paged_append(const moa_paged_cache *cache, const void *k_new, const void *v_new, int64_t row_stride, int32_t n,
                            const int32_t *n_new, void *stream);

/* Attention of n new rows per sequence (n = 1: the next token; up to MOA_PAGED_MAX_ROWS: a kept tree):
 *   out[b, i, h] = sum_j softmax_j(scale * q[b, i, h] . k_j) v_j
 * over the slots j < len[b] and, when n_new = n, the rows' own slots len[b] + j' that row i sees: bit j' of mask[b, i]
 * (device uint64 [batch, n], as moa_tree_attn_mask packs it for n <= 64), or j' <= i when mask is NULL. n_new = 0: the
 * committed slots only, as in a cross-attention. A row whose mask word is 0 (an unused slot) sees nothing, and a row that
 * sees nothing gives zeros. A new slot that no row sees is not read, and infinities and NaN among a slot's values reach the
 * rows that see it only.
 *   q           T [batch, n, hq, head_dim], rows q_stride elements apart; head h belongs to key / value head h / (hq / hkv)
 *   k_new,v_new T [batch, n, hkv, head_dim], rows new_stride elements apart: appended by this call as moa_paged_append
 *               would (keys and values of slots that no row sees are not written), or NULL when the rows are in the pages already
 *   scale       0 means 1 / sqrt(head_dim); at most 2e38
 *   out         T [batch, n, hq, head_dim]
 *   weight_out  device float [batch, hkv, max_pages * page_size], may be cache->weight, or NULL; n = 1 only: for every slot
 *               that the row sees, cache->weight (0 for the new slot, or without it) + the sum over the group's query heads
 *               of the softmax weights. Other entries stay as they were.
 *   ws          device scratch of moa_paged_workspace_bytes bytes. ZERO IT ONCE after allocating it: its first bytes count the
 *               parts of the work that have been joined, and a call leaves them at zero again
 * Scores, statistics and sums are fp32. bf16 values are multiplied by probabilities of two bf16 terms; calls of many query rows
 * (n > 1, more than 16 of them per key / value head, pages of at least 8 rows, and a cache with room for enough work, by its size
 * and not by the lengths) run on tensor memory and round each probability once to bf16, which puts an output off by at most 2^-8
 * of sum p |v|. A wait inside that kernel that runs out (about 2 s; it means a fault of the device) leaves NaN in the rows
 * concerned: these calls have no status word. hq / hkv <= 128; batch * hkv * (n * hq / hkv / 8, rounded up) * (max_pages *
 * page_size / 64, rounded up) <= 2^30. */
moa_status moa_paged_workspace_bytes(const moa_paged_cache *cache, int32_t n, int32_t hq, int32_t weights, size_t *bytes);
moa_status moa_paged_attention(const moa_paged_cache *cache, const void *q, int64_t q_stride, const void *k_new, const void *v_new,
                               int64_t new_stride, int32_t n, int32_t n_new, int32_t hq, const uint64_t *mask, float scale, void *out,
                               float *weight_out, void *ws, size_t ws_bytes, void *stream);

/* Ends a cycle for n uncommitted rows. With acc_slot (device int32 [batch, cap]) and acc_len (device int32 [batch]), as
 * moa_verify_greedy writes them: the accepted rows' keys and values move to slots len[b] .. len[b] + acc_len[b] - 1, the
 * others are given up (n <= MOA_PAGED_MAX_ROWS; the listed slots rise). The pages of the n rows have to be in the table: of a
 * row on a missing page nothing is stored, so it cannot be kept; a listed row that comes from such a page leaves its new slot
 * as it was, one that goes to such a page is lost, and the other listed rows are kept all the same. advance != 0: len (and
 * seen) grow by acc_len, or by n when acc_len is NULL. With several layers that share len: the layers' calls without advance, then one with it. */
moa_status moa_paged_commit(const moa_paged_cache *cache, int32_t n, const int32_t *acc_slot, const int32_t *acc_len, int32_t cap,
                            int32_t advance, void *stream);

/* Eviction by accumulated attention weight. Of a sequence with len[b] > budget every key / value head keeps budget slots of
 * its own: those of positions < sink and >= seen[b] - recent, and of the others the ones with the largest weight (a NaN
 * after all numbers, equal weights by the lower slot). The kept slots behind the budget move to the freed slots before it,
 * both in rising order; slots from the budget on are free afterwards. Slots on a page that the table does not have hold no
 * row: behind the budget they are given up before all others; before it they stay as they are and count towards it. Only
 * calls of one row per sequence accumulate weights: a slot that came in with a tree, or a prompt, has weight 0 until tokens
 * attended to it, and where all weights are equal the lowest slots are kept beside the protected positions. Needs
 * cache->weight, pos and seen; sink + recent <= budget.
 *   weight_out, pos_out  shaped as cache->weight and pos and may be them: entries of the slots in use afterwards
 *   len_out     device int32 [batch], may be cache->len, or NULL: min(len, budget), so the negative length of a sequence that is
 *               not in use
 *   ws          device scratch of moa_paged_evict_workspace_bytes bytes */
moa_status moa_paged_evict_workspace_bytes(const moa_paged_cache *cache, int32_t budget, size_t *bytes);
moa_status moa_paged_evict(const moa_paged_cache *cache, int32_t budget, int32_t sink, int32_t recent, float *weight_out, int32_t *pos_out,
                           int32_t *len_out, void *ws, size_t ws_bytes, void *stream);

/* The record of the tokens that a sequence holds, for the penalties: counts device int32 [batch, vocab] and seen device
 * uint32 [batch, ceil(vocab / 32)] (bit t % 32 of word t / 32), both zeroed by the caller for a new sequence. Adds tokens
 * tok[b][0 .. n_tok[b]-1] (device int32 [batch, cap]; n_tok device int32 [batch], NULL: all cap): their bits in seen, and 1
 * each in counts. A prompt, which only the repetition penalty counts, is added with counts NULL. Tokens outside
 * 0 .. vocab-1 are left out, so acc_tok of moa_verify_greedy can be passed as it is. vocab <= 2^20. */
moa_status moa_token_record(int32_t *counts, uint32_t *seen, int32_t batch, int32_t vocab, const int32_t *tok, const int32_t *n_tok, int32_t cap,
                            void *stream);

/* Rules for logits. Every pointer may be NULL (that rule is off). */
typedef struct {
  const int32_t *counts;     /* device int32 [batch, vocab]: times each token was generated */
  const uint32_t *seen;      /* device uint32 [batch, ceil(vocab / 32)]: tokens of prompt and answer. With seen, counts are
                                read where its bit is set only; without it, a token is in the context when its count > 0 */
  const float *repetition;   /* device float [batch]: divides positive and multiplies other logits of the context's tokens */
  const float *frequency;    /* device float [batch]: subtracted once per generation */
  const float *presence;     /* device float [batch]: subtracted when generated at all */
  const int32_t *bias_id;    /* device int32 [batch, n_bias]; ids outside 0 .. vocab-1 mark unused entries */
  const float *bias_value;   /* device float [batch, n_bias]: added; the values of an id that is listed twice are summed in order */
  const uint32_t *allow;     /* device uint32 [batch, n, ceil(vocab / 32)]: a token whose bit is 0 gets -inf, whatever its logit */
  int32_t n_bias;            /* <= 1024 */
} moa_logit_rule_set;

/* Applies the rules to logits [batch, n, vocab] of logits_dtype, in the order of the struct, in fp32, each step rounded once;
 * out (the logits' type, may be the logits themselves, or NULL) gets the result rounded once, choice (device int32 [batch, n]
 * or NULL) the arg-max of the unrounded result: ties to the smallest id, NaN never, and 0 when nothing is above -inf.
 * With tok and parent (device int32 [batch, n], a kept tree as moa_tree_expand writes it, n <= 256) the tokens on the path
 * from the root to slot i, both included, count as generated for row i: the record holds the tokens before the root. The row
 * of an unused slot has no path. batch * n <= 65535, vocab <= 2^20. */
moa_status moa_logit_rules(const moa_logit_rule_set *rules, const int32_t *tok, const int32_t *parent, int32_t batch, int32_t n,
                           const void *logits, int32_t logits_dtype, int32_t vocab, void *out, int32_t *choice, void *stream);
/* moa_verify_greedy with the choices of moa_logit_rules; no adjusted logits are written. */
moa_status moa_verify_greedy_rules(const moa_logit_rule_set *rules, const int32_t *tok, const int32_t *parent, int32_t batch, int32_t n,
                                   const void *target_logits, int32_t logits_dtype, int32_t vocab, int32_t cap, int32_t *choice,
                                   int32_t *acc_slot, int32_t *acc_tok, int32_t *acc_len, int32_t *next_tok, void *stream);

/* Reads back the device status word kept in st->tree (0 = no device-side problem seen). Synchronises the stream. */
moa_status moa_state_status(moa_ctx *ctx, moa_state *st, void *stream);

/* Measurement hooks (no counterpart in the paper). Between moa_profile_begin and moa_profile_end every
 * launch of the LM-head kernel (the step's dominant HBM stream, Eq. 1) is bracketed by CUDA events on the
 * caller's stream; moa_profile_end synchronises those events and returns their summed duration in
 * milliseconds and the number of launches timed (at most 512 per begin/end pair; later ones are skipped).
 * Do not use inside a stream capture. */
moa_status moa_profile_begin(moa_ctx *ctx);
moa_status moa_profile_end(moa_ctx *ctx, double *ms_total, int32_t *launches);
/* Phase timing of the LAST dense LSA pass (on the bf16 path an LSA pass of more than 256 (token, layer) rows runs as
 * one persistent kernel made of phases separated by grid-wide barriers). Valid when that launch was made between
 * moa_profile_begin and moa_profile_end with the same workspace. us_out[i] = microseconds phase i took on CTA 0
 * including its closing barrier, wait_us_out[i] (may be NULL) = the part of it CTA 0 spent in that barrier,
 * kind_out[i] = its kind (0 GEMM, 1 row norm, 2 residual + norm, 3 layer mean + norm, 4 cache append,
 * 5 layer self-attention).
 * Synchronises the stream. HOST output arrays of `cap` entries. */
moa_status moa_profile_phases(moa_ctx *ctx, const void *ws, size_t ws_bytes, int32_t cap, double *us_out,
                              double *wait_us_out, int32_t *kind_out, int32_t *n_out, void *stream);
/* Kernels launched so far by this host thread through the library. */
int64_t moa_launch_count(void);
/* Stage trace (no counterpart in the paper; only in a library built with -DMOA_TRACE, otherwise both calls return
 * MOA_ERR_STATE and the kernels carry no trace code). Between the two calls every kernel of the library stores one
 * entry when its first thread is released by the completion of the kernel before it in the stream:
 * dev_buf[2 i] = the GPU's nanosecond timer, dev_buf[2 i + 1] = kernel id << 32 | gridDim.x (ids: 1 embedding,
 * 2 GEMM, 3 attention, 4 attention merge, 5 LM-head merge, 6 tree expansion, 7 row norm, 8 residual + norm,
 * 9 SwiGLU, 10 sum + cast, 11 rotary, 12 cache append, 13 layer mean, 0 other). The difference of two consecutive
 * entries is what the earlier kernel cost inside the chain. dev_buf: device uint64 [2 * cap], caller-owned.
 * moa_trace_end synchronises the device and returns the number of entries made (entries beyond cap are dropped). */
moa_status moa_trace_begin(void *dev_buf, int32_t cap);
moa_status moa_trace_end(int32_t *n_out);

#ifdef __cplusplus
}
#endif
#endif /* MOA_H_ */
