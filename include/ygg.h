/*
 * ygg.h -- C ABI of the MI355X (gfx950) tree-verification library.
 *
 * Three operations make up one verification step of a static-shape, equal-growth
 * draft token tree (Yggdrasil, arXiv 2512.23858):
 *
 *   ygg_equal_growth_expand   one draft step of the Equal-Growth Tree (Sec. 4.2)
 *   ygg_tree_attention        tree-masked attention of the verifier pass (Sec. 2, Sec. 4.2)
 *   ygg_accept_and_compact    acceptance of the matching draft path (Sec. 1, Sec. 5) and the
 *                             TokenTree's K/V bookkeeping (Sec. 6), done on the device
 *
 * Around them: ygg_equal_growth_attach (the same draft step with free attachment, Sec. 4.2),
 * ygg_prune_for_verification (verification-width pruning, Sec. 4.2), and ygg_debug_validate, which
 * reports the data-dependent contract violations that the three calls above do not check.
 *
 * What a decode step needs beside them:
 *
 *   ygg_tree_rotary           rotary positions of a tree's (or a prompt's) queries and keys
 *   ygg_tree_attention_block8 the verifier's attention over a cache in 8 bits with a scale per 64 tokens and head
 *   ygg_block8_append         writes accepted (or prompt) tokens into that cache
 *   ygg_constrain_logits      penalties, biases and grammar masks on logits, node by node, and their first maxima
 *   ygg_count_tokens          the counts of confirmed tokens that the penalties go by
 *
 * A prompt's way into the cache, and a cache in 4 bits:
 *
 *   ygg_tree_norm_rotary      RMS norms of every head of the queries and keys and their rotary positions, in one pass
 *   ygg_prompt_attention      causal attention of whole prompts, or of the next chunk of them, sequences of different lengths
 *   ygg_block4_append         writes accepted (or prompt) tokens into a cache in 4 bits with a scale per 32 values
 *   ygg_tree_attention_block4 the verifier's attention (or plain decoding) over that cache
 *
 * Conventions shared by every call
 *   - All tensor pointers are DEVICE pointers owned by the caller; the ygg_shape struct is HOST
 *     memory and is only read during the call.  The library never allocates, frees or keeps
 *     device memory; scratch space is the caller's `workspace` (size from ygg_workspace_bytes,
 *     256-byte aligned, contents undefined on entry and on return).  Calls that may run
 *     concurrently need workspaces of their own.
 *   - Calls only enqueue kernels on `hip_stream` (a hipStream_t passed as void*; NULL = the
 *     default stream) and never synchronise, so a sequence of calls can be captured in a HIP
 *     graph.  All shapes are static: nothing on the host depends on device data.  This is the
 *     static-runtime property the paper asks of the drafting algorithm (Sec. 3, Sec. 4.2).
 *     The first launching call on a device (or ygg_init) raises the dynamic shared-memory limits
 *     of the library's kernels, once, under a lock; call ygg_init before capturing if the first
 *     call of a process would otherwise be made under stream capture.  That per-device flag is
 *     the library's only state.
 *   - The return code reports host-checkable errors only (null pointers, inconsistent shape,
 *     unsupported type, workspace too small, launch failure).  Data-dependent contract
 *     violations (parent_idx not topological, seq_lens[b] > max_seq_len, NaN logits) are
 *     undefined behaviour, except that no kernel reads or writes outside the buffers as
 *     described by ygg_shape; ygg_debug_validate reports them.
 *   - Tensors are dense, row-major, token-major: [.., token, head, head_dim].
 *   - Tree layout: node 0 is the root (the last confirmed token, whose K/V is not yet in the
 *     cache); parent_idx[b][0] = -1 and 0 <= parent_idx[b][i] < i.  For the expansion call the
 *     tree is level structured: depth d (1..D) occupies nodes 1+(d-1)W .. dW, N = 1 + D*W.
 *     Attention and acceptance accept any topologically ordered tree of N nodes whose depth
 *     does not exceed `depth`.
 */
#ifndef YGG_H
#define YGG_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    YGG_OK = 0,
    YGG_ERR_NULL = 1,        /* a required pointer is NULL */
    YGG_ERR_SHAPE = 2,       /* inconsistent or out-of-range shape field / argument */
    YGG_ERR_UNSUPPORTED = 3, /* dtype / head_dim / size outside what the kernels implement */
    YGG_ERR_WORKSPACE = 4,   /* workspace missing, misaligned or too small */
    YGG_ERR_LAUNCH = 5       /* the HIP runtime refused a launch */
} ygg_status;

typedef enum {
    YGG_F32 = 0,
    YGG_BF16 = 1,
    YGG_FP8_E4M3 = 2,  /* K and V (cache and tree) as 8-bit E4M3 codes, Q and O bf16; head_dim 128;
                          accepted by ygg_tree_attention_fp8kv and ygg_accept_and_compact only */
    YGG_FP8_BLOCK = 3, /* the cache is a ygg_block8_cache, everything else is bf16; accepted by
                          ygg_tree_attention_block8, ygg_block8_append and ygg_tree_rotary, and by
                          ygg_accept_and_compact with n_layers = 0 */
    YGG_FP4_BLOCK = 5  /* the cache is a ygg_block4_cache, everything else is bf16; accepted by ygg_tree_attention_block4,
                          ygg_block4_append, ygg_tree_norm_rotary and ygg_tree_rotary, and by ygg_accept_and_compact with
                          n_layers = 0 (4 is no type) */
} ygg_dtype;

typedef enum {
    YGG_OP_ATTENTION = 0, YGG_OP_EXPAND = 1, YGG_OP_ACCEPT = 2, YGG_OP_ATTACH = 3,
    YGG_OP_ATTENTION_BLOCK8 = 4, YGG_OP_CONSTRAIN = 5, YGG_OP_ATTENTION_BLOCK4 = 6, YGG_OP_PROMPT_ATTENTION = 7
} ygg_op;

typedef struct {
    int32_t batch;         /* B >= 1 sequences, one tree each */
    int32_t n_q_heads;     /* Hq */
    int32_t n_kv_heads;    /* Hkv, Hq % Hkv == 0; query head h uses kv head h / (Hq/Hkv) */
    int32_t head_dim;      /* Dh: 64 or 128 */
    int32_t depth;         /* D >= 0: number of draft steps = maximum node depth */
    int32_t width;         /* W: nodes added per draft step (1..64) */
    int32_t n_nodes;       /* N (1..1024); must equal 1 + D*W for ygg_equal_growth_expand */
    int32_t vocab;         /* V (only used by expand / accept) */
    int32_t kv_dtype;      /* ygg_dtype of Q, K, V and O (see YGG_FP8_E4M3 for the mixed case) */
    float softmax_scale;   /* multiplies q.k; typically 1/sqrt(Dh); must be finite and > 0 where K/V are used */
    int64_t kv_capacity;   /* token slots per sequence in the cache, >= max_seq_len + D + 1 */
    int32_t max_seq_len;   /* host-known upper bound of seq_lens[b] (sizes the launch grids) */
} ygg_shape;

/* Bytes of workspace the given operation needs for this shape (0 if the shape is invalid). */
size_t ygg_workspace_bytes(const ygg_shape *shape, int32_t op /* ygg_op */, int32_t n_layers);

/* Static, human-readable name of a status code. */
const char *ygg_status_string(int32_t status);

/*
 * Optional: prepares the current device (raises the kernels' shared-memory limits).  Every launching
 * call does the same on first use; calling it up front keeps that out of a stream capture.  Thread safe.
 * Returns YGG_ERR_LAUNCH when there is no usable device.
 */
int32_t ygg_init(void);

/*
 * Tree-masked verify attention for one layer (paper Sec. 2 "Source of Improvements": the
 * speculative tokens are verified in one parallel pass under a sequence-level mask; Sec. 4.2,
 * last paragraph: the mask follows the tree's causal dependency).
 *
 * For every sequence b, node i and query head h (kv head g = h / (Hq/Hkv)):
 *     keys   J(i) = cache rows 0 .. seq_lens[b]-1  U  tree rows {i, parent[i], ..., 0}
 *     out[b,i,h,:] = sum_j softmax_j(softmax_scale * q[b,i,h,:] . k_j[g,:]) * v_j[g,:]
 *     lse[b,i,h]   = ln sum_j exp(softmax_scale * q . k_j)            (optional)
 * Scores, softmax and accumulation are fp32; bf16 inputs use bf16 matrix instructions with the
 * softmax weights rounded to bf16 before the value product.
 *
 *   q          [B,N,Hq,Dh]      kv_dtype
 *   k_cache    [B,cap,Hkv,Dh]   kv_dtype, rows [0,seq_lens[b]) valid, others never read
 *   v_cache    [B,cap,Hkv,Dh]
 *   seq_lens   [B] int32        0 <= seq_lens[b] <= max_seq_len
 *   k_tree     [B,N,Hkv,Dh]     K/V of the tree's own tokens; must not overlap the cache
 *   v_tree     [B,N,Hkv,Dh]
 *   parent_idx [B,N] int32
 *   out        [B,N,Hq,Dh]      kv_dtype (written)
 *   lse        [B,N,Hq] fp32    written, or NULL
 * Inputs are read-only; out/lse/workspace must not alias them.
 */
int32_t ygg_tree_attention(const ygg_shape *shape,
                           const void *q, const void *k_cache, const void *v_cache,
                           const int32_t *seq_lens, const void *k_tree, const void *v_tree,
                           const int32_t *parent_idx, void *out, float *lse,
                           void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The same attention with K and V stored in 8 bits (shape->kv_dtype == YGG_FP8_E4M3).  The paper
 * leaves the K/V precision open (Sec. 6: the TokenTree owns the K/V tensors); this variant halves
 * the bytes of the prefix, which is what bounds verification of small trees over long or batched
 * prefixes.  A stored element is an E4M3 code (1 sign, 4 exponent bits with bias 7, 3 mantissa
 * bits, subnormals, no infinities; codes 0x7f and 0xff are NaN and must not occur) and stands for
 *     K = k_scale[g] * value(code),   V = v_scale[g] * value(code)        (g = kv head)
 * The codes are widened to bf16 exactly, so the result is that of ygg_tree_attention on the
 * dequantised K/V with the scales applied in fp32.
 *
 *   q, out     [B,N,Hq,Dh] bf16;  lse [B,N,Hq] fp32 or NULL
 *   k_cache, v_cache [B,cap,Hkv,Dh] uint8;  k_tree, v_tree [B,N,Hkv,Dh] uint8
 *   k_scale, v_scale [Hkv] fp32 device, finite and > 0
 * Everything else as for ygg_tree_attention; workspace size is ygg_workspace_bytes(ATTENTION).
 */
int32_t ygg_tree_attention_fp8kv(const ygg_shape *shape,
                                 const void *q, const void *k_cache, const void *v_cache,
                                 const int32_t *seq_lens, const void *k_tree, const void *v_tree,
                                 const float *k_scale, const float *v_scale,
                                 const int32_t *parent_idx, void *out, float *lse,
                                 void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * One draft step d (1..D) of the Equal-Growth Tree (paper Sec. 4.2 "Draft Width Selection":
 * exactly W_draft leaves are grown per draft step, at the positions with the largest path-wise
 * gain, using generation probabilities as acceptance surrogates).  Candidates are the
 * (frontier node p, token v) pairs of the previous depth, F = 1 row (the root) for d = 1 and
 * F = W rows otherwise:
 *     score(p,v) = cum_logprob[frontier p] + log_softmax(draft_logits[b,p,:])[v]
 * The W best candidates (higher score first; equal scores: lower p*V+v first) become nodes
 * 1+(d-1)W .. dW in that order: parent_idx <- frontier node, token_ids <- v, cum_logprob <-
 * score rounded to fp32.  Scores are evaluated in fp64.
 *
 *   draft_logits [B,F,V] fp32    row p belongs to node 1+(d-2)W+p (node 0 for d = 1)
 *   parent_idx, token_ids [B,N] int32 and cum_logprob [B,N] fp32: in/out; depth d-1 entries are
 *   read, depth d entries written.  The caller initialises node 0 (parent -1, cum 0).
 * Requires N == 1 + D*W and F*V >= W.
 */
int32_t ygg_equal_growth_expand(const ygg_shape *shape, int32_t d, const float *draft_logits,
                                int32_t *parent_idx, int32_t *token_ids, float *cum_logprob,
                                void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * ygg_equal_growth_expand for callers that cannot allocate or carry a workspace: code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation.  Same operation, same kernels, same results; the
 * scratch is a fixed array inside the library's device image (YGG_STATIC_SCRATCH_BYTES per GPU, held until the
 * process ends), so the call allocates nothing and takes no workspace argument.  Shapes whose
 * ygg_workspace_bytes(shape, YGG_OP_EXPAND) exceeds YGG_STATIC_SCRATCH_BYTES are rejected with
 * YGG_ERR_WORKSPACE.  All calls on one GPU share that array: calls that may overlap on one GPU (different
 * streams, concurrent graphs) race and must use ygg_equal_growth_expand with workspaces of their own.
 */
#define YGG_STATIC_SCRATCH_BYTES (4u << 20)
int32_t ygg_equal_growth_expand_static(const ygg_shape *shape, int32_t d, const float *draft_logits,
                                       int32_t *parent_idx, int32_t *token_ids, float *cum_logprob,
                                       void *hip_stream);

/*
 * Equal growth with free attachment: draft step t (1..D) of the Equal-Growth Tree as the paper words
 * it (Sec. 4.2 "Draft Width Selection": every step grows exactly W_draft leaves, and they may hang
 * anywhere in the partial tree, at the positions with the largest path-wise gain).  Reading: every
 * node, once the drafter has run on it, offers its W most probable tokens (larger logit first, equal
 * logits: lower token first), each scored cum_logprob[node] + log_softmax(row)[token] in fp64; the
 * pool holds the offers not yet taken.  Step t adds the offers of the nodes grown at step t-1 (the
 * root for t = 1; F = 1 or W rows of draft_logits, in node order), orders the pool by (score
 * descending, node*V + token ascending) and turns the first W entries into nodes 1+(t-1)W .. tW in
 * that order: parent_idx <- offering node, token_ids, cum_logprob <- score rounded to fp32.  Node
 * depth no longer equals the step; it never exceeds t.
 *
 *   draft_logits [B,F,V] fp32; parent_idx, token_ids [B,N] int32 and cum_logprob [B,N] fp32 in/out
 *   pool         device memory owned by the caller and carried from step to step, at least
 *                ygg_attach_pool_bytes(shape) bytes, 16-byte aligned.  Step 1 initialises it.  Per
 *                sequence: int32 count, 12 bytes padding, then W*max(D-1,1) records {double score;
 *                int32 node; int32 token}, the first `count` valid and ordered best first.  After
 *                step t it holds the best W*(D-t) untaken offers: an entry of rank r cannot be
 *                taken before r/W more steps, so nothing else can ever become a node.
 * Requires N == 1 + D*W, V >= W, N*V < 2^32 and W*F + W*(D-t+1) <= 4096.
 */
size_t ygg_attach_pool_bytes(const ygg_shape *shape);
int32_t ygg_equal_growth_attach(const ygg_shape *shape, int32_t t, const float *draft_logits,
                                int32_t *parent_idx, int32_t *token_ids, float *cum_logprob,
                                void *pool, size_t pool_bytes,
                                void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Verification-width pruning (paper Sec. 4.2 "Verification Width Pruning": after drafting, the
 * maximum-value subtree with W_verify nodes is kept for verification; Eq. 3 with every term but
 * W_verify fixed decides the width).  The value of a node is the probability that its whole path is
 * accepted with the drafter's probabilities as surrogates, exp(cum_logprob[i]) (the root counts 1:
 * the bonus token); the sum over a kept set estimates the accepted length.
 *
 *   w_verify     HOST integer 1..N: the static width of the verifier pass that follows
 *   parent_idx, token_ids [B,N] int32, cum_logprob [B,N] fp32: the drafted tree, with
 *                cum_logprob[child] <= cum_logprob[parent] (true of sums of log-probabilities; the
 *                kept set is the w_verify largest values, which is the optimal connected subtree
 *                under exactly that condition)
 *   t_verifier   [N+1] fp32 device, t_verifier[n] > 0 = verifier latency with n tokens; NULL if
 *                best_width is NULL.  t_draft >= 0: total drafting latency, same unit (host scalar)
 *   kept_nodes   [B,w_verify] int32 out: kept original indices, ascending (still topological)
 *   new_parent   [B,w_verify] int32 out: parent in the renumbered tree (-1 for the root)
 *   new_token    [B,w_verify] int32 out
 *   expected_len [B] fp32 out or NULL: sum of the kept values
 *   best_width   [B] int32 out or NULL: the n in 1..N maximising (sum of the n largest values) /
 *                (t_draft + t_verifier[n]), first maximum -- a hint for the next step's width; it
 *                stays on the device
 * The renumbered tree feeds ygg_tree_attention / ygg_accept_and_compact with n_nodes = w_verify.
 * Needs no workspace.
 */
int32_t ygg_prune_for_verification(const ygg_shape *shape, int32_t w_verify,
                                   const int32_t *parent_idx, const int32_t *token_ids,
                                   const float *cum_logprob, const float *t_verifier, float t_draft,
                                   int32_t *kept_nodes, int32_t *new_parent, int32_t *new_token,
                                   float *expected_len, int32_t *best_width, void *hip_stream);

/*
 * Greedy acceptance and K/V compaction (paper Sec. 1: draft tokens that match the verifier's
 * own output are accepted; Sec. 5: the "accept speculation management" stage; Sec. 4.1 under
 * Eq. 2: the verifier's token after the last accepted one is the bonus token; Sec. 6: the
 * TokenTree owns the K/V tensors).  Everything stays on the device:
 *     t*[i]    = argmax_v target_logits[b,i,v]          (first maximum)
 *     match[0] = 1;  match[i] = match[parent[i]] and token_ids[i] == t*[parent[i]]
 *     best     = matched node of greatest depth (lowest index among equals)
 *     accept_path[b,:] = root .. best, padded with -1;  accept_len[b] = depth(best)+1
 *     bonus_token[b]   = t*[best]
 *     for every layer: cache[layer,b,seq_lens[b]+k] = tree[layer,b,accept_path[b,k]], K and V
 *     seq_lens[b] += accept_len[b]
 *
 *   target_logits [B,N,V] fp32, or NULL when target_tokens [B,N] int32 (the argmax) is given;
 *                 exactly one of the two must be non-NULL
 *   parent_idx, token_ids [B,N] int32
 *   k_tree, v_tree   [n_layers,B,N,Hkv,Dh]    kv_dtype (may be NULL when n_layers == 0)
 *   k_cache, v_cache [n_layers,B,cap,Hkv,Dh]  kv_dtype, updated in place
 *                    (with YGG_FP8_E4M3 the four K/V arrays hold one-byte codes; rows are copied as bytes)
 *   seq_lens [B] int32 in/out; accept_len [B], accept_path [B,D+1], bonus_token [B] int32 out
 */
int32_t ygg_accept_and_compact(const ygg_shape *shape, int32_t n_layers,
                               const float *target_logits, const int32_t *target_tokens,
                               const int32_t *parent_idx, const int32_t *token_ids,
                               const void *k_tree, const void *v_tree,
                               void *k_cache, void *v_cache, int32_t *seq_lens,
                               int32_t *accept_len, int32_t *accept_path, int32_t *bonus_token,
                               void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * A K/V cache in 8 bits with one scale per block of YGG_KV_BLOCK tokens and kv head, for one layer (or, given to
 * ygg_block8_append, for n_layers layers, one behind the other in each array).  nblk = ceil(kv_capacity / 64) blocks a sequence.
 *
 *   k_codes, v_codes [B,Hkv,nblk,64*Dh] E4M3 codes (as for ygg_tree_attention_fp8kv): a stored element is scale * value(code)
 *   k_scale, v_scale [B,Hkv,nblk] fp32, at least 2^-100 and finite
 *   k_tail,  v_tail  [B,128,Hkv,Dh] bf16: the row of token p is p % 128
 *
 * With L = seq_lens[b], tokens 0 .. 64*(L/64) - 1 are read from the blocks and the last L % 64 from the tail; nothing else of a
 * cache is read.  A block is written when its last token arrives, from the bf16 rows of all its tokens.  The tail keeps rows while
 * their block is open: those with which an append completes a block go into codes only.  So seq_lens[b] may be taken back to any
 * token of the open block, to any multiple of 64, and in the block before the open one up to the length from which the append that
 * completed it began, where that lies in the block and no rows of a later block have come into its half of the tail since.  No
 * other length finds its rows.
 * Inside a block the codes lie in the order in which the matrix instructions of gfx950 take them, so that a block is streamed as
 * it is stored: with token t (0..63) and dimension d, the code is at byte 1024*chunk + 16*lane + e,
 *   K: chunk = 2*((t/32)*(Dh/64) + d/64) + d/16%2,  lane = 32*(d/32%2) + t%32,  e = d%16
 *   V: chunk = 2*(d/32) + t/32,                     lane = 32*(t/4%2) + d%32,   e = 4*(t%32/8) + t%4
 */
#define YGG_KV_BLOCK 64
typedef struct {
    void *k_codes, *v_codes;   /* 16-byte aligned, as the tails */
    float *k_scale, *v_scale;
    void *k_tail, *v_tail;
} ygg_block8_cache;

/*
 * Tree attention (see ygg_tree_attention) of one layer over such a cache; shape->kv_dtype == YGG_FP8_BLOCK, head_dim 64 or 128.
 * A tree of one node (n_nodes 1, depth 0) is plain decoding.  q and the keys and values of cache and tree must be finite, below 2^60 in
 * magnitude, with scores softmax_scale * q.k below 2^23 in magnitude (fp32, to 2^-24 of a score).
 *   q, out [B,N,Hq,Dh] bf16;  k_tree, v_tree [B,N,Hkv,Dh] bf16;  lse [B,N,Hq] fp32 or NULL;  seq_lens, parent_idx int32
 * q (bf16, 8 bits of significand) and the softmax weights enter the products as sums of two E4M3 values, that is with 8 bits and
 * an exponent per row and tile; softmax and accumulation are fp32 (the matrix instructions of 8-bit values cut each product at
 * 2^-13 of the largest of its group before they add).  A weight below 2^-126 of its row's largest may count as that much.
 * Workspace: ygg_workspace_bytes(ATTENTION_BLOCK8).
 */
int32_t ygg_tree_attention_block8(const ygg_shape *shape, const void *q, const ygg_block8_cache *cache /* host struct */,
                                  const int32_t *seq_lens, const void *k_tree, const void *v_tree,
                                  const int32_t *parent_idx, void *out, float *lse,
                                  void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Appends new tokens to such a cache, all layers in one launch: the K/V bookkeeping that ygg_accept_and_compact does for plain
 * caches (call it with n_layers = 0 and hand its accept_path, accept_len and seq_lens to this), or a prompt's K/V.
 *   k_new, v_new [n_layers,B,n_rows,Hkv,Dh] bf16: the tree's, or the prompt's, rows, finite
 *   rows         [B,max_new] int32: token k of the new ones is row rows[b][k]; NULL: row k.  Out-of-range rows count as zeros
 *   n_new        [B] int32: new tokens of sequence b, 0 .. max_new (clamped to that)
 *   seq_lens     [B] int32: the lengths AFTER the append (only read; clamped to kv_capacity); tokens seq_lens[b] - n_new[b] ..
 *                seq_lens[b] - 1 are written
 * Rows of the open block go to the tail as they are; a block that is completed is encoded: scale = max|x| / 448 over its 64
 * tokens of one head (1 if all are zero, never below 2^-100), code = the E4M3 value nearest to x * (1 / scale) in fp32, ties to even.
 * Requires max_new <= n_rows unless rows is given.  Needs no workspace.
 */
int32_t ygg_block8_append(const ygg_shape *shape, int32_t n_layers, const void *k_new, const void *v_new, int32_t n_rows,
                          const int32_t *rows, int32_t max_new, const int32_t *n_new, const int32_t *seq_lens,
                          const ygg_block8_cache *cache /* host struct */, void *hip_stream);

/*
 * Rotary positions.  For pair j of the first rotary_dim dimensions of every head of token i of sequence b, at position p,
 *     (x_j, x_j') <- scale * (x_j cos a - x_j' sin a,  x_j' cos a + x_j sin a),   a = p * frequencies[j]
 * with (j, j') = (j, j + rotary_dim/2), or (2j, 2j+1) if interleaved; further dimensions are copied.  Angles are formed in fp64.
 *   p            seq_lens[b] + depth of node i (parent_idx), or positions[b][i] if positions is given (then n_nodes is any number of
 *                tokens per sequence, not a tree's, and seq_lens and parent_idx are not read)
 *   q, q_out [B,N,Hq,Dh], k, k_out [B,N,Hkv,Dh]: fp32 for kv_dtype YGG_F32, else bf16.  One of the pairs may be NULL.  Tokens of
 *                q and k are q_stride and k_stride elements apart (0: dense), so that parts of a fused projection can be given;
 *                outputs are dense and may be the inputs where these are dense, else must not overlap them
 *   frequencies  [rotary_dim/2] fp64 device, radians per position: scaled ones for long contexts are the caller's table
 *   rotary_dim   a multiple of 16 up to head_dim;  scale: finite (1, or the factor that goes with a frequency scaling)
 */
int32_t ygg_tree_rotary(const ygg_shape *shape, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                        void *q_out, void *k_out, const double *frequencies, int32_t rotary_dim, int32_t interleaved,
                        float scale, const int32_t *seq_lens, const int32_t *parent_idx, const int32_t *positions,
                        void *hip_stream);

/*
 * The same rotation behind a norm of every head, in one pass over q and k: with x a head's values of one token and w its weights,
 *     y_d = x_d * w_d / sqrt(sum_d x_d^2 / head_dim + eps)   in fp32, not rounded; then the pairs of y as above, rounded once
 *   q_weight, k_weight [Dh] fp32 device, or [Hq,Dh] and [Hkv,Dh] if weights_per_head, 16-byte aligned; needed with their tensor
 *   eps          finite, >= 0.  The sum of a head's squares must stay below fp32's largest value; a head whose mean square and eps
 *                together are below 2^-126 (zeros, with eps = 0) comes out as zeros, one with a NaN as NaN throughout
 * Everything else as for ygg_tree_rotary.
 */
int32_t ygg_tree_norm_rotary(const ygg_shape *shape, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                             void *q_out, void *k_out, const float *q_weight, const float *k_weight, int32_t weights_per_head,
                             float eps, const double *frequencies, int32_t rotary_dim, int32_t interleaved, float scale,
                             const int32_t *seq_lens, const int32_t *parent_idx, const int32_t *positions, void *hip_stream);

/*
 * Causal attention of whole prompts, or of the next chunk of them behind keys that are cached already, for one layer.  Sequence b has
 * its queries in rows q_first[b] .. + q_len[b] - 1 of q and out, and its keys in rows k_first[b] .. + k_len[b] - 1 of k and v: packed
 * sequences, padded ones and slabs of a cache [B,cap,Hkv,Dh] (k_first[b] = b * cap) alike.  The last query sees every key:
 *     keys J(i) = { j : j <= i + k_len[b] - q_len[b] }   for query i of sequence b, i = 0 .. q_len[b] - 1
 *     out[q_first[b]+i,h,:] = sum_j softmax_j(softmax_scale * q_i . k_j[g,:]) * v_j[g,:],  lse = ln sum_j exp(softmax_scale * q_i . k_j)
 * A query that sees no key (q_len > k_len) gets zeros, and -inf as lse.  Scores, softmax and accumulation are fp32; with bf16 the softmax
 * weights are rounded to bf16 for the value product.
 *
 *   shape        kv_dtype YGG_F32 or YGG_BF16; batch = sequences; n_nodes = rows of q and out, those of all sequences together, up to 2^25;
 *                kv_capacity = rows of k and v, below 2^31; max_seq_len = a bound of k_len, at most kv_capacity and 2^30; depth, width and
 *                vocab are not read.  n_nodes * n_q_heads + 128 * batch * n_kv_heads up to 2^29 is accepted, more may be refused
 *   q, out [n_nodes,Hq,Dh];  k, v [kv_capacity,Hkv,Dh];  lse [n_nodes,Hq] fp32 or NULL.  Rows of q, k and v are q_stride, k_stride and
 *                v_stride elements apart (0: dense; k's and v's at most 2^24), so that parts of a fused projection can be given; out is dense
 *                and overlaps nothing
 *   q_first, q_len, k_first, k_len [B] int32 device.  No two sequences share rows of q; they may share keys.  Of a sequence that
 *                ends behind the rows those that exist are taken, of keys max_seq_len at most; one that begins outside of them (a negative
 *                first too) or whose length is negative has none.  What sees what goes by the lengths that this leaves: the last query left
 *                sees every key left.  Rows of out and lse of no sequence are not written.
 *                A sequence's q, k and v are finite, below 2^60 in magnitude, with scores softmax_scale * q . k below 2^126 (fp32, to 2^-24 of a
 *                score; sums of weights and values are not normalised before their end); what lies outside of the sequences may be anything
 * Workspace: ygg_workspace_bytes(PROMPT_ATTENTION), which may be 0; what serves max_seq_len serves every smaller one.
 */
int32_t ygg_prompt_attention(const ygg_shape *shape, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                             const void *v, int64_t v_stride, const int32_t *q_first, const int32_t *q_len,
                             const int32_t *k_first, const int32_t *k_len, void *out, float *lse,
                             void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * A K/V cache in 4 bits.  Blocks, tails, lengths and what a length can be taken back to are those of ygg_block8_cache; a block holds
 * E2M1 codes (1 sign, 2 exponent bits, 1 of significand: 0, 0.5, 1, 1.5, 2, 3, 4, 6) two to a byte, the even one in the low half, with
 * a power of two to 32 values: of K to the 32 dimensions 32i .. 32i+31 of a token, of V to the 32 tokens 32i .. 32i+31 of the block of a
 * dimension, which are the groups that gfx950's matrix instructions scale by themselves.  A stored element is 2^(scale - 127) * value(code).
 *
 *   k_codes, v_codes [B,Hkv,nblk,32*Dh] bytes;  k_scale, v_scale [B,Hkv,nblk,2*Dh] bytes, 27 .. 253 (2^-100 .. 2^126)
 *   k_tail, v_tail   [B,128,Hkv,Dh] bf16;  all 16-byte aligned
 * Inside a block, with token t and dimension d, the code is number 2048*chunk + 32*lane + e and the scale byte lane*(Dh/32) + chunk:
 *   K: chunk = t/32*(Dh/64) + d/64,  lane = 32*(d/32%2) + t%32,  e = d%32
 *   V: chunk = d/32,                 lane = 32*(t/32) + d%32,    e = 16*(t/4%2) + 4*(t%32/8) + t%4
 */
typedef struct {
    void *k_codes, *v_codes;
    void *k_scale, *v_scale;
    void *k_tail, *v_tail;
} ygg_block4_cache;

/*
 * Tree attention (see ygg_tree_attention) of one layer over such a cache; shape->kv_dtype == YGG_FP4_BLOCK.  Everything else as for
 * ygg_tree_attention_block8, the ranges of values and the two E4M3 values for each of q and the weights included.
 * Workspace: ygg_workspace_bytes(ATTENTION_BLOCK4).
 */
int32_t ygg_tree_attention_block4(const ygg_shape *shape, const void *q, const ygg_block4_cache *cache /* host struct */,
                                  const int32_t *seq_lens, const void *k_tree, const void *v_tree,
                                  const int32_t *parent_idx, void *out, float *lse,
                                  void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Appends new tokens to such a cache, all layers in one launch.  Arguments are those of ygg_block8_append.  A block that is completed
 * is encoded: the scale of 32 values is the least 2^e, e >= -100, with max|x| <= 7 * 2^e, and a code the nearest to x / 2^e, ties to the
 * even code, what lies beyond 6 as 6 (values between 6 and 7 are off by no more than those between 4 and 6 may be).
 */
int32_t ygg_block4_append(const ygg_shape *shape, int32_t n_layers, const void *k_new, const void *v_new, int32_t n_rows,
                          const int32_t *rows, int32_t max_new, const int32_t *n_new, const int32_t *seq_lens,
                          const ygg_block4_cache *cache /* host struct */, void *hip_stream);

/*
 * Adds tokens to the counts that ygg_constrain_logits goes by.
 *   tokens [B,n_tokens] int32;  rows [B,max_new] int32 or NULL: the k-th token added is tokens[b][rows[b][k]], or tokens[b][first+k]
 *   n_new  [B] int32: tokens to add, 0 .. max_new (clamped to that);  prompt != 0: marks them as the prompt's instead of counting
 *   counts [B,V] int32, in/out: bits 0-30 how often a token occurs in the confirmed reply, sign bit: it occurs in the prompt
 * After ygg_accept_and_compact: tokens = the tree's token_ids, rows = accept_path, n_new = accept_len.  Tokens outside [0,V) and
 * rows outside [0,n_tokens) are left out.  The caller zeroes counts when a sequence begins.
 */
int32_t ygg_count_tokens(const ygg_shape *shape, const int32_t *tokens, int32_t n_tokens, const int32_t *rows, int32_t first,
                         int32_t max_new, const int32_t *n_new, int32_t prompt, int32_t *counts, void *hip_stream);

/*
 * Constrains the logits of every tree node and / or finds each row's first maximum.  With c = the token's count in `counts` plus its
 * occurrences on the node's path (root .. node, token_ids), x = logit of node i of sequence b and token v, in fp32 and in this order:
 *     if v occurs in counts[b] (reply or prompt) or on the path:  x <- x > 0 ? x / repetition[b] : x * repetition[b]
 *     x <- x - frequency[b] * c;   if c > 0:  x <- x - presence[b];   x <- x + bias[b][v]
 *     if mask_index[b][i] = m >= 0 and bit v%32 of masks[m][v/32] is 0:  x <- -inf
 *     out[b,i,v] = x;   best[b,i] = argmax_v x (first maximum; a NaN that no mask covers counts as the largest value)
 * `out` feeds ygg_equal_growth_expand / _attach and ygg_accept_and_compact, `best` the latter's target_tokens.
 */
typedef struct {
    const int32_t *counts;      /* [B,V] device (ygg_count_tokens), or NULL: only the path counts */
    const float *repetition;    /* [B] device, > 0, or NULL: 1 */
    const float *presence;      /* [B] device or NULL: 0 */
    const float *frequency;     /* [B] device or NULL: 0 */
    const float *bias;          /* [B,V] device or NULL; -inf forbids a token */
    int32_t bias_shared;        /* != 0: bias is [V], the same for all sequences */
    int32_t n_masks;
    const uint32_t *masks;      /* [n_masks, ceil(V/32)] device or NULL */
    const int32_t *mask_index;  /* [B,N] device, required with masks; an index beyond n_masks - 1 counts as the last */
} ygg_logit_rules;

/*
 *   logits     [B,N,V]: fp32 or bf16 (logits_dtype YGG_F32 / YGG_BF16), rows row_stride elements apart (0: V)
 *   out        [B,N,V] fp32, or NULL; may be `logits` where those are dense and fp32
 *   best       [B,N] int32, or NULL (then no workspace is needed); one of out and best must be given
 * Workspace: ygg_workspace_bytes(CONSTRAIN).
 */
int32_t ygg_constrain_logits(const ygg_shape *shape, const void *logits, int32_t logits_dtype, int64_t row_stride,
                             const int32_t *parent_idx, const int32_t *token_ids, const ygg_logit_rules *rules /* host struct */,
                             float *out, int32_t *best, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Debug validator for the data-dependent part of the contract above (the paper's runtime keeps the
 * tree-structure array, the KV lengths and the token ids in a TokenTree object, Sec. 6; the calls
 * here trust them).  Writes one bit mask per sequence to flags[b] (device memory, [B] int32); every
 * input may be NULL, its checks are then skipped.  Not on the verification path: call it while
 * bringing a caller up, read the flags after synchronising.
 *   parent_idx [B,N]: YGG_BAD_PARENT if parent_idx[b][0] != -1 or some parent_idx[b][i] not in
 *                     [0, i); otherwise YGG_BAD_DEPTH if some node is deeper than `depth`
 *   seq_lens   [B]:   YGG_BAD_SEQ_LEN if outside [0, max_seq_len]
 *   token_ids  [B,N]: YGG_BAD_TOKEN if outside [0, vocab)
 *   logits     [B,logit_rows,V] fp32: YGG_BAD_LOGIT if any entry is NaN
 */
typedef enum {
    YGG_BAD_PARENT = 1, YGG_BAD_SEQ_LEN = 2, YGG_BAD_DEPTH = 4, YGG_BAD_TOKEN = 8, YGG_BAD_LOGIT = 16
} ygg_violation;
int32_t ygg_debug_validate(const ygg_shape *shape, const int32_t *parent_idx, const int32_t *seq_lens,
                           const int32_t *token_ids, const float *logits, int32_t logit_rows,
                           int32_t *flags, void *hip_stream);

/*
 * The launch plan ygg_tree_attention uses for a shape, for tests and tuning (host only, no GPU needed):
 * plan[0] = 1 matrix-core kernel / 0 vector kernel, plan[1] = wavefronts per workgroup, plan[2] = 2 if
 * wavefront pairs split every key tile else 1, plan[3] = workgroups along the query rows of one kv head,
 * plan[4] = key splits (the last three are 0 / meaningless for the vector kernel except plan[4]).
 */
int32_t ygg_debug_attention_plan(const ygg_shape *shape, int32_t *plan /* [5], host */);

/*
 * More of the same plan, for tests: launch[0] = 1 if the two wavefronts of a SIMD run in opposite phases, launch[1] = key tiles
 * by which the last key split's share is smaller than an equal one where that shortens the longest, launch[2] = bytes of shared
 * memory of a workgroup (all 0 for the vector kernel).
 */
int32_t ygg_debug_attention_launch(const ygg_shape *shape, int32_t *launch /* [3], host */);

/*
 * The launch plan of ygg_tree_attention_block8 for a shape (host only): plan[0] = 32-row blocks to a workgroup, plan[1] = such
 * workgroups along the query rows of one kv head, plan[2] = row blocks of the workgroups of the rows beyond them (0: none),
 * plan[3] and plan[4] = equal runs that either kind cuts the batch's keys into (0: a workgroup to each sequence), plan[5] = 1 if a
 * workgroup has twice the wavefronts, plan[6] = lanes to a row in the merge of partial results (0: no merge).
 */
int32_t ygg_debug_block8_plan(const ygg_shape *shape, int32_t *plan /* [7], host */);
/* .. and that of ygg_tree_attention_block4, likewise. */
int32_t ygg_debug_block4_plan(const ygg_shape *shape, int32_t *plan /* [7], host */);

/*
 * The launch plan of ygg_prompt_attention for a shape (host only): plan[0] = rows (queries x heads of a group) to a workgroup, plan[1] =
 * parts into which a workgroup's keys are split, plan[2] = row tiles that the batch can have per kv head.
 */
int32_t ygg_debug_prompt_plan(const ygg_shape *shape, int32_t *plan /* [3], host */);

/*
 * Tuning hook: forces the workgroup shape (wavefronts, 32-row blocks per wavefront, key shares) and/or the number
 * of key splits of every later ygg_tree_attention call of this process; a field left 0 keeps the library's own
 * choice, an unknown shape is ignored, and (0, 0, 0, 0) removes the override.  The workspace must be sized
 * (ygg_workspace_bytes) while the same override is in force.  Process-wide; meant for sweeps, not for production.
 */
int32_t ygg_debug_set_attention_plan(int32_t waves, int32_t rblocks, int32_t nsplit, int32_t kshares);

/*
 * Measurement hook for benchmarks (not part of the verification path): ygg_tree_attention without the launch that
 * merges the key splits, i.e. the main kernel alone, enqueued like any other call.  `out` and `lse` are only
 * complete for shapes with a single key split.  Timing a captured sequence of such calls gives the main kernel's
 * duration without event pairs, host gaps or library state.  Same arguments and errors as ygg_tree_attention.
 */
int32_t ygg_debug_tree_attention_main(const ygg_shape *shape,
                                      const void *q, const void *k_cache, const void *v_cache,
                                      const int32_t *seq_lens, const void *k_tree, const void *v_tree,
                                      const int32_t *parent_idx, void *out, float *lse,
                                      void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* YGG_H */
