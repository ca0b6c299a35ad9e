/*
 * hawk.h - C ABI of the B200 (sm_100a) verify step of speculative decoding for autoregressive
 * image generation (Hawk).
 *
 * The verify step takes a block of K drafted image tokens per sequence and decides how many of
 * them the target model accepts.  It has three parts, one entry point each:
 *   hawk_verify_attn  block-causal attention of the K draft queries over the cached context, for
 *                     the conditional and the unconditional guidance stream;
 *   hawk_head_proj    projection of the K hidden states onto the image-token codebook;
 *   hawk_cfg_accept   guidance combine, temperature, top-k, softmax and speculative rejection
 *                     sampling, returning the accepted length and the correction token;
 *   hawk_tree_accept  the same for a candidate tree with several candidates per depth.
 *   hawk_spec_cache_*, hawk_pool_*  the cache of vertical predictions and the sampling pool that feed it;
 *   hawk_head_proj_cfg, hawk_*_accept_guided  the head with the guidance combine in its epilogue;
 *   hawk_qk_norm_rope, hawk_rope_append, hawk_paged_attn  what surrounds the attention when the cache is paged:
 *                     norm and rotation of the heads, writing the new rows, attention of a chunk of them;
 *   hawk_sample       a token from a row of logits (guidance, temperature, top-k, top-p, min-p), for steps without drafts
 *                     and for the draft side, whose distributions the verification reads;
 *   hawk_pages_*      the paged cache between two steps: streams grow, are cut, forked and freed, pages are copied and
 *                     packed, the rows of an accepted path move to the front.
 *
 * Conventions common to all entry points
 *   - Every pointer is a DEVICE pointer owned by the caller unless the comment says "host".  The
 *     library allocates no device memory, frees nothing, never synchronises and keeps no pointer
 *     after the call returns.  All work is queued on `stream`.  (Two calls keep state of their own and
 *     say so in their comments: hawk_verify_step_host owns one stream and two events per device,
 *     hawk_cfg_accept_noalloc a fixed array in the library's device image.)
 *   - Tensors are dense, row-major in the index order written in brackets, base address aligned
 *     to 16 bytes.  bf16 is the 16 high bits of an IEEE fp32.
 *   - The return value is the only error channel.  On any error nothing is launched and the
 *     outputs are untouched.  Conditions that only the device can see (a draft id out of range,
 *     a NaN logit, a wait that ran out) are OR-ed into *dev_status (HAWK_DEV_* bits) when that
 *     pointer is not NULL; the caller clears the word.  No kernel traps or asserts.
 *   - B sequences, S = 2B guidance streams: stream b is the conditional one of sequence b,
 *     stream B+b its unconditional one.  K drafts per sequence.
 */
#ifndef HAWK_H
#define HAWK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st *hawk_stream_t; /* a cudaStream_t / CUstream; 0 = the default stream */

typedef enum {
    HAWK_OK = 0,
    HAWK_ERR_NULL = 1,        /* a required pointer is NULL                                     */
    HAWK_ERR_SHAPE = 2,       /* a size is negative or sizes contradict each other              */
    HAWK_ERR_ALIGN = 3,       /* a tensor base is not 16-byte aligned                           */
    HAWK_ERR_UNSUPPORTED = 4, /* a value outside what the kernels are built for (see each call) */
    HAWK_ERR_WORKSPACE = 5,   /* workspace missing or smaller than *_workspace_bytes says       */
    HAWK_ERR_PARAM = 6,       /* a scalar parameter is not a usable number                      */
    HAWK_ERR_CUDA = 7         /* the CUDA runtime or driver refused a call (launch, tensor map) */
} hawk_status;

/* bits of *dev_status */
#define HAWK_DEV_TIMEOUT 1    /* a bounded wait inside a kernel ran out; outputs are not valid  */
#define HAWK_DEV_BAD_DRAFT 2  /* a draft id lay outside [v_begin, v_end) and was clamped into it */
#define HAWK_DEV_NONFINITE 4  /* a NaN or +inf logit was treated as -inf                        */
#define HAWK_DEV_BAD_PREFIX 8 /* a prefix length lay outside [0, L_cap - K] and was clamped     */
#define HAWK_DEV_BAD_TREE 16  /* a child range or draft-row index of the tree was out of range    */
#define HAWK_DEV_BAD_ROWS 64  /* row_begin does not cut the new rows into streams as the call says; the stream was skipped */
#define HAWK_DEV_BAD_PAGE 128 /* a page id lay outside [0, n_pages)                             */
#define HAWK_DEV_BAD_POSITION 256 /* a rotation position lay outside [0, n_positions) and was clamped */
#define HAWK_DEV_NO_PAGES 512 /* more pages were needed than are free; streams that found none stay as they were */
#define HAWK_DEV_BAD_SETTING 1024 /* a row's temperature, top_p or min_p was no usable number and taken as off */
#define HAWK_DEV_BOUNDS 32    /* libraries built with -DHAWK_DEBUG only: an index lay outside its array, the access was skipped */

const char *hawk_status_string(hawk_status status);
int hawk_version(void); /* major*10000 + minor*100 + patch */

/* ------------------------------------------------------------------------------------------------
 * hawk_verify_attn - attention of the K draft queries against the cached prefix.
 *
 * Operation (Sec. 3, "Speculative Sampling": one forward pass of the target model verifies the
 * drafted tokens in parallel; the KV cache is the one App. C mentions).  For stream s, query head
 * h and draft position i, with n = prefix_len[s] + i + 1 visible keys and kv head g = h / (H/H_kv):
 *     e_j = sm_scale * <q[s,i,h,:], k_cache[s,g,j,:]>,  j < n
 *     out[s,i,h*D:(h+1)*D] = sum_j softmax(e)_j * v_cache[s,g,j,:]
 * The block's own K rows must already be stored in the caches at rows prefix_len[s] .. +K-1; rows
 * past that are never used (they may hold anything).  Scores and sums are fp32.
 *
 *   q            bf16 [S][K][H][D]
 *   k_cache      bf16 [S][H_kv][L_cap][D]
 *   v_cache      bf16 [S][H_kv][L_cap][D]
 *   prefix_len   int32 [S], each in [0, L_cap - K]
 *   out          bf16 [S][K][H*D]
 *   max_prefix_len  upper bound of prefix_len[] known on the host (sizes the launch only)
 *   sm_scale     score scale, > 0, normally 1/sqrt(D)
 *   workspace    scratch of at least hawk_verify_attn_workspace_bytes(...) bytes, 16-byte aligned;
 *                may be NULL when that function returns 0.  Contents need no initialisation and
 *                are garbage afterwards.
 * Supported: D in {64, 128}; 1 <= K <= 64; H a multiple of H_kv; S*H_kv*L_cap < 2^31.
 * Errors: NULL, SHAPE (negative sizes, max_prefix_len + K > L_cap), ALIGN, UNSUPPORTED, WORKSPACE,
 * PARAM (sm_scale not a positive finite number), CUDA.  S == 0 returns HAWK_OK without a launch.
 * ---------------------------------------------------------------------------------------------- */
size_t hawk_verify_attn_workspace_bytes(int S, int K, int H, int H_kv, int D, int max_prefix_len);

hawk_status hawk_verify_attn(const void *q, const void *k_cache, const void *v_cache,
                             const int32_t *prefix_len, void *out, int S, int K, int H, int H_kv,
                             int D, int L_cap, int max_prefix_len, float sm_scale, void *workspace,
                             size_t workspace_bytes, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_verify_attn_tree - the same attention for a candidate tree.
 *
 * Operation (Sec. 4.2: all candidates of the tree are verified in one forward pass of the target
 * model): the N tree nodes of a stream are N queries; node i attends to the whole
 * cached prefix and, inside the block, only to the nodes on its own path from the root:
 *     key j <  prefix_len[s]                  visible to every node
 *     key j == prefix_len[s] + m, 0 <= m < N  visible to node i iff bit m of anc_mask[i] is set
 * Node i's own key/value row is cache row prefix_len[s] + i, so anc_mask[i] has bit i set.
 * hawk_verify_attn is the special case anc_mask[i] = 2^(i+1) - 1.
 *
 *   q         bf16 [S][N][H][D]
 *   anc_mask  uint64 [N], device memory, shared by all streams
 *   out       bf16 [S][N][H*D]
 * Everything else, the workspace (hawk_verify_attn_workspace_bytes with K = N) and the errors are
 * those of hawk_verify_attn; 1 <= N <= 64.
 * ---------------------------------------------------------------------------------------------- */
hawk_status hawk_verify_attn_tree(const void *q, const void *k_cache, const void *v_cache,
                                  const int32_t *prefix_len, const uint64_t *anc_mask, void *out, int S,
                                  int N, int H, int H_kv, int D, int L_cap, int max_prefix_len,
                                  float sm_scale, void *workspace, size_t workspace_bytes,
                                  int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_head_proj - output head: hidden states onto the token codebook.
 *
 * Operation (Sec. 3: the decoding head after the final hidden layer maps a hidden state to
 * logits over the codebook of image tokens):
 *     logits[m][v] = sum_c x[m][c] * w[v][c]      for v_begin <= v < v_end
 * bf16 operands, fp32 accumulation on the tensor cores, fp32 result.  Columns outside
 * [v_begin, v_end) are not written.
 *
 *   x       bf16 [M][hidden]   one row per (stream, draft position): M = 2*B*K
 *   w       bf16 [V][hidden]   one row per token id
 *   logits  fp32 [M][V]
 * Supported: hidden a multiple of 64 (and >= 64).
 * Errors: NULL, SHAPE (negative sizes, range outside [0, V]), ALIGN, UNSUPPORTED, CUDA.
 * M == 0 or an empty range returns HAWK_OK without a launch.
 * ---------------------------------------------------------------------------------------------- */
hawk_status hawk_head_proj(const void *x, const void *w, float *logits, int M, int hidden, int V,
                           int v_begin, int v_end, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_cfg_accept - target distribution and speculative rejection sampling of a draft chain.
 *
 * Operation, per sequence b and draft position i = 0, 1, ... (Sec. 3: accept draft x with
 * probability min(1, p(x)/q(x)), otherwise resample from norm(max(0, p - q)); Sec. 4.2, Eq.
 * "recur": a pass moves one position deeper, the first rejection ends the chain; generation
 * settings of Sec. 5: guidance scale, temperature, top-k):
 *   1. l[v] = lu[v] + cfg_scale*(lc[v] - lu[v]) over the valid ids, lc/lu the conditional and
 *      unconditional logit rows; -inf in either gives -inf.  Evaluated in fp32 as subtract, fused
 *      multiply-add, then divide by temperature.
 *   2. With 0 < top_k < number of finite l: keep every l >= the top_k-th largest (ties at the
 *      threshold are all kept); the rest become -inf.
 *   3. p = softmax(l); ids outside [v_begin, v_end) have p = 0.
 *   4. x = draft[b][i]; accept iff u_accept[b][i] * q[b][i][x] < p[x]; on a pass go to i+1.
 *   5. On the first rejection: r = max(0, p - q[b][i][:]); if r has no mass, r = p;
 *      out_token[b] = the smallest id whose running sum of r (ascending id) exceeds
 *      u_resample[b][i] * sum(r); accept_len[b] = i.
 *   6. All K accepted: accept_len[b] = K; out_token[b] = -1, or with has_bonus_row the same draw
 *      from p of row K with u_resample[b][K].
 * The paper's "accept length" counts the correction token: it equals accept_len + 1.
 *
 *   logits      fp32 [2B][K + has_bonus_row][V]
 *   q_probs     fp32 [B][K][V]   draft probabilities, used as given
 *   draft       int32 [B][K]
 *   u_accept    fp32 [B][K]      uniforms in [0,1)
 *   u_resample  fp32 [B][K+1]    uniforms in [0,1)
 *   accept_len  int32 [B]  (out)
 *   out_token   int32 [B]  (out)
 *   p_debug     optional fp32 [B][K + has_bonus_row][V]: receives p over the valid ids; NULL in
 *               normal use (p never leaves the chip)
 *   workspace   at least hawk_cfg_accept_workspace_bytes(...) bytes, 16-byte aligned; needs no
 *               initialisation
 * Every row is judged by a thread block of its own.  A call with more rows than the GPU runs at once
 * lets the blocks of later positions look at the verdicts their sequence already has, and a row
 * behind a rejection (step 5 never reads it) does no work; the results do not depend on it, and with
 * p_debug every row is computed.
 * Supported: 1 <= K <= 16; 1 <= v_end - v_begin <= 32768 (one row is held in one
 * thread block's registers); temperature > 0.
 * Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE, PARAM (cfg_scale or temperature not finite,
 * temperature <= 0), CUDA.  B == 0 returns HAWK_OK without a launch.
 * ---------------------------------------------------------------------------------------------- */
size_t hawk_cfg_accept_workspace_bytes(int B, int K, int V);

hawk_status hawk_cfg_accept(const float *logits, const float *q_probs, const int32_t *draft,
                            const float *u_accept, const float *u_resample, int B, int K, int V,
                            int v_begin, int v_end, float cfg_scale, float temperature, int top_k,
                            int has_bonus_row, int32_t *accept_len, int32_t *out_token,
                            float *p_debug, void *workspace, size_t workspace_bytes,
                            int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_tree_accept - verification of a candidate tree: several candidates per depth, each with its
 * own draft distribution.
 *
 * Operation (Sec. 4.2, "Sampling and Verification", Eq. "recur"; distribution preservation: App. A).
 * The tree is shared by the batch: node 0 is the root (the last committed token), the children of
 * node n are the nodes child_begin[n] .. child_begin[n+1]-1 (all ids > n), verified in that order.
 * Per sequence b, starting at the root with depth 0:
 *   1. p = target distribution of the node's logit rows (steps 1-3 of hawk_cfg_accept).
 *   2. For each child c in order, with x = node_token[b][c], q = q_probs[b][node_q[c]]:
 *      accept iff u_accept[b][c] * q[x] < p[x]; on a pass move to node c, one level deeper, step 1.
 *      On a rejection p <- norm(max(0, p - q)); a residual without mass leaves p as it is.
 *   3. Every child rejected, or the node has none: out_token[b] = inverse-CDF draw (ascending id)
 *      from p as refined so far with u_resample[b][node]; accept_len[b] = depth; stop.
 * q may come from a different draft head for every candidate (horizontal or vertical), which is what
 * shrinks the probability that all candidates of a level are rejected.
 * A chain of K drafts is the tree with N = K + 1 nodes and child_begin[n] = n + 1.
 *
 *   logits      fp32 [2B][N][V]  row n: logits for the token that follows node n (b conditional, B+b not)
 *   q_probs     fp32 [B][NQ][V]  draft probabilities, used as given
 *   node_token  int32 [B][N]     candidate token of node n (entry 0 unused)
 *   node_q      int32 [N]        row of q_probs the token of node n was drawn from (entry 0 unused)
 *   child_begin int32 [N+1]      device memory, like everything else
 *   u_accept    fp32 [B][N]      uniforms in [0,1), one per candidate node (entry 0 unused)
 *   u_resample  fp32 [B][N]      uniforms in [0,1), entry n used if the walk stops at node n
 *   accept_len  int32 [B] (out)  number of accepted candidates
 *   out_token   int32 [B] (out)  correction token; -1 if the refined target has no mass at all
 *   path        optional int32 [B][max_depth] (out): accepted nodes in order, -1 beyond accept_len
 *   workspace   at least hawk_tree_accept_workspace_bytes(B, N) bytes, 16-byte aligned, no initialisation
 * Every node is judged by its own thread block, so the cost is at most B*N rows; in a call with more
 * rows than the GPU runs at once, a node whose parent is already known not to have picked it does no
 * work (the walk cannot reach it; the results do not depend on this).  Supported: 1 <= N <= 65536; at most 16 children per node; valid ids as hawk_cfg_accept.
 * A child range that breaks these rules is clamped and flagged HAWK_DEV_BAD_TREE; the walk always ends.
 * Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE, PARAM, CUDA.  B == 0 returns HAWK_OK.
 * ---------------------------------------------------------------------------------------------- */
size_t hawk_tree_accept_workspace_bytes(int B, int N);

hawk_status hawk_tree_accept(const float *logits, const float *q_probs, const int32_t *node_token,
                             const int32_t *node_q, const int32_t *child_begin, const float *u_accept,
                             const float *u_resample, int B, int N, int NQ, int V, int v_begin, int v_end,
                             float cfg_scale, float temperature, int top_k, int max_depth,
                             int32_t *accept_len, int32_t *out_token, int32_t *path, void *workspace,
                             size_t workspace_bytes, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * Guidance fused into the output head (generation settings of Sec. 5: guidance scale and temperature
 * applied to the target's logits before top-k and sampling).  The paper does not separate these
 * steps; the three calls below are the two-call form of hawk_head_proj + hawk_cfg_accept /
 * hawk_tree_accept in which the conditional and the unconditional logit rows never reach memory.
 *
 * hawk_head_proj_cfg: guided[b*rows + i][v] = (lu + cfg_scale * (lc - lu)) / temperature, with
 *     lc = sum_c x[b*rows + i][c] * w[v][c],   lu = sum_c x[(B + b)*rows + i][c] * w[v][c]
 * for v_begin <= v < v_end: the accumulators of hawk_head_proj combined in fp32 by subtract, fused
 * multiply-add, divide (step 1 of hawk_cfg_accept, on the same numbers), so the two-call form decides
 * exactly as the three-call form does.  (Where a call has few tiles and a long hidden dimension, both
 * hawk_head_proj and this call sum each logit as two halves of the hidden dimension, in the same way.)
 *   x       bf16 [2B][rows][hidden]   conditional streams first, as everywhere
 *   w       bf16 [V][hidden]
 *   guided  fp32 [B][rows][V]         columns outside [v_begin, v_end) are not written
 * Supported: hidden a multiple of 64.  Errors as hawk_head_proj, plus PARAM (temperature <= 0, NaN, inf).
 *
 * hawk_cfg_accept_guided / hawk_tree_accept_guided: hawk_cfg_accept / hawk_tree_accept from step 2 on,
 * reading `guided` fp32 [B][K(+1)][V] / [B][N][V] instead of the two logit rows (no guidance scale,
 * no temperature: both are already applied).  NaN or +inf in `guided` is treated as -inf and flagged
 * HAWK_DEV_NONFINITE.  All other arguments, limits, workspaces and errors as the calls they mirror.
 * ---------------------------------------------------------------------------------------------- */
hawk_status hawk_head_proj_cfg(const void *x, const void *w, float *guided, int B, int rows, int hidden, int V,
                               int v_begin, int v_end, float cfg_scale, float temperature, int32_t *dev_status,
                               hawk_stream_t stream);

hawk_status hawk_cfg_accept_guided(const float *guided, const float *q_probs, const int32_t *draft,
                                   const float *u_accept, const float *u_resample, int B, int K, int V, int v_begin,
                                   int v_end, int top_k, int has_bonus_row, int32_t *accept_len, int32_t *out_token,
                                   float *p_debug, void *workspace, size_t workspace_bytes, int32_t *dev_status,
                                   hawk_stream_t stream);

hawk_status hawk_tree_accept_guided(const float *guided, const float *q_probs, const int32_t *node_token,
                                    const int32_t *node_q, const int32_t *child_begin, const float *u_accept,
                                    const float *u_resample, int B, int N, int NQ, int V, int v_begin, int v_end,
                                    int top_k, int max_depth, int32_t *accept_len, int32_t *out_token, int32_t *path,
                                    void *workspace, size_t workspace_bytes, int32_t *dev_status,
                                    hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * Speculation cache and spatial sampling pool (Sec. 4.2, "Dual Direction Drafting Heads" and "Spatial
 * Sampling Pool", Eqs. 1-5): the step that hands hawk_tree_accept its draft distributions and tokens.
 *
 * Eq. 1: the vertical draft head of depth d (1 <= d <= VSD), run at raster position T of an image IW
 * tokens wide, predicts the token at T + IW * d.  Eq. 2: those predictions wait in a cache of
 * IW * VSD * (VSD + 1) / 2 rows per sequence until decoding reaches their target.  Eqs. 3-5: the pool
 * of speculation point T + n is the horizontal head's distribution for T + n followed, for
 * dv = 1 .. VSD, by the cached depth-dv prediction made at T + n - IW * dv.
 *
 * Device layout, owned by the caller, B sequences:
 *   cache_rows  fp32  [B][slots][V]   slots = hawk_spec_cache_slots(IW, VSD)
 *   cache_tags  int32 [B][slots]      raster position that wrote the slot, -1 = never written
 * hawk_spec_cache_slot gives the slot of the depth-d prediction made at `position`: predictions of one
 * image column and depth that are alive at the same time come from d consecutive rows, so the row
 * modulo d tells them apart.  Positions of a sequence must not decrease between calls (a new image
 * starts with hawk_spec_cache_clear).  A lookup whose slot carries another position finds nothing: no
 * forward pass started there (the position was accepted inside a step) or it lies above the image.
 *
 * hawk_spec_cache_slots    slots per sequence (Eq. 2); 0 if IW < 1 or VSD < 1.  Host only.
 * hawk_spec_cache_slot     slot index as above, -1 for arguments out of range.  Host only.
 * hawk_spec_cache_clear    marks every slot of B sequences unwritten.
 * hawk_spec_cache_put      stores q_vert fp32 [B][VSD][V] (row d-1 = depth d) made at position[b]
 *                          (int32 [B], device; a negative position stores nothing for that sequence).
 * hawk_pool_build          q_horiz fp32 [B][K][V] (row n-1 = the horizontal distribution for T + n),
 *                          position int32 [B] (T of every sequence) ->
 *                          pool_q fp32 [B][K*(1+VSD)][V], row (n-1)*(1+VSD) + j: j = 0 horizontal,
 *                          j = dv >= 1 the cached vertical prediction, or a copy of the horizontal row
 *                          where none is cached; pool_source int32 [B][K*(1+VSD)] (may be NULL): 0, dv,
 *                          or -dv for the stand-in.  pool_q is laid out as hawk_tree_accept's q_probs
 *                          with NQ = K*(1+VSD).
 * hawk_pool_sample         draws one token per pool row by inverse CDF in ascending id over
 *                          [v_begin, v_end) with u fp32 [B][NQ] in [0,1) (negative weights count as
 *                          zero; a row without mass gives -1), then fills
 *                          node_token int32 [B][N]: node_token[b][i] = draw of row node_q[i]
 *                          (node_q int32 [N], device, as in hawk_tree_accept; the root, i = 0, gets 0).
 *                          The candidate tree is the Cartesian product of the per-position draws, so
 *                          all nodes that stand for one pool row carry the same token.  A node_q entry
 *                          outside [0, NQ) is clamped and flagged HAWK_DEV_BAD_TREE in *dev_status.
 *                          workspace: hawk_pool_sample_workspace_bytes(B, NQ) bytes, 16-byte aligned.
 * All pointers are device pointers unless stated; rows are copied with 16-byte accesses when V % 4 == 0
 * and the buffers are 16-byte aligned, element by element otherwise.  Limits: VSD <= 8; the valid id
 * range of hawk_pool_sample at most 32768 wide.  Launches are asynchronous on `stream`.
 * Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE, CUDA.  B == 0 (or K == 0) returns HAWK_OK.
 * ---------------------------------------------------------------------------------------------- */
int hawk_spec_cache_slots(int IW, int VSD);

int hawk_spec_cache_slot(int IW, int VSD, int position, int depth);

hawk_status hawk_spec_cache_clear(int32_t *cache_tags, int B, int IW, int VSD, hawk_stream_t stream);

hawk_status hawk_spec_cache_put(const float *q_vert, const int32_t *position, float *cache_rows,
                                int32_t *cache_tags, int B, int IW, int VSD, int V, hawk_stream_t stream);

hawk_status hawk_pool_build(const float *q_horiz, const float *cache_rows, const int32_t *cache_tags,
                            const int32_t *position, float *pool_q, int32_t *pool_source, int B, int K, int IW,
                            int VSD, int V, hawk_stream_t stream);

size_t hawk_pool_sample_workspace_bytes(int B, int NQ);

hawk_status hawk_pool_sample(const float *pool_q, const float *u, const int32_t *node_q, int32_t *node_token,
                             int B, int NQ, int N, int V, int v_begin, int v_end, void *workspace,
                             size_t workspace_bytes, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_cfg_accept_noalloc - hawk_cfg_accept without a caller-provided workspace.
 *
 * The paper has no counterpart of this call; it exists for the way the library gets embedded.
 * Some callers cannot obtain device memory at the moment they need a verdict: a decode loop running
 * inside a serving engine whose memory manager took the whole device at start-up (a fresh
 * allocation there fails, or stalls every stream while the driver serves it), or a plug-in that is
 * handed its input and output buffers by a host application and owns nothing else.  For them the
 * per-row verdicts go to a fixed 64 KiB array that is part of the library's device image; every GPU
 * that loads the library carries that array until the process exits.
 *
 * Same operation, arguments and results as hawk_cfg_accept, minus p_debug, workspace and
 * workspace_bytes.  Limit: B * (K + 1) <= hawk_cfg_accept_noalloc_max_rows() (16384); a larger step
 * returns HAWK_ERR_WORKSPACE and launches nothing.  The call allocates and frees nothing.
 *
 * The first call on each device looks up the array's device address (one runtime query, made with
 * that device current); make that first call outside any stream capture.
 * All calls on a device share the one array, and it keeps the previous call's contents.  Nothing in
 * it has to start at zero (each row's slot is rewritten before it is read), but two calls whose
 * kernels overlap on the GPU - different streams without an ordering between them - race on it:
 * order such calls, or give the concurrent ones their own workspace through hawk_cfg_accept.
 * ---------------------------------------------------------------------------------------------- */
size_t hawk_cfg_accept_noalloc_max_rows(void);

hawk_status hawk_cfg_accept_noalloc(const float *logits, const float *q_probs, const int32_t *draft,
                                    const float *u_accept, const float *u_resample, int B, int K, int V,
                                    int v_begin, int v_end, float cfg_scale, float temperature,
                                    int top_k, int has_bonus_row, int32_t *accept_len,
                                    int32_t *out_token, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_verify_step_host - one whole verify step with the per-step inputs in HOST memory.
 *
 * Runs, on `stream`: host->device copies of the step's inputs into the caller's device staging,
 * hawk_verify_attn, hawk_head_proj, hawk_cfg_accept (contracts above, no bonus row), and
 * device->host copies of accept_len and out_token.  The attention output and the head input are
 * separate tensors: the layers between them (output projection, MLP, norm) are not part of this
 * library, so x is an input of the step like q.  The inputs that only the accept stage reads are
 * copied on a second stream that the library owns (created by the first call on a device: make that
 * call outside stream capture), forked from and joined back into `stream` by events, so they travel
 * while attention and the head projection run.  The call returns once everything is queued; the
 * results are valid after the stream has been synchronised.  Use pinned host memory for the copies
 * to be asynchronous.  The KV cache, the head weight and the prefix lengths are resident device
 * state; all d_* staging and workspaces are device memory owned by the caller.
 * State kept by this call: the first call on a device creates one non-blocking stream and two events
 * for that device and keeps them until the process exits (no device memory).  Every call on the device
 * uses them, so the queuing part of a call runs under a per-device mutex: calls from several host
 * threads are queued one after the other, each correctly ordered against its own `stream`, and the
 * late copies of steps that are in flight together share the one side stream.
 * Errors: the argument checks of all three stage calls run before anything is queued, on the staging
 * pointers and sizes the stages will be given, so a call refused for its arguments (any code but
 * HAWK_ERR_CUDA) has queued no copy and no kernel.  HAWK_ERR_CUDA means the runtime refused a copy,
 * an event or a launch after the call had started to queue work.
 * ---------------------------------------------------------------------------------------------- */
typedef struct {
    /* sizes and sampling parameters */
    int B, K, H, H_kv, D, L_cap, max_prefix_len, V, v_begin, v_end, top_k;
    float sm_scale, cfg_scale, temperature;
    /* per-step inputs, host */
    const void *h_q;            /* bf16 [2B][K][H][D]      */
    const void *h_x;            /* bf16 [2B*K][H*D]        */
    const float *h_q_probs;     /* fp32 [B][K][V]          */
    const int32_t *h_draft;     /* [B][K]                  */
    const float *h_u_accept;    /* [B][K]                  */
    const float *h_u_resample;  /* [B][K+1]                */
    /* per-step results, host */
    int32_t *h_accept_len;      /* [B] */
    int32_t *h_out_token;       /* [B] */
    /* resident device state */
    const void *d_k_cache, *d_v_cache;   /* bf16 [2B][H_kv][L_cap][D] */
    const int32_t *d_prefix_len;         /* [2B] */
    const void *d_w;                     /* bf16 [V][H*D] */
    /* device staging for the inputs, intermediates and results (same shapes as above) */
    void *d_q, *d_x;
    float *d_q_probs;
    int32_t *d_draft;
    float *d_u_accept, *d_u_resample;
    void *d_attn_out;           /* bf16 [2B][K][H*D] */
    float *d_logits;            /* fp32 [2B*K][V]    */
    int32_t *d_accept_len, *d_out_token;
    void *d_attn_workspace;
    size_t attn_workspace_bytes;
    void *d_accept_workspace;
    size_t accept_workspace_bytes;
    int32_t *d_status;          /* optional */
} hawk_step_host_args;

hawk_status hawk_verify_step_host(const hawk_step_host_args *args, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * Heads, pages and chunks: the calls around a PAGED key/value cache.
 *
 * The paper's target model runs its attention on rotated (and, for some models, normalised) query and
 * key heads over a KV cache (App. C mentions the cache; Sec. 5 the model); it gives none of these steps.
 * The calls below are the textbook operations on the cache layout that serving engines use.
 *
 * Batch layout shared by hawk_rope_append and hawk_paged_attn.  S streams bring new rows of unequal
 * number, packed one stream after the other:
 *   row_begin    int32 [S+1], device, non-decreasing, within [0, T]: stream s owns rows
 *                row_begin[s] .. row_begin[s+1]-1 of the T rows; n_s = their number (0: the stream is
 *                idle).  Rows of no stream (padding in front or behind) are neither read into a
 *                result nor written.
 *   kv_len       int32 [S], device: keys of the stream INCLUDING its n_s new rows; new row i is cache row
 *                kv_len[s] - n_s + i.  Entries of idle streams are ignored.
 *   block_table  int32 [S][table_width], device: entry j is the page that holds cache rows
 *                j * page_size .. (j+1) * page_size - 1.  Entries past the last used page may hold anything.
 *   k_pages, v_pages  16-bit, element (page, head, row, d) at page * page_stride + head * head_stride +
 *                row * row_stride + d (strides in elements): [n_pages][H_kv][page_size][D], the same with
 *                rows before heads, keys and values in one buffer are all expressible.  A dense cache
 *                [S][H_kv][L_cap][D] is the paged one with page_size = L_cap and block_table[s][0] = s.
 * dtype is HAWK_BF16 or HAWK_F16 and holds for every 16-bit tensor of the call.  All 16-bit bases are
 * 16-byte aligned and all strides multiples of 8 elements (16 bytes); D is 64 or 128.
 * ---------------------------------------------------------------------------------------------- */
#define HAWK_BF16 0
#define HAWK_F16 1

#define HAWK_NORM_NONE 0
#define HAWK_NORM_RMS 1
#define HAWK_NORM_LAYER 2

/* ------------------------------------------------------------------------------------------------
 * hawk_qk_norm_rope - norm of every query and key head, then the position rotation, in one pass.
 *
 * Operation, per row t and head h of q (and likewise of k), with x = q[t][h][0..D-1] in fp32:
 *   HAWK_NORM_RMS    x <- x / sqrt(mean(x^2) + eps) * weight
 *   HAWK_NORM_LAYER  x <- (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) * weight + bias
 *   HAWK_NORM_NONE   x as it is
 * then with c_i = cos_sin[position[t]][i], s_i = cos_sin[position[t]][rot_dim/2 + i], i < rot_dim/2, each
 * pair (a, b) of elements becomes (a*c_i - b*s_i, b*c_i + a*s_i); the pair is (x[i], x[i + rot_dim/2]), or
 * (x[2i], x[2i+1]) with `interleaved`.  Elements from rot_dim on are not rotated.  Everything is fp32
 * up to ONE rounding to the output type.  The table is the caller's: one axis (angle = position * base^(-2i/rot_dim)),
 * or an image's raster (half the angles by row, half by column), and nodes of a candidate tree at the same depth
 * simply share a position.
 *
 *   q, k         16-bit [T][H][D], [T][H_kv][D] at row and head strides (elements), so that both may be parts of
 *                one projection's output.  H or H_kv may be 0 (that tensor is absent).
 *   q_out, k_out the same shapes, own strides; may be q and k themselves (same strides), else must not overlap them
 *   q_weight, k_weight, q_bias, k_bias   16-bit [D], or with per_head [H][D] / [H_kv][D]; weights are required by a
 *                norm of that tensor; a bias may be NULL (none) and goes with HAWK_NORM_LAYER only; all four are ignored
 *                with HAWK_NORM_NONE
 *   position     int32 [T]
 *   cos_sin      fp32 [n_positions][rot_dim], 16-byte aligned
 * Supported: D in {64, 128}; rot_dim a multiple of 16, 0 <= rot_dim <= D (0: no rotation, position and
 * cos_sin are not read).  A position outside [0, n_positions) is clamped and flagged HAWK_DEV_BAD_POSITION.
 * Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, PARAM (eps not a finite number >= 0, unknown dtype or norm, a bias under
 * HAWK_NORM_RMS), CUDA.
 * T == 0 returns HAWK_OK without a launch.
 * ---------------------------------------------------------------------------------------------- */
typedef struct hawk_qk_rope_args {
    int dtype, T, H, H_kv, D;
    int norm, per_head, rot_dim, n_positions, interleaved;
    float eps;
    const void *q, *k;
    void *q_out, *k_out;
    long long q_row_stride, q_head_stride, k_row_stride, k_head_stride;
    long long q_out_row_stride, q_out_head_stride, k_out_row_stride, k_out_head_stride;
    const void *q_weight, *k_weight, *q_bias, *k_bias;
    const int32_t *position;
    const float *cos_sin;
} hawk_qk_rope_args;

hawk_status hawk_qk_norm_rope(const hawk_qk_rope_args *args, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_rope_append - the new rows' keys and values into the paged cache, normalised and rotated on the way.
 *
 * Operation: k goes through hawk_qk_norm_rope's operation and lands in k_pages, v is copied to v_pages, at
 * the cache row the batch layout above gives each new row; q (H > 0) goes through the same operation
 * into q_out.  Rows of no stream are skipped in all three.  qk.k_out and its strides are ignored.
 *   v   16-bit [T][H_kv][D] at its own strides
 * page_size may be any positive number here.  Two rows sent to the same place of the same page (streams that
 * share a page they both write) leave either.
 * A cache row outside [0, table_width * page_size) skips the row's k and v and is flagged HAWK_DEV_BAD_PREFIX, a page id
 * outside [0, n_pages) the same with HAWK_DEV_BAD_PAGE; q_out is written all the same.
 * Errors as hawk_qk_norm_rope.  T == 0 or S == 0 returns HAWK_OK without a launch.
 * ---------------------------------------------------------------------------------------------- */
typedef struct hawk_rope_append_args {
    hawk_qk_rope_args qk;
    const void *v;
    long long v_row_stride, v_head_stride;
    void *k_pages, *v_pages;
    long long k_page_stride, k_page_head_stride, k_page_row_stride;
    long long v_page_stride, v_page_head_stride, v_page_row_stride;
    int n_pages, page_size, S, table_width;
    const int32_t *block_table, *row_begin, *kv_len;
} hawk_rope_append_args;

hawk_status hawk_rope_append(const hawk_rope_append_args *args, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_paged_attn - attention of a chunk of new rows over the paged cache.
 *
 * Operation: for new row i of stream s (its own key already in the cache), query head h, kv head g = h / (H/H_kv),
 * with p = kv_len[s] - n_s cache rows in front of the chunk:
 *     visible keys   j <= p + i                                       (anc_mask NULL: chain)
 *                    j < p, and j = p + m, m < n_s, iff bit m of anc_mask[i] is set   (anc_mask: tree)
 *     out[row][h*D:(h+1)*D] = sum_j softmax(sm_scale * <q[row][h], k_j>)_j * v_j
 * A row that sees no key (p + i < 0; an empty mask without a prefix) gives zeros.  n_s = 1 is a decode step, up
 * to 64 rows a verify step (hawk_verify_attn, hawk_verify_attn_tree), thousands a chunk of a prompt; one call may mix
 * them.  Scores, maxima, sums and accumulators are fp32; the probabilities are rounded to the 16-bit type for the
 * second product, the result once.
 * Cache rows from kv_len[s] on are never used (they may hold anything, NaN included).  Rows below kv_len[s] must be
 * finite: a NaN or infinity among a stream's own rows may reach rows of that stream that do not see it.  Scores may have any
 * size that fp32 holds, before and after sm_scale.
 *
 *   q          16-bit [T][H][D] at row and head strides
 *   out        16-bit [T][H*D], dense; must not overlap any input
 *   anc_mask   uint64 [max_new], device, or NULL; row i of every stream uses entry i.  max_new <= 64 with it.
 *   max_new    upper bound of n_s known on the host; a stream with more rows is skipped, HAWK_DEV_BAD_ROWS
 *   max_kv     upper bound of kv_len of the streams that are not idle, <= table_width * page_size (sizes the launch
 *              and the workspace); a kv_len outside [0, max_kv] is clamped, HAWK_DEV_BAD_PREFIX
 *   workspace  at least hawk_paged_attn_workspace_bytes(...) bytes, 16-byte aligned, may be NULL when that is 0;
 *              no initialisation; the size is for exactly these arguments (a smaller call may need more).  Calls
 *              that may overlap on the GPU need one each.
 * A page id outside [0, n_pages) reads as zeros and is flagged HAWK_DEV_BAD_PAGE.
 * Supported: D in {64, 128}; page_size a multiple of 8; S <= 4096; max_kv <= 2^30; H a multiple of H_kv, H/H_kv <= 128.
 * Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE, PARAM, CUDA.  S == 0, T == 0 or max_new == 0 returns HAWK_OK
 * without a launch.
 * ---------------------------------------------------------------------------------------------- */
typedef struct hawk_paged_attn_args {
    int dtype, S, T, max_new, max_kv, H, H_kv, D;
    int n_pages, page_size, table_width;
    float sm_scale;
    const void *q;
    long long q_row_stride, q_head_stride;
    const void *k_pages, *v_pages;
    long long k_page_stride, k_page_head_stride, k_page_row_stride;
    long long v_page_stride, v_page_head_stride, v_page_row_stride;
    const int32_t *block_table, *row_begin, *kv_len;
    const uint64_t *anc_mask;
    void *out;
    void *workspace;
    size_t workspace_bytes;
} hawk_paged_attn_args;

size_t hawk_paged_attn_workspace_bytes(int S, int T, int max_new, int H, int H_kv, int D, int max_kv);

hawk_status hawk_paged_attn(const hawk_paged_attn_args *args, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_sample - one token from every row of logits, by given random numbers.
 *
 * The plain step beside the verification (Sec. 5 gives its settings: guidance, temperature, top-k): the first token behind a
 * prompt, streams without drafts, and the draft side, which draws its tokens and hands hawk_cfg_accept and hawk_tree_accept the
 * distributions they were drawn from (`probs`, laid out as their q_probs).
 *
 * Operation, per row r over the ids v_begin <= v < v_end:
 *   1. l[v] = lu[v] + cfg_scale*(lc[v] - lu[v]) in fp32 (subtract, fused multiply-add; -inf in either gives -inf), or the logit itself
 *      without guidance.  NaN and +inf count as -inf and are flagged HAWK_DEV_NONFINITE.
 *   2. top-k, 0 < top_k: ids below the top_k-th largest l leave; ties with it stay (as in hawk_cfg_accept).
 *   3. w[v] = exp((l[v] - max l) / temperature), 0 for ids that left.  top-p, top_p < 1: with t the largest value for which
 *      the w of all l >= t sum to at least top_p times the sum of all w, ids below t leave; ties with t stay.
 *   4. min-p, 0 < min_p: ids with exp((l - max l) / temperature) < min_p leave; the maximum always stays.
 *   5. token = the smallest id whose running sum of w (ascending id) exceeds u * sum(w); p = w / sum(w).
 * temperature 0: the lowest id of the maximum, with p = 1; steps 2 to 5 have no say.  A row without a finite logit: token -1, p = 0.
 * Exponentials are taken in fp64 and held as whole multiples of 2^-44 of the largest, sums of them in 64-bit integers: no order
 * changes a sum, so equal inputs give equal tokens whatever the launch (a w below 2^-45 counts as 0 and is never drawn, though
 * probs may show its p).
 *
 *   dtype        HAWK_F32, HAWK_BF16 or HAWK_F16: the logits' type
 *   logits       [R][V] at row_stride (elements, not negative; 0: all rows draw from one; any alignment that the type needs)
 *   uncond       the same at uncond_row_stride: the unconditional rows; NULL: no guidance
 *   temperature, top_k, top_p, min_p, cfg_scale      for all rows; top_k <= 0, top_p >= 1 and min_p <= 0 are off
 *   row_temperature, row_top_k, row_top_p, row_min_p, row_cfg_scale   device [R] or NULL: take the place of the number above.
 *                A row's NaN, or a temperature that is negative or infinite, is flagged HAWK_DEV_BAD_SETTING and taken as off
 *                (temperature 1).  row_cfg_scale is used as it is (one that is not finite leaves its row without a finite logit).
 *   u            fp32 [R], uniforms in [0,1); others are clamped into it
 *   token        int32 [R] (out)
 *   token_prob   fp32 [R] (out) or NULL: p of the token
 *   probs        fp32 [R][V] at probs_row_stride (out) or NULL: p, 0 outside the range
 * Supported: 1 <= v_end - v_begin <= 262144, R < 2^28.  No workspace.
 * Errors: NULL, SHAPE (a range outside [0, V], a negative stride, rows of probs that overlap), ALIGN (a base that its type cannot have), UNSUPPORTED,
 * PARAM (dtype; a temperature that is negative or not finite, a cfg_scale that is not finite, a NaN), CUDA.  R == 0 returns HAWK_OK without a launch.
 * ---------------------------------------------------------------------------------------------- */
#define HAWK_F32 2

typedef struct hawk_sample_args {
    int dtype, R, V, v_begin, v_end, top_k;
    float temperature, top_p, min_p, cfg_scale;
    const void *logits, *uncond;
    long long row_stride, uncond_row_stride;
    const float *row_temperature, *row_top_p, *row_min_p, *row_cfg_scale;
    const int32_t *row_top_k;
    const float *u;
    int32_t *token;
    float *token_prob, *probs;
    long long probs_row_stride;
} hawk_sample_args;

hawk_status hawk_sample(const hawk_sample_args *args, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_pages_* - the paged cache between two steps.
 *
 * State of a cache, in device memory and the caller's:
 *   block_table  int32 [S][table_width] and kv_len int32 [S], as for hawk_paged_attn: stream s uses its first
 *                ceil(kv_len[s] / page_size) entries; the others may hold anything and are not written
 *   page_refs    int32 [n_pages]: table entries in use that name the page.  0: the page is free.  A caller keeps a page out of use, or
 *                holds a prompt that no stream uses at the moment, by a count of its own on top.
 * The calls below work on the state alone, once for all layers, and say which pages have to be copied:
 *   copies       int32 [.][3]: page to copy from, page to copy to, rows (the first ones); -1, -1, 0: nothing
 * hawk_pages_copy does that for the pages of all layers, and hawk_pages_keep moves rows inside them.  Every out_* may be the tensor it
 * comes from (in place) unless the call says otherwise; tensors that overlap in part are not supported.  What is counted in this
 * section is whole numbers; results do not depend on the launch.
 * Lengths outside [0, table_width * page_size] are flagged HAWK_DEV_BAD_PREFIX and their streams stay as they are (without
 * entries, where it is the stream's own length that is out of range); a page id outside
 * [0, n_pages) is flagged HAWK_DEV_BAD_PAGE and nothing is counted for it.
 * Supported: S <= 4096, n_pages <= 2^20, page_size <= 65536, S * table_width and table_width * page_size + 65536 below 2^31.
 * page_refs, out_refs, workspaces and pages are 16-byte aligned, the other tensors as their type is.  A tensor without elements (a table
 * of no width, no layers) may be NULL, but for hawk_pages_keep's path, whose NULL says that there is none.
 *
 * hawk_pages_resize: stream s goes from kv_len[s] to new_len[s] keys.
 *   1. Streams that shrink release the entries they need no more (to 0: the stream is freed).  A count that is 0 already stays 0,
 *      HAWK_DEV_BAD_PAGE.
 *   2. A stream that grows takes ceil(new/page_size) - ceil(old/page_size) pages; and one more if its last page is partly filled and,
 *      after step 1, named by other entries too: it gets a copy of its own, copies[s] = (shared page, new page, old % page_size), and
 *      releases the shared one (all streams that grow into a shared page do, the last of them as well).
 *      (A last page whose count is then 0 or less, which its entry contradicts, is flagged HAWK_DEV_BAD_PAGE; by its count it is free, and
 *      may be given to a stream.)
 *      Pages are those that are free after step 1, lowest id first, to streams in ascending order, each stream's entries in ascending
 *      order (the copy's is the first).
 *   3. When the pages run out, the streams from there on that need any stay as they were, HAWK_DEV_NO_PAGES.
 *   out_len[s] = new_len[s], or kv_len[s] for a stream that stayed.  out_table gets the entries that are then in use.
 *   new_len may be out_len.  Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, CUDA.  S == 0: out_refs is copied.
 * ---------------------------------------------------------------------------------------------- */
typedef struct hawk_pages_resize_args {
    int S, table_width, n_pages, page_size;
    const int32_t *block_table, *kv_len, *new_len, *page_refs;
    int32_t *out_table, *out_len, *out_refs;
    int32_t *copies; /* [S][3] */
} hawk_pages_resize_args;

hawk_status hawk_pages_resize(const hawk_pages_resize_args *args, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_pages_fork - streams that continue others: out stream t has the first min(length[t], kv_len[p]) keys of stream p = parent[t]
 * (length NULL: all), none for p = -1.  Pages are shared: out_table[t] names the parent's, and out_refs = page_refs less the entries in
 * use of the S old streams plus those of the S_out new ones, whatever that gives.  So one call reorders a batch, has several streams go on from one, keeps some and
 * frees others.  hawk_pages_resize makes the copy when one of them grows into a shared page.
 * A parent outside [-1, S) is flagged HAWK_DEV_BAD_ROWS and taken as -1; a negative length counts as 0 and is flagged HAWK_DEV_BAD_PREFIX; a
 * stream whose kv_len is out of range has no entries.
 *   parent     int32 [S_out], length int32 [S_out] or NULL
 *   out_table  int32 [S_out][table_width], out_len int32 [S_out]: not block_table and kv_len (PARAM)
 * Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, PARAM, CUDA.
 * ---------------------------------------------------------------------------------------------- */
typedef struct hawk_pages_fork_args {
    int S, S_out, table_width, n_pages, page_size;
    const int32_t *block_table, *kv_len, *page_refs, *parent, *length;
    int32_t *out_table, *out_len, *out_refs;
} hawk_pages_fork_args;

hawk_status hawk_pages_fork(const hawk_pages_fork_args *args, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_pages_compact - pages in use to the lowest ids, at most max_moves of them a call: with f_0 < f_1 < ... the free pages and
 * u_0 > u_1 > ... the pages in use, all from first_page on, page u_i becomes page f_i for as long as f_i < u_i and i < max_moves.
 *   copies     int32 [max_moves][3]: copies[i] = (u_i, f_i, page_size)
 *   out_table  the table with the new ids, out_refs the counts that moved with them
 *   top        int32 [1] or NULL: all pages from this id on are free then (at least first_page, which is at most n_pages)
 *   workspace  at least hawk_pages_compact_workspace_bytes(n_pages, max_moves) bytes, 16-byte aligned, no initialisation; calls that may
 *              overlap on the GPU need one each
 * A page that the caller holds by a count of its own moves like the others (copies tell where).  n_pages >= 1.
 * Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE, CUDA.
 * ---------------------------------------------------------------------------------------------- */
typedef struct hawk_pages_compact_args {
    int S, table_width, n_pages, page_size, first_page, max_moves;
    const int32_t *block_table, *kv_len, *page_refs;
    int32_t *out_table, *out_refs;
    int32_t *copies; /* [max_moves][3] */
    int32_t *top;
    void *workspace;
    size_t workspace_bytes;
} hawk_pages_compact_args;

size_t hawk_pages_compact_workspace_bytes(int n_pages, int max_moves);

hawk_status hawk_pages_compact(const hawk_pages_compact_args *args, int32_t *dev_status, hawk_stream_t stream);

/* ------------------------------------------------------------------------------------------------
 * hawk_pages_copy - rows of pages to other pages, keys and values of all layers: for each of the n_copies entries (a, b, n) of
 * `copies` with a >= 0, rows 0 .. n-1 of page a to page b (n is clamped to [0, page_size]).  No page may be written by two
 * entries, or written by one and read by another (what the calls above give never is).  An id outside [0, n_pages) skips the
 * entry, HAWK_DEV_BAD_PAGE.
 *   k_pages, v_pages   16-bit, element (layer, page, head, row, d) at layer * layer_stride + page * page_stride +
 *                      head * head_stride + row * row_stride + d (strides in elements, multiples of 8; bases 16-byte aligned)
 * Supported: D a multiple of 8; page_size, H_kv and D at most 65536, H_kv * page_size * D <= 2^30; layers <= 32767.
 * Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, CUDA.  n_copies == 0 or layers == 0 returns HAWK_OK without a launch.
 *
 * hawk_pages_keep - the rows of an accepted path to the front of their block, and the length that the stream then has.  Stream s
 * has brought n_s rows (row_begin, kv_len: the batch of hawk_paged_attn, its keys at cache rows base = kv_len[s] - n_s on), and
 * a_s = accept_len[s % B] of them were accepted behind the first `first` rows, which stay: with path, row base + path[s % B][i] moves to
 * row base + first + i for i < a_s, and out_len[s] = base + min(n_s, first + a_s).
 * first = 1 and path, accept_len are what hawk_tree_accept gives for streams b and B + b of sequence b, whose row 0 is the root.  Without
 * path (NULL: a chain, whose rows lie in order) nothing moves, the page arguments are not looked at, and only out_len is written.
 * The path has to ascend, from `first` on and below n_s, as the nodes of a tree do; a stream whose path does not, or whose accept_len lies
 * outside [0, path_width] (without path: is negative), stays as it was with out_len = kv_len, HAWK_DEV_BAD_TREE.  An idle stream (n_s = 0)
 * stays as well.  A stream whose rows or length contradict the batch is flagged HAWK_DEV_BAD_ROWS or HAWK_DEV_BAD_PREFIX and stays; a row
 * with a page id outside [0, n_pages) on either side is skipped, HAWK_DEV_BAD_PAGE.  The rows that move lie in pages of their stream alone
 * (hawk_pages_resize sees to that when it makes room for them).
 *   path  int32 [B][path_width] or NULL, accept_len int32 [B], S a multiple of B; out_len int32 [S], not kv_len (PARAM)
 * Limits of the pages as above.  Errors: NULL, SHAPE, ALIGN, UNSUPPORTED, PARAM, CUDA.  S == 0 returns HAWK_OK without a launch.
 * ---------------------------------------------------------------------------------------------- */
typedef struct hawk_page_tensors {
    int layers, n_pages, H_kv, page_size, D;
    void *k_pages, *v_pages;
    long long k_layer_stride, k_page_stride, k_head_stride, k_row_stride;
    long long v_layer_stride, v_page_stride, v_head_stride, v_row_stride;
} hawk_page_tensors;

hawk_status hawk_pages_copy(const hawk_page_tensors *pages, const int32_t *copies, int n_copies, int32_t *dev_status,
                            hawk_stream_t stream);

typedef struct hawk_pages_keep_args {
    hawk_page_tensors pages;
    int S, B, table_width, path_width, first;
    const int32_t *block_table, *row_begin, *kv_len, *path, *accept_len;
    int32_t *out_len;
} hawk_pages_keep_args;

hawk_status hawk_pages_keep(const hawk_pages_keep_args *args, int32_t *dev_status, hawk_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* HAWK_H */
