/*
 * fspad.h - C ABI of the tree-verification hot path of draft-then-verify
 * lossless speculative decoding (arXiv 2408.15562, section "Preliminaries").
 *
 * One verification step of the target model over a flattened draft tree:
 *   1. tree-masked attention: every tree node attends to the whole prefix
 *      KV cache and, among the tree tokens, only to its ancestors and itself
 *      (Preliminaries: the draft phase ends by deriving the target's attention
 *      mask from the token tree; the validation phase applies it);
 *   2. lossless acceptance over the per-node logits: strict comparison of the
 *      tree with the target's results, differing tokens and their descendants
 *      discarded (Preliminaries, validation-phase paragraph), either greedy
 *      (temperature 0) or by rejection sampling that leaves the target's output
 *      distribution unchanged (Experiments, "Settings": temperature 1, and the
 *      caption of Table 1: acceptance conditions are not relaxed); also in the
 *      general form for drafts sampled from a draft distribution
 *      (fspad_tree_accept_sample_draft).
 * and the calls around that step:
 *   3. the same acceptance straight from the target's last hidden states, fused
 *      with the LM head (fspad_tree_accept_{greedy,sample}_lm_head);
 *   4. the commit of the accepted path's keys / values to the cache
 *      (fspad_kv_commit);
 *   5. on the draft side: the Feature Sampler (Methodology, "Feature Sampling":
 *      fspad_feature_sampler), the draft decoder layer with the doubled MLP
 *      output ("Partial Alignment Distillation": fspad_draft_layer), the top-k cut of
 *      a draft step's output and the
 *      choice of the tree from the candidates (Preliminaries, last paragraph:
 *      fspad_draft_topk, fspad_tree_build);
 *   6. the same attention over a paged 4-bit cache, with the calls that keep it (fspad_tree_attn_paged,
 *      fspad_page_map, fspad_kv_store_paged, fspad_kv_load_paged), and over a paged 8-bit one
 *      (fspad_tree_attn_paged_byte, fspad_kv_store_paged_byte, fspad_kv_load_paged_byte);
 *   7. sequences that share pages of either: fspad_page_fork, fspad_page_release, fspad_page_compact,
 *      fspad_page_copy.
 *
 * Conventions that hold for every entry point:
 *   - "dev" pointers are device (HBM) addresses, "host" pointers are host
 *     addresses. Every buffer is owned by the caller. The library allocates
 *     nothing, frees nothing and never synchronises: device work is enqueued
 *     on the caller's HIP stream (`hip_stream` is a hipStream_t, NULL = the
 *     default stream) and the call returns at once.
 *   - The return code covers what the host can see (null pointers, shapes,
 *     workspace size, launch errors). Tree well-formedness of device arrays is
 *     the caller's contract; fspad_tree_validate checks host copies.
 *   - Results are deterministic from call to call (no floating-point atomics).
 *   - Tree layout: nodes 0..N-1 in topological order, node 0 is the root (the
 *     last token the target already emitted, always accepted; its K/V are not
 *     yet in the cache). parent[0] = -1 and 0 <= parent[i] < i. Siblings are
 *     ordered by draft rank; that order is the order of the rejection tests.
 */
#ifndef FSPAD_H
#define FSPAD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FSPAD_MAX_NODES 64 /* one 64-bit ancestor word per node */

typedef enum {
  FSPAD_OK = 0,
  FSPAD_ERR_NULL = 1,        /* a required pointer is NULL */
  FSPAD_ERR_SHAPE = 2,       /* B<1, N<1, N>64, D not in {64,128}, Hq%Hkv!=0, V<1, n_nodes[b] not in 1..Nmax,
                                kv_len[b]<0, strides too small or not 16-byte multiples, row_stride<V */
  FSPAD_ERR_TREE = 3,        /* validate(): parent[0]!=-1, parent[i] not in [0,i), token not in [0,V),
                                two siblings with the same token */
  FSPAD_ERR_DTYPE = 4,       /* io_dtype / out_dtype combination not supported */
  FSPAD_ERR_WORKSPACE = 5,   /* workspace NULL or smaller than *_workspace_bytes() says */
  FSPAD_ERR_TEMPERATURE = 6, /* temperature <= 0 or not finite */
  FSPAD_ERR_HIP = 7          /* a HIP launch failed; hipGetLastError() has the cause */
} fspad_status;

typedef enum { FSPAD_F32 = 0, FSPAD_BF16 = 1 } fspad_dtype;

/* Geometry of one attention call. All strides are in elements of io_dtype. */
typedef struct {
  int32_t batch;           /* B >= 1 */
  int32_t n_nodes_max;     /* Nmax, 1..64: row pitch of every [B,Nmax,...] array */
  int32_t n_q_heads;       /* Hq */
  int32_t n_kv_heads;      /* Hkv, divides Hq; query head h reads kv head h / (Hq/Hkv) */
  int32_t head_dim;        /* D: 64 or 128, contiguous in every array */
  int32_t io_dtype;        /* fspad_dtype of q, k_tree, v_tree, k_cache, v_cache */
  int32_t out_dtype;       /* FSPAD_F32, or the same as io_dtype */
  float softmax_scale;     /* 0 => 1/sqrt(D) */
  int64_t cache_stride_batch; /* k_cache/v_cache element (b,g,j,d) is at                */
  int64_t cache_stride_head;  /*   b*stride_batch + g*stride_head + j*stride_token + d  */
  int64_t cache_stride_token; /* >= D; all three multiples of 8 elements (16 bytes bf16) */
  int32_t workgroups;      /* tuning: 0 = the built-in choice; 1..4096 forces the number of workgroups the
                              bf16 path spreads its key blocks over. Results do not depend on it beyond
                              fp32 rounding of the merge; fspad_tree_attn_workspace_bytes reads it too, so
                              sizing and call must see the same value */
  int32_t reserved;        /* 0 */
} fspad_attn_desc;

/*
 * Tree-masked attention (Preliminaries, validation phase: one forward of the
 * target over the flattened tree with the tree mask).
 *
 *   out[b,i,h,:] = sum_j softmax_j( scale * q[b,i,h,:] . K_j ) * V_j
 * where j runs over the kv_len[b] prefix positions of kv head g = h/(Hq/Hkv)
 * (all visible) followed by the tree tokens t < n_nodes[b] whose bit t is set
 * in anc_mask[b,i] (the ancestors of i and i itself).
 *
 *   q        dev [B,Nmax,Hq,D]   io_dtype (already position-encoded)
 *   k_tree   dev [B,Nmax,Hkv,D]  io_dtype, keys of the tree tokens
 *   v_tree   dev [B,Nmax,Hkv,D]  io_dtype
 *   k_cache  dev strided [B,Hkv,>=kv_len,D] io_dtype (may be NULL if all kv_len are 0)
 *   v_cache  dev strided, same strides
 *   kv_len   HOST [B] prefix lengths >= 0 (host, so that the split plan needs no device read)
 *   n_nodes  HOST [B] 1..Nmax
 *   anc_mask dev [B,Nmax] u64, bit t of word [b,i] set <=> t is i or an ancestor of i
 *   out      dev [B,Nmax,Hq,D] out_dtype; rows i >= n_nodes[b] are written as zeros
 *   workspace dev, at least fspad_tree_attn_workspace_bytes(desc, max_b kv_len[b]) bytes,
 *            16-byte aligned; contents on entry are ignored, undefined on exit.
 *            Two calls that may overlap in time need different workspaces.
 * Accumulation is fp32; bf16 inputs are multiplied on the matrix cores with
 * probabilities rounded to bf16.
 */
size_t fspad_tree_attn_workspace_bytes(const fspad_attn_desc* desc, int32_t max_kv_len);

fspad_status fspad_tree_attn(const fspad_attn_desc* desc,
                             const void* q, const void* k_tree, const void* v_tree,
                             const void* k_cache, const void* v_cache,
                             const int32_t* kv_len, const int32_t* n_nodes,
                             const uint64_t* anc_mask, void* out,
                             void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Greedy lossless acceptance (Preliminaries, validation phase: strict
 * comparison, differing tokens and their descendants discarded).
 *
 *   a[i]   = argmax_v logits[b,i,v]   (fp32 compare; ties -> lowest v; NaN never wins)
 *   walk   : cur = 0; while some child c of cur (lowest index first) has
 *            draft_tokens[c] == a[cur]: cur = c
 *   path   = root .. cur ; tokens = draft tokens of path[1..] then the bonus a[cur]
 *
 *   logits       dev [B,Nmax,V] fp32, row (b,i) starts at (b*Nmax+i)*row_stride
 *   draft_tokens dev [B,Nmax] i32; [b,0] is the root's token (not compared)
 *   parent       dev [B,Nmax] i32; [b,0] = -1, parent[i] < i
 *   n_nodes      dev [B] i32, 1..Nmax
 *   path         dev [B,Nmax] i32 out; path[b,0] = 0; entries >= path_len[b] are -1
 *   path_len     dev [B] i32 out, >= 1
 *   tokens       dev [B,Nmax] i32 out; tokens[b,0..len-2] = draft tokens of path[b,1..len-1],
 *                tokens[b,len-1] = bonus token (the next step's root); later entries -1
 *   n_tokens     dev [B] i32 out, = path_len[b]
 *   workspace    dev, >= fspad_tree_accept_workspace_bytes(B,Nmax,V), 16-byte aligned
 */
size_t fspad_tree_accept_workspace_bytes(int32_t B, int32_t Nmax, int32_t V);

fspad_status fspad_tree_accept_greedy(int32_t B, int32_t Nmax, int32_t V,
                                      const float* logits, int64_t row_stride,
                                      const int32_t* draft_tokens, const int32_t* parent,
                                      const int32_t* n_nodes,
                                      int32_t* path, int32_t* path_len,
                                      int32_t* tokens, int32_t* n_tokens,
                                      void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * fspad_tree_accept_greedy for callers that cannot allocate device memory or pass a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * kernels, arguments and results, with the per-(row, chunk) statistics kept in a fixed device
 * array that is part of the library image instead of a caller workspace.
 *
 *   limit   fspad_tree_accept_workspace_bytes(B,Nmax,V) <= FSPAD_STATIC_SCRATCH_BYTES (1 MiB; e.g.
 *           B*Nmax = 512 rows of V = 128256); larger problems return FSPAD_ERR_WORKSPACE and
 *           nothing is launched
 *   memory  every GPU the library runs on holds the 1 MiB array until the process ends; its
 *           address is looked up once per device, on the first call there
 *   calls   allocates nothing, frees nothing, never synchronises. All calls on one GPU share that
 *           GPU's array: two calls that may overlap in time (different streams) race; calls
 *           on one stream are ordered and need nothing cleared between them
 * Errors otherwise as for fspad_tree_accept_greedy; FSPAD_ERR_HIP if the array's address cannot
 * be resolved.
 */
#define FSPAD_STATIC_SCRATCH_BYTES (1u << 20)
fspad_status fspad_tree_accept_greedy_static(int32_t B, int32_t Nmax, int32_t V,
                                             const float* logits, int64_t row_stride,
                                             const int32_t* draft_tokens, const int32_t* parent,
                                             const int32_t* n_nodes,
                                             int32_t* path, int32_t* path_len,
                                             int32_t* tokens, int32_t* n_tokens, void* hip_stream);

/*
 * Sampling (temperature > 0) lossless acceptance: rejection sampling down the
 * tree against the residual distribution, with caller-supplied uniforms, so
 * that the emitted tokens are distributed exactly as the target's own samples
 * (Experiments "Settings", temperature 1; caption of Table 1). The draft
 * proposal at a child is a point mass (children are a deterministic top-k of
 * the draft's output, Preliminaries, last paragraph), which reduces the
 * accept-or-resample rule of the speculative sampling the paper builds on to:
 *
 *   cur = 0
 *   loop: w[v] = exp((logits[cur,v] - max_v logits[cur,v]) / T), Z = sum_v w[v]   (fp64)
 *         for each child c of cur, lowest index first, x = draft_tokens[c]:
 *             if u_acc[c] * Z < w[x]: accept, cur = c, restart loop
 *             else: Z -= w[x]; w[x] = 0         (residual: p with x removed, renormalised)
 *         none accepted: t = u_bonus[cur] * Z;
 *             bonus = first v in vocabulary order whose running sum of w exceeds t
 *             (if rounding leaves none: the last v with w[v] > 0); stop.
 *
 * Arguments as for greedy, plus:
 *   temperature  > 0, finite
 *   uniforms     dev [B,2,Nmax] fp32 in [0,1): [b,0,i] = u_acc(i) tested when node i is
 *                proposed, [b,1,i] = u_bonus(i) used if the walk stops at node i
 * w, Z and the running sums are fp64. A result is only defined bit-for-bit when
 * every comparison above has a relative margin well above fp64 rounding (the
 * tests require 1e-9).
 */
fspad_status fspad_tree_accept_sample(int32_t B, int32_t Nmax, int32_t V,
                                      const float* logits, int64_t row_stride,
                                      const int32_t* draft_tokens, const int32_t* parent,
                                      const int32_t* n_nodes,
                                      float temperature, const float* uniforms,
                                      int32_t* path, int32_t* path_len,
                                      int32_t* tokens, int32_t* n_tokens,
                                      void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Lossless acceptance for drafts that were SAMPLED from a draft distribution (Introduction: the
 * draft-then-verify scheme of speculative sampling, whose accept-or-resample rule is what keeps the
 * target's output distribution; fspad_tree_accept_sample is its special case for the deterministic
 * top-k drafts of the paper's trees, where the draft distribution is a point mass).
 *
 * At a node with target distribution p = softmax(logits / T) and draft distribution
 * q = softmax(draft_logits / T), the children -- drawn from q one after another without
 * replacement, stored in that order -- are tested in order:
 *   accept x  <=>  u_acc * q(x) < p(x)                       (probability min(1, p(x) / q(x)))
 *   reject x   :   p <- max(p - q, 0) / sum_v max(p - q, 0);  q(x) <- 0,  q <- q / sum_v q
 * When no child is accepted (or the node is a leaf) the step's last token is the first v whose
 * running sum of p (vocabulary order) exceeds u_draw * sum_v p. Every emitted token then follows
 * the target's distribution at its position.
 *
 *   logits, draft_logits  dev [B,Nmax,V] fp32 with the same row_stride (>= V); row (b,i) of
 *                draft_logits is the distribution node i's children were drawn from. NaN
 *                entries carry no mass; a row of logits with +infinity has none at all (token 0).
 *   draft_tokens, parent, n_nodes, temperature, uniforms, path, path_len, tokens, n_tokens:
 *                as for fspad_tree_accept_sample (tokens outside [0,V) are never accepted)
 *   workspace    dev, 16-byte aligned, >= fspad_tree_accept_sample_draft_workspace_bytes(B,Nmax,V)
 *                (3 V fp64 entries per sequence and the chunk statistics of both logit arrays); two
 *                calls that may overlap need different ones
 * All arithmetic that takes a decision is fp64. With at most 256 sequences and a vocabulary of at
 * most 8192 * min(64, 256 / B) entries (the quotient rounded down: 524288 up to 4 sequences, 8192
 * from 129 on) and at least about 8 + 2 Nmax / 3, a sequence is walked by up to 64 workgroups that
 * keep their shares of the node's two rows in registers and exchange their sums after every
 * rejection; if some of them cannot run (other streams hold the compute units) those that can take
 * all shares, with the same result, after a wait of about the time that this takes them. Other calls
 * take one workgroup per sequence. Either way the cost is a few passes over the two rows of every
 * node on the accepted path (not over all B*Nmax rows).
 * Error reporting on the device: path_len[b] = n_tokens[b] = -1 says that the workgroups of
 * sequence b, all of them running, stopped waiting for one another after about a million polls; the other
 * outputs of that sequence are then undefined. It does not happen on a working device: nobody waits for a
 * workgroup that has not started.
 */
size_t fspad_tree_accept_sample_draft_workspace_bytes(int32_t B, int32_t Nmax, int32_t V);
fspad_status fspad_tree_accept_sample_draft(int32_t B, int32_t Nmax, int32_t V,
                                            const float* logits, const float* draft_logits, int64_t row_stride,
                                            const int32_t* draft_tokens, const int32_t* parent,
                                            const int32_t* n_nodes,
                                            float temperature, const float* uniforms,
                                            int32_t* path, int32_t* path_len,
                                            int32_t* tokens, int32_t* n_tokens,
                                            void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Greedy acceptance straight from the target's last hidden states, fused with the LM head
 * (Methodology, "LM Head": the final linear map from features to the vocabulary distribution;
 * Preliminaries, validation phase; Experiments "Settings": temperature 0). The [B*Nmax, V]
 * logits are never written to memory:
 *
 *   logits[b,i,v] = sum_k hidden[b,i,k] * lm_head[v,k]     bf16 inputs, exact products, fp32 sums
 *   target[b,i]   = the v with the largest logit (lowest v among equals; NaN never wins; a row
 *                   with nothing above -infinity takes token 0)
 *   then the walk of fspad_tree_accept_greedy with target[] in place of the row argmaxes.
 *
 *   hidden       dev [B,Nmax,hidden_dim] bf16, contiguous, 16-byte aligned (rows of unused tree
 *                slots are read but never used)
 *   lm_head      dev [V,hidden_dim] bf16, contiguous, 16-byte aligned (the weight matrix as the
 *                models store it: one row per token)
 *   flags        0, or FSPAD_WEIGHTS_PACKED (defined below): lm_head went through
 *                fspad_pack_weight(V, hidden_dim, ...) and is in tile order (same results)
 *   hidden_dim   multiple of 256, 256..65536
 *   draft_tokens, parent, n_nodes, path, path_len, tokens, n_tokens: as for fspad_tree_accept_greedy
 *   node_target  dev [B,Nmax] i32 out, may be NULL: target[b,i] (-1 in unused slots)
 *   node_top     dev [B,Nmax] f32 out, may be NULL: the winning logit (-infinity in unused slots)
 *   workspace    dev, 16-byte aligned, >= fspad_tree_accept_lm_head_workspace_bytes(B,Nmax,V)
 * The sums are accumulated in fp32 by the matrix cores in an order of the library's choosing: a
 * target token is only defined bit-for-bit where the winning logit leads the runner-up by more
 * than the fp32 accumulation error (about 1e-6 of sum_k |hidden*lm_head|); the tests require that.
 * Identical weight rows give identical logits (and the lower token wins) only inside one aligned
 * group of 128 tokens: each group sums over k starting from a different offset. Results are
 * the same from run to run.
 * More than 256 rows (B*Nmax) are processed in equal groups of at most 256 that each stream the
 * weights again.
 * Errors as for fspad_tree_accept_greedy; never synchronises, allocates nothing.
 */
size_t fspad_tree_accept_lm_head_workspace_bytes(int32_t B, int32_t Nmax, int32_t V);
fspad_status fspad_tree_accept_greedy_lm_head(int32_t B, int32_t Nmax, int32_t V, int32_t hidden_dim,
                                              const void* hidden, const void* lm_head, int32_t flags,
                                              const int32_t* draft_tokens, const int32_t* parent,
                                              const int32_t* n_nodes,
                                              int32_t* path, int32_t* path_len,
                                              int32_t* tokens, int32_t* n_tokens,
                                              int32_t* node_target, float* node_top,
                                              void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Tree rejection sampling straight from the target's last hidden states, fused with the LM head
 * (Methodology, "LM Head"; Preliminaries, validation phase; Experiments "Settings": temperature 1,
 * acceptance not relaxed). The walk of fspad_tree_accept_sample over
 *
 *   logits[b,i,v] = sum_k hidden[b,i,k] * lm_head[v,k]     bf16 inputs, exact products, fp32 sums
 *
 * without the [B*Nmax, V] logits ever being written: the GEMM leaves, per row and group of 128
 * tokens, the maximum and the sum of exp((l - max)/T), and sets aside the logit of every node's
 * own token under its parent's row; the last token is drawn by locating the group that holds the
 * crossing of u_bonus * Z and recomputing that group's 128 logits.
 *
 * Arguments as for fspad_tree_accept_greedy_lm_head (without node_target / node_top) plus
 * temperature and uniforms as for fspad_tree_accept_sample; same workspace size.
 * The exponentials are evaluated in fp32 on fp32 sums of the library's own order (the recomputed
 * group is summed in yet another order), the sums in fp64: a decision (an accept test, the
 * crossing of the last draw) is only defined where its relative margin is above about 1e-5; the
 * tests compare sequences whose smallest margin exceeds 1e-4.
 * Errors as for fspad_tree_accept_sample; never synchronises, allocates nothing.
 */
fspad_status fspad_tree_accept_sample_lm_head(int32_t B, int32_t Nmax, int32_t V, int32_t hidden_dim,
                                              const void* hidden, const void* lm_head, int32_t flags,
                                              const int32_t* draft_tokens, const int32_t* parent,
                                              const int32_t* n_nodes,
                                              float temperature, const float* uniforms,
                                              int32_t* path, int32_t* path_len,
                                              int32_t* tokens, int32_t* n_tokens,
                                              void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Commit of the accepted path to the KV cache. The paper leaves this step implied
 * (Preliminaries: the tokens that pass validation extend the sequence from which the
 * next draft phase starts): the keys and values the verification forward computed for
 * the accepted nodes are appended to the cache in path order, so that the next
 * cycle's prefix holds them and its root is the bonus token.
 *
 *   for j < path_len[b], every kv head g:
 *       k_cache[b,g,kv_len[b]+j,:] = k_tree[b,path[b,j],g,:]      (v likewise)
 *   kv_len_out[b] = kv_len[b] + path_len[b]
 *
 *   desc     batch, n_nodes_max, n_kv_heads, head_dim, io_dtype and the cache strides are
 *            read; the other fields are ignored
 *   k_tree, v_tree   dev [B,Nmax,Hkv,D] io_dtype (this layer's tree keys / values)
 *   k_cache, v_cache dev strided, written; every (b,g) row must hold cache_capacity tokens
 *   cache_capacity   tokens per (b,g) row; kv_len[b] + Nmax <= cache_capacity is required
 *            (FSPAD_ERR_SHAPE otherwise: the path length is only known on the device)
 *   kv_len   HOST [B] prefix lengths before the commit (the ones the attention call took)
 *   path, path_len   dev [B,Nmax], [B]: outputs of an acceptance call. Entries outside
 *            [0,Nmax) and lengths outside [0,Nmax] are not followed (nothing is moved for them)
 *   kv_len_out       dev [B] i32 out, may be NULL
 * Cache positions other than kv_len[b] .. kv_len[b]+path_len[b]-1 are left untouched.
 */
fspad_status fspad_kv_commit(const fspad_attn_desc* desc, const void* k_tree, const void* v_tree,
                             void* k_cache, void* v_cache, int32_t cache_capacity,
                             const int32_t* kv_len, const int32_t* path, const int32_t* path_len,
                             int32_t* kv_len_out, void* hip_stream);

/*
 * Paged 4-bit cache (no passage of the paper: a storage format for serving long prompts, 17/64 of the bf16 cache's bytes).
 * Four calls: fspad_page_map keeps block tables, slots and lengths on the device, fspad_kv_store_paged puts keys and values
 * into pages, fspad_kv_load_paged takes them out, fspad_tree_attn_paged is the tree attention over them. Lengths and node
 * counts are read from the DEVICE, so that a captured step replays with whatever the step before it accepted.
 *
 * Values. A block is 32 neighbouring channels of one token and kv head. An element is 4 bits, a sign on top of a code for 0,
 * 1/2, 1, 3/2, 2, 3, 4, 6; a block's scale is 2^(s-127) for a byte s, and s = 255 makes all of the block NaN (the FP4 format of
 * the OCP microscaling specification). The store rounds a block whose largest magnitude is a so:
 *   s    = the smallest of 2..252 with a <= 7 * 2^(s-127)  (252 where that is too small too; 255 if any value is NaN or infinite)
 *   code = the element nearest to x / 2^(s-127), ties to the even code, at most 6
 * which is off by at most 2^(s-127) < a * 2/7 for a from 2^-123 to 7 * 2^125. What reads a cache takes s from 2 to 252, and 255;
 * other scales are not specified.
 *
 * Pages. A page holds page_tokens tokens (16, 32, 64, 128 or 256) of all kv heads of one layer, one head after the other, of each
 * (P = page_tokens, D = head_dim), in bytes:
 *   K codes  [P][D/2]
 *   V codes  [P*D/512][16][512/D][D/32]  groups of 512/D tokens; of a group, 16 runs of D/16 channels; of a run, token after token
 *   K scales [D/32][P]
 *   V scales [D/32][P]
 * with the even channel of a byte in its low half: fspad_kv_page_bytes = Hkv * P * D * 17/16 in all. Pages start page_stride
 * bytes apart (a multiple of 16 below 2^32, at least the page's bytes: pools of several layers may be interleaved) in a pool of n_pages;
 * n_pages * page_tokens <= 2^31 - 1. Token t of page p is slot p * page_tokens + t.
 */
typedef struct {
  int32_t batch;          /* B >= 1 (attention only, <= 1024) */
  int32_t n_nodes_max;    /* Nmax, 1..64 (attention only) */
  int32_t n_q_heads;      /* Hq (attention only) */
  int32_t n_kv_heads;     /* Hkv, divides Hq */
  int32_t head_dim;       /* D: 64 or 128 */
  int32_t io_dtype;       /* FSPAD_BF16: q, k_tree, v_tree, and the rows that are stored and loaded */
  int32_t out_dtype;      /* FSPAD_BF16 or FSPAD_F32 (attention only) */
  float softmax_scale;    /* 0 => 1/sqrt(D); else of any sign, 2^-125 .. 2^127 in magnitude (attention only) */
  int32_t page_tokens;    /* P: 16, 32, 64, 128 or 256 */
  int32_t n_pages;        /* pages of the pool, >= 1 */
  int64_t page_stride;    /* bytes from page to page, below 2^32 */
  int32_t table_width;    /* entries of a block table's row, >= 1 (attention only) */
  int32_t max_kv_len;     /* no sequence is longer, 0..table_width * P (attention only): the launch is laid out for it */
  int64_t table_stride;   /* entries from row to row of the block table, >= table_width (attention only) */
  int32_t workgroups;     /* tuning of the attention: 0 = the built-in choice; 1..4096 cuts the keys into about that many pieces
                             beside one for each (sequence, kv head, group of query rows). Results do not depend on it beyond
                             fp32 rounding of the join; the workspace's size does */
  int32_t reserved;       /* 0; not looked at */
} fspad_paged_desc;

/* Bytes of one page, 0 for an unsupported shape. */
size_t fspad_kv_page_bytes(int32_t n_kv_heads, int32_t head_dim, int32_t page_tokens);

/*
 * Page map: what a step changes of the block tables, in sequence order and by one rule on the device. Sequence b holds
 * ceil(kv_len[b] / P) pages, the first entries of its row of the table. The stack free_pages[0 .. n_free-1] names the pages
 * that nobody holds.
 *   n_new[b] < 0   b ends: its pages go onto the stack (first those of the first sequence that ends, each row from its first
 *                  entry on), kv_len_out[b] = 0, granted[b] = 0. Its row of the table keeps its entries.
 *   n_new[b] >= 0  b grows by n_new[b] tokens. The pages it lacks for kv_len[b] + n_new[b] come off the top of the stack (which has
 *                  the pages of the sequences that end by then), sequence after sequence, into its row: kv_len_out[b] = kv_len[b] +
 *                  n_new[b], granted[b] = 1.
 * A sequence is refused, kv_len_out[b] = kv_len[b] and granted[b] = 0 with its row as it was, if it would not fit its row, if
 * n_new[b] > max_new or its rows would end past n_slots, or if it needs pages and those of all sequences up to it (refused for
 * lack of pages or not, but not those refused for another reason) are more than the stack has.
 *
 * Slots of the new tokens (-1: none), for fspad_kv_store_paged:
 *   max_new > 0, no path   slots [B,max_new]: token j < n_new[b] of a granted sequence has slots[b,j]
 *   max_new > 0, path      slots [B,max_new] by tree node: place j < n_new[b] of the path has slots[b,path[b,j]] (path and path_len
 *                          of an acceptance call as path and n_new, Nmax as max_new, at most 64; path entries outside [0,max_new) are
 *                          not followed, of a node that is named twice the first place counts). The store then takes k_tree and v_tree as they are.
 *   max_new = 0            slots [n_slots]: the sequences' rows one behind the other, max(n_new[b], 0) each whether granted or
 *                          not; the rest of the array is -1. n_slots <= 2^22
 *
 *   B           1..2048;  table_width * P <= 2^31 - 1, B * table_width and B * max_new <= 2^30
 *   kv_len, n_new, path    dev [B], [B], [B,max_new] i32 (negative lengths count as 0)
 *   block_table dev [B] rows of table_width i32, table_stride entries apart: written where a sequence gets pages
 *   free_pages  dev [n_pages] i32, in and out;  n_free dev [1] i32 (taken as 0..n_pages)
 *   slots       dev out, may be NULL if it has no entries
 *   kv_len_out, n_free_out, granted   dev [B], [1], [B] i32 out; kv_len_out may be kv_len and n_free_out n_free
 * The pages of a sequence that ends must be its own, and no page may stand in two rows that end or on the stack twice. A table
 * entry of a held page outside [0,n_pages) gives no slot. No workspace; allocates nothing, never synchronises.
 */
fspad_status fspad_page_map(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride,
                            const int32_t* kv_len, const int32_t* n_new, const int32_t* path, int32_t max_new,
                            int32_t n_slots, int32_t* block_table, int32_t* free_pages, const int32_t* n_free,
                            int32_t* slots, int32_t* kv_len_out, int32_t* n_free_out, int32_t* granted,
                            void* hip_stream);

/*
 * Keys and values of `rows` tokens into the slots they are given, rounded as above (a prompt's tokens, or the tree's nodes with
 * the slots that fspad_page_map made of the accepted path).
 *   k, v      dev bf16, 16-byte aligned: channel c of head g of row r at r*row_stride + g*head_stride + c (elements, multiples
 *             of 8, >= 0, the same for both)
 *   slots     dev [rows] i32; a row whose slot is outside [0, n_pages * page_tokens) goes nowhere. No slot may be
 *             given to two rows of a call (what it holds then is not specified)
 *   pages     dev, 16-byte aligned; bytes of other slots stay as they are
 * rows = 0 does nothing (no pointer is looked at). Reads n_kv_heads, head_dim, io_dtype, page_tokens, n_pages and page_stride of
 * the descriptor, as fspad_kv_load_paged does.
 */
fspad_status fspad_kv_store_paged(const fspad_paged_desc* desc, int32_t rows, const void* k, const void* v,
                                  int64_t row_stride, int64_t head_stride, const int32_t* slots,
                                  void* pages, void* hip_stream);

/*
 * The reverse: row r of k and v (bf16, exact) is what slots[r] holds, zeros where the slot is outside [0, n_pages * page_tokens).
 * Strides as for the store, both at least head_dim, and no two (row, head) pairs may share elements: the rows may be
 * those of a cache that fspad_tree_attn reads. A slot may be given to several rows.
 */
fspad_status fspad_kv_load_paged(const fspad_paged_desc* desc, int32_t rows, const int32_t* slots, const void* pages,
                                 void* k, void* v, int64_t row_stride, int64_t head_stride, void* hip_stream);

/*
 * Tree-masked attention over the pages: fspad_tree_attn with the prefix read through a block table from the 4-bit pool, and
 * lengths and node counts from the device. One node (Nmax = 1, mask word 1) is plain decoding.
 *
 *   out[b,i,h,:] = sum_j softmax_j( scale * q[b,i,h,:] . K_j ) * V_j
 * where j runs over the prefix positions t < kv_len[b] of kv head g = h/(Hq/Hkv) (slot
 * block_table[b, t / P] * P + t % P) and then over the tree tokens t < n_nodes[b] whose bit t is set in anc_mask[b,i].
 *
 *   q, k_tree, v_tree   dev bf16 [B,Nmax,Hq,D], [B,Nmax,Hkv,D], 16-byte aligned, contiguous
 *   pages       dev, 16-byte aligned
 *   block_table dev [B] rows of table_width i32, table_stride entries apart. Positions on an entry outside [0,n_pages) are
 *               left out, as if they were masked; entries past ceil(kv_len[b] / P) are not looked at
 *   kv_len      DEV [B] i32, taken as 0 .. max_kv_len;  n_nodes DEV [B] i32, taken as 0 .. Nmax
 *   max_kv_len  of the descriptor: all that is known of the lengths when the call is launched. Results do not depend on it beyond
 *               their last bits, as long as it holds. Short calls take longer under one far above the lengths, which starts the kernels
 *               of long sequences and a second launch that then has nothing to join: one token, 511 tokens on 8 kv heads, 9.1 us under
 *               its own length and 11.6 under 8192 or more; a tree of 26 nodes, 2048 tokens, 16.5 and 21.1; 64 single tokens of up to
 *               4000, D = 64, 19.1 and 21.6. Calls that are laid out for cut keys either way take the same (4 trees of 60 nodes, 4096
 *               tokens: 46). A table no wider than the longest sequence that is served is bound enough
 *   anc_mask    dev [B,Nmax] u64 as for fspad_tree_attn
 *   out         dev [B,Nmax,Hq,D] out_dtype, 16-byte aligned. Rows i >= n_nodes[b], and rows that see nothing, are zeros
 *   workspace   dev, 16-byte aligned, >= fspad_tree_attn_paged_workspace_bytes(desc) (0: unsupported shape); contents ignored on entry,
 *               undefined on exit; two calls that may overlap in time need different ones
 * What a row does not see has no part in it, NaN and infinity included. Cached keys enter the products as they are stored, against
 * the sum of two fp8 rows that holds a query (exact down to 2^-14 of the row's largest value, off by 2^-22 of that below); products with tree keys
 * and with values are of bf16 values (cached ones are exact in bf16, probabilities are rounded to bf16). Sums are fp32, the
 * sum of the probabilities over the rounded ones; a score times scale * log2(e) has to be a finite fp32 number. The same inputs
 * give the same bits from run to run; a sequence's results may differ in their last bits with the batch it is in, which decides how
 * its keys are cut.
 */
/* How a call is dealt out decides its size, which a smaller batch or bound may well raise: a buffer for several descriptors has the largest of their sizes. */
size_t fspad_tree_attn_paged_workspace_bytes(const fspad_paged_desc* desc);

fspad_status fspad_tree_attn_paged(const fspad_paged_desc* desc,
                                   const void* q, const void* k_tree, const void* v_tree,
                                   const void* pages, const int32_t* block_table,
                                   const int32_t* kv_len, const int32_t* n_nodes,
                                   const uint64_t* anc_mask, void* out,
                                   void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Paged 8-bit cache (no passage of the paper: a storage format between the bf16 cache, of which it takes half, and the 4-bit one; values are off by
 * 1/16 at most where they are not small beside the largest of their block). Block tables, slots, lengths and the stack of free pages are those of the 4-bit cache: fspad_page_map keeps
 * them, and descriptors are the same (page_tokens: 32, 64, 128 or 256).
 *
 * Values. A block is 32 neighbouring tokens of a page (from a multiple of 32 on) and one kv head; K and V have scales of their own. An element is
 * an 8-bit float: a sign, 4 bits of exponent, 3 of mantissa, the smallest 2^-9, the largest 448, all bits below the sign NaN (E4M3 of the OCP
 * formats). A block's scale is 2^(s-127) for a byte s. What a store does to a block that some of its rows go to, whose largest finite magnitude
 * is a:
 *   t    = the smallest of 10..246 with a <= 448 * 2^(t-127) (246 where that is too small too)
 *   s    = t if one of the rows goes to the block's first token: the call begins the block (what it holds of tokens that are not in the call
 *          is not specified then). Else the larger of t and the s that the block has; where it grows, the tokens that the block held are
 *          rounded again, value / 2^(s-127), as below
 *   code = the element nearest to x / 2^(s-127), ties to the even one, at most 448; NaN and infinity become NaN
 * so that a value up to 7 * 2^125 is off by at most 1/16 of it from 2^(s-133) on, and by at most 2^(s-137) below that, when it is stored (what is below 2^-19 of
 * its block's largest becomes 0). A scale grows by powers of two: rounding again changes only values that come to lie below 2^(s-133) of
 * the new s, and those by 2^(s-137) at most. All growths' errors add up to less than twice the last one's: a value that a block holds under s is
 * off by less than 1/16 of what was stored plus 2^(s-136), however often the scale has grown. What reads a cache takes s from 10 to
 * 246; other scales are not specified.
 *
 * Pages. A page holds page_tokens tokens of all kv heads of one layer, one head after the other, of each (P = page_tokens, D = head_dim,
 * E = D / 32), in bytes:
 *   K codes  [P/32][D/16][32][16]     token t, channel c at [t/32][c/16][t%32][c%16]
 *   V codes  [P/32][E][2][32][16]     token t, channel c at [t/32][c%E][t%32/16][c/E][t%16]
 *   K scales [8]                      of block t/32, the first P/32 of them used
 *   V scales [8]
 * fspad_kv_page_bytes_byte = Hkv * (2 * P * D + 16) in all. page_stride and n_pages as for the 4-bit cache.
 */

/* Bytes of one page, 0 for an unsupported shape. */
size_t fspad_kv_page_bytes_byte(int32_t n_kv_heads, int32_t head_dim, int32_t page_tokens);

/*
 * Keys and values of `rows` tokens into the slots they are given, as fspad_kv_store_paged, rounded as above.
 *   k, v, slots, row_stride, head_stride   as there. The rows of a block may stand anywhere in the call. No slot may be given to two rows of a
 *             call (what its block holds then, of its other tokens too, is not specified)
 *   rows      0..1048560; 0 does nothing (no pointer is looked at)
 *   pages     dev, 16-byte aligned. Tokens of other blocks stay as they are; no other call may use a block that this one stores to meanwhile
 *   workspace dev, 16-byte aligned, >= fspad_kv_store_paged_byte_workspace_bytes(desc, rows): 0 up to 2048 rows (may be NULL then), 4 bytes a
 *             slot of the pool for more; contents ignored on entry, undefined on exit; two calls that may overlap in time need different ones
 * Reads n_kv_heads, head_dim, io_dtype, page_tokens, n_pages and page_stride of the descriptor, as fspad_kv_load_paged_byte does.
 */
size_t fspad_kv_store_paged_byte_workspace_bytes(const fspad_paged_desc* desc, int32_t rows);

fspad_status fspad_kv_store_paged_byte(const fspad_paged_desc* desc, int32_t rows, const void* k, const void* v,
                                      int64_t row_stride, int64_t head_stride, const int32_t* slots, void* pages,
                                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* The reverse, as fspad_kv_load_paged: row r of k and v (bf16, exact) is what slots[r] holds, zeros where the slot is outside the pool. */
fspad_status fspad_kv_load_paged_byte(const fspad_paged_desc* desc, int32_t rows, const int32_t* slots, const void* pages,
                                     void* k, void* v, int64_t row_stride, int64_t head_stride, void* hip_stream);

/*
 * fspad_tree_attn_paged over 8-bit pages: arguments, masks, lengths, outputs, workspace and errors are those of that call. Products with cached
 * keys and values, and the roundings of queries, weights and sums, are those that stand there too (cached values are exact in bf16).
 * max_kv_len decides more here: also how rows are dealt out, so that batches of short sequences take longer under a bound far above them. 256 single tokens of
 * 100 tokens, 32 heads on 8, 17.9 us under their own length and 40.4 under 8192; 64 trees of 60 nodes, 500 tokens, 61 and 67; 2000 tokens, 168 and 174; one
 * token, 511 tokens, 8.6 and 11.1; 4 trees on 52 heads, 4096 tokens, 45 either way.
 */
/* As fspad_tree_attn_paged_workspace_bytes: a smaller batch or bound may take more (60 nodes on 32 heads, 8 of keys, D = 128, under 2500: 64 sequences 8 KB, 11 29 MB, 4 2 KB). */
size_t fspad_tree_attn_paged_byte_workspace_bytes(const fspad_paged_desc* desc);

fspad_status fspad_tree_attn_paged_byte(const fspad_paged_desc* desc,
                                       const void* q, const void* k_tree, const void* v_tree,
                                       const void* pages, const int32_t* block_table,
                                       const int32_t* kv_len, const int32_t* n_nodes,
                                       const uint64_t* anc_mask, void* out,
                                       void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Shared pages (no passage of the paper: several continuations of one prompt hold its pages once). Beside the block tables, lengths and stack of
 * fspad_page_map there is an array shared [n_pages] i32: how many sequences hold a page beside the first, 0 for pages that one holds or none
 * (counts below zero are taken as 0). It starts as zeros; fspad_page_map neither reads nor changes it, since pages that it gives are new. Sequences of whose pages
 * any may be shared end by fspad_page_release, not by n_new < 0. Only full pages are ever shared, so that growth writes to pages of a
 * sequence's own. The calls are about block tables: they serve the 4-bit and the 8-bit cache alike, all layers at once.
 *
 *   B           rows of the block table, 1..2048;  page_tokens 16, 32, 64, 128 or 256;  n_pages 1..2^19 (n_pages and table_width times page_tokens <= 2^31 - 1)
 *   block_table dev [B] rows of table_width i32, table_stride entries apart (B * table_width <= 2^30)
 *   kv_len      dev [B] i32 (negative lengths count as 0); sequence b holds the first ceil(kv_len[b] / P) entries of its row
 *   free_pages  dev [n_pages] i32, n_free dev [1] i32 (taken as 0..n_pages): the stack of fspad_page_map. Its first n_free entries are pages, none twice and
 *               none that is held (others would not be read or written past, but a fork would be granted without its page, and a compaction
 *               would leave a held page among those that it calls free); what lies behind them is not looked at
 *   outputs     kv_len_out may be kv_len, n_free_out n_free, shared_out shared; else they do not overlap with inputs
 * Entries of tables outside [0,n_pages) count for no page. None of the calls allocates or synchronises; results are the same from run to run.
 */

/*
 * Forks: for f < n_forks in order, row dst[f] becomes the first n_tokens[f] tokens of row src[f] (all lengths before the call).
 *   full pages   the first n_tokens[f] / P entries of row src[f], which both rows hold from now on: each page's count goes up by one for each fork
 *   the rest     n_tokens[f] % P tokens, if there are any, go to a page off the top of the stack: copy_src[f] = the page in row src[f], copy_dst[f] = the new
 *                one, for fspad_page_copy in every layer's pool, before the row is read or stored to
 * granted[f] = 1 and kv_len_out[dst[f]] = n_tokens[f]; lengths of other rows are those before the call. copy_src[f] = copy_dst[f] = -1 where nothing is to be copied.
 * A fork is refused, granted[f] = 0 with nothing changed for it, if src[f] or dst[f] is outside [0,B), or they are the same, if row dst[f] has tokens or a fork
 * before f in the call names it too (refused or not), if n_tokens[f] is below zero, above kv_len[src[f]], or more than a row holds, or if it needs a page and there
 * are as many forks before it that need one (refused for lack of pages or not, but not those refused for another reason) as the stack has.
 *   n_forks     0..2048;  src, dst dev [n_forks] i32;  n_tokens dev [n_forks] i32, NULL: all tokens of src
 *   copy_src, copy_dst, granted   dev [n_forks] i32 out;  n_free_out dev [1] out;  shared_out dev [n_pages] out
 * No workspace. The stack itself is not written to.
 */
fspad_status fspad_page_fork(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride, int32_t n_forks,
                             const int32_t* src, const int32_t* dst, const int32_t* n_tokens, const int32_t* kv_len,
                             int32_t* block_table, const int32_t* free_pages, const int32_t* n_free, const int32_t* shared,
                             int32_t* copy_src, int32_t* copy_dst, int32_t* kv_len_out, int32_t* n_free_out,
                             int32_t* shared_out, int32_t* granted, void* hip_stream);

/*
 * Ends: sequences b with ended[b] != 0 give up the pages they hold, kv_len_out[b] = 0 (others keep their lengths). A page that more of them hold than its
 * count says is held by nobody then: it goes onto the stack, with a count of 0, the pages of a call in ascending order. Counts of others go down by the
 * sequences that held them. Rows of the table keep their entries.
 *   ended       dev [B] i32;  free_pages is written behind the first n_free entries
 *   workspace   dev, 16-byte aligned, >= fspad_page_release_workspace_bytes(B, n_pages, table_width) (0 for small calls: may be NULL then);
 *               contents ignored on entry, undefined on exit; two calls that may overlap in time need different ones
 */
size_t fspad_page_release_workspace_bytes(int32_t B, int32_t n_pages, int32_t table_width);

fspad_status fspad_page_release(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride,
                                const int32_t* ended, const int32_t* kv_len, const int32_t* block_table,
                                int32_t* free_pages, const int32_t* n_free, const int32_t* shared,
                                int32_t* kv_len_out, int32_t* n_free_out, int32_t* shared_out,
                                void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Compaction: what is held moves to the first keep = n_pages - n_free pages of the pool, so that the rest of it can be given back (or a larger pool begin).
 * Pages from keep on that are not on the stack go to the pages before keep that are, both in ascending order. copy_src[i], copy_dst[i] are the moves, in this order, -1
 * behind the last one: for fspad_page_copy in every layer's pool, before it is read or stored to. Held entries of the tables and counts follow their
 * pages; the stack is n_pages - 1, n_pages - 2, .. keep, its height what it was, -1 behind.
 *   copy_src, copy_dst   dev [n_pages / 2] i32 out (may be NULL if n_pages is 1)
 *   block_table_out      dev [B] rows of table_width i32, out_stride entries apart: may be block_table (with its stride); else entries that are not held are copied
 *   free_out, shared_out dev [n_pages] i32 out: may be free_pages and shared
 * No workspace.
 */
fspad_status fspad_page_compact(int32_t B, int32_t page_tokens, int32_t n_pages, int32_t table_width, int64_t table_stride, int64_t out_stride,
                                const int32_t* kv_len, const int32_t* block_table, const int32_t* free_pages,
                                const int32_t* n_free, const int32_t* shared, int32_t* copy_src, int32_t* copy_dst,
                                int32_t* block_table_out, int32_t* free_out, int32_t* shared_out,
                                void* hip_stream);

/*
 * Copies: page copy_dst[i] of a pool becomes what page copy_src[i] is, for i < n_copies where both lie in [0,n_pages) (other pairs are passed over). No
 * page that is written may stand in another pair of the call.
 *   pages       dev, 16-byte aligned; n_pages >= 1 pages of page_bytes, page_stride bytes apart (both multiples of 16, page_bytes <= 2^31 - 1, page_stride below 2^32):
 *               of interleaved pools of several layers, page_bytes may be all of them
 *   n_copies    >= 0; copy_src, copy_dst dev [n_copies] i32 (0: no pointer is looked at)
 */
fspad_status fspad_page_copy(void* pages, int32_t n_pages, int64_t page_stride, int64_t page_bytes, int32_t n_copies,
                             const int32_t* copy_src, const int32_t* copy_dst, void* hip_stream);

/*
 * Tile order for the weights of the skinny projections (an option of fspad_feature_sampler,
 * fspad_draft_layer and the LM-head acceptance; no passage of the paper: it is a storage format). A row-major [n_rows][k] bf16
 * matrix is cut into tiles of 16 rows x 32 columns, stored tile row by tile row, within a tile row
 * along k; the 1 KB of a tile holds, at byte 16 * (n + 16 g), the eight values
 * w[16 t + n][32 s + 8 g .. + 7] (t: tile row, s: tile along k, n in 0..15, g in 0..3). Rows past
 * n_rows in the last tile row are zeros. A wavefront then streams contiguous kilobytes instead of
 * four rows x 256 bytes per request, at the same rate on gfx950 (Feature Sampler at 4096 / 11008: 55 and
 * 54 us); results are bit-identical to those from row-major weights.
 *
 *   n_rows >= 1; k a multiple of 32; w dev [n_rows][k] bf16; packed dev,
 *   fspad_packed_weight_bytes(n_rows, k) = ceil(n_rows / 16) * 16 * k * 2 bytes (0 = bad shape);
 *   both 16-byte aligned and not overlapping. Done once per weight matrix, ahead of time.
 */
#define FSPAD_SAMPLER_RESIDUAL 1 /* fspad_feature_sampler flags: add the residual f */
#define FSPAD_WEIGHTS_PACKED 2   /* flags of fspad_feature_sampler and of the LM-head acceptance: the weight
                                    matrices are in tile order */
size_t fspad_packed_weight_bytes(int32_t n_rows, int32_t k);
fspad_status fspad_pack_weight(int32_t n_rows, int32_t k, const void* w, void* packed, void* hip_stream);

/*
 * Feature Sampler of the draft model (Methodology, "Feature Sampling": three projectors and a
 * sampling operation in the intermediate space). The Up Projector lifts the feature f, the Gate
 * Projector lifts the token embedding e, the lifted embedding goes through SiLU and multiplies the
 * lifted feature element by element, the Down Projector maps the product back to the hidden size,
 * and the residual connection of the feature path is added:
 *
 *   eta[r,:] = W_down (SiLU(W_gate e[r,:]) * (W_up f[r,:])) + f[r,:]
 *   (without "+ f" unless flags has FSPAD_SAMPLER_RESIDUAL)
 *
 *   rows              1..128: the tokens of one draft step (sequences x expanded nodes)
 *   hidden_dim, intermediate_dim   multiples of 256
 *   f, e              dev [rows,hidden_dim] bf16
 *   w_up, w_gate      dev [intermediate_dim,hidden_dim] bf16 (one row per intermediate channel)
 *   w_down            dev [hidden_dim,intermediate_dim] bf16
 *   flags             FSPAD_SAMPLER_RESIDUAL | FSPAD_WEIGHTS_PACKED (the three weight matrices are then
 *                     each in the tile order of fspad_pack_weight); other bits are an error
 *   eta               dev [rows,hidden_dim] bf16 out
 *   workspace         dev, 16-byte aligned, >= fspad_feature_sampler_workspace_bytes(...)
 * All pointers 16-byte aligned, all arrays contiguous. bf16 products are exact, sums are fp32 (in a
 * fixed order: the result is the same from run to run); the gated product is rounded to bf16 before
 * the Down Projector, eta once more at the end. Never synchronises, allocates nothing.
 */
size_t fspad_feature_sampler_workspace_bytes(int32_t rows, int32_t hidden_dim, int32_t intermediate_dim);
fspad_status fspad_feature_sampler(int32_t rows, int32_t hidden_dim, int32_t intermediate_dim,
                                   const void* f, const void* e,
                                   const void* w_up, const void* w_gate, const void* w_down,
                                   int32_t flags, void* eta,
                                   void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The draft model: one transformer decoder layer over the draft's token tree (Methodology, first
 * paragraph: the draft model is a Transformer Decoder Layer that maps the sequence eta to the next
 * features; "Partial Alignment Distillation": the output dimension of its MLP is doubled and both
 * halves share one residual connection, which gives the two features f~ (mapped to tokens by the
 * LM head) and f (the Feature Sampler's input of the next step)).
 *
 *   x        = eta
 *   q, k, v  = split(W_qkv rmsnorm(x; gain_attn)); q and k rotary-encoded at `positions`
 *   h        = x + W_o attn          attn = fspad_tree_attn(q, k, v | draft cache, anc_mask)
 *   m        = W_down (SiLU(W_gate rmsnorm(h; gain_mlp)) * (W_up rmsnorm(h; gain_mlp)))
 *   f~       = h + m[:, :Hd]         f = h + m[:, Hd:]
 *
 * The layer is LLaMA's: rmsnorm(x; g) = x / sqrt(mean(x^2) + rms_eps) * g; the rotary encoding
 * turns the pair (entry i, entry i + D/2) of every query and key head by
 * positions[b,n] * rope_theta^(-2i/D); no biases. The caller commits the accepted rows of k_tree /
 * v_tree to the draft's cache with fspad_kv_commit.
 *
 *   desc.attn   geometry of the draft's attention and of its cache as for fspad_tree_attn;
 *               io_dtype and out_dtype FSPAD_BF16; batch * n_nodes_max <= 128;
 *               n_q_heads * head_dim a multiple of 256
 *   hidden_dim, intermediate_dim  Hd, I: multiples of 256
 *   weights     dev bf16, row-major [out][in], 16-byte aligned: w_qkv [(Hq+2Hkv) D, Hd] (query,
 *               key, value rows in that order), w_o [Hd, Hq D], w_gate and w_up [I, Hd],
 *               w_down [2 Hd, I] (rows 0..Hd-1 produce f~, rows Hd.. produce f), gain_attn and
 *               gain_mlp [Hd]; with weights_packed = 1 the five matrices are each in the tile order
 *               of fspad_pack_weight (the gains stay as they are)
 *   eta         dev [B,Nmax,Hd] bf16
 *   positions   dev [B,Nmax] i32 (prefix length + depth of the node)
 *   k_cache, v_cache, kv_len (HOST), n_nodes (HOST), anc_mask: as for fspad_tree_attn
 *   k_tree, v_tree  dev [B,Nmax,Hkv,D] bf16 OUT: keys (rotary-encoded) and values of the nodes
 *   f_tilde, f  dev [B,Nmax,Hd] bf16 OUT; rows of unused tree slots hold unspecified values
 *   workspace   dev, 16-byte aligned, at least fspad_draft_layer_workspace_bytes(desc,
 *               max_b kv_len[b]) bytes (0 = unsupported shape); contents ignored on entry, undefined on
 *               exit; two calls that may overlap in time need different workspaces
 * Products of bf16 values are summed in fp32 in a fixed order; the activations between the
 * projections (normalised inputs, q / k / v, attention output, h, the gated product) are rounded to
 * bf16 once each, as a bf16 model stores them.
 */
typedef struct {
  fspad_attn_desc attn;
  int32_t hidden_dim;
  int32_t intermediate_dim;
  float rms_eps;     /* >= 0 */
  float rope_theta;  /* > 0, e.g. 10000 */
  int32_t weights_packed; /* 0: row-major weight matrices; 1: tile order */
} fspad_draft_layer_desc;

typedef struct {
  const void* w_qkv;
  const void* w_o;
  const void* w_gate;
  const void* w_up;
  const void* w_down;
  const void* gain_attn;
  const void* gain_mlp;
} fspad_draft_layer_weights;

size_t fspad_draft_layer_workspace_bytes(const fspad_draft_layer_desc* desc, int32_t max_kv_len);

fspad_status fspad_draft_layer(const fspad_draft_layer_desc* desc, const fspad_draft_layer_weights* weights,
                               const void* eta, const int32_t* positions,
                               const void* k_cache, const void* v_cache,
                               const int32_t* kv_len, const int32_t* n_nodes, const uint64_t* anc_mask,
                               void* k_tree, void* v_tree, void* f_tilde, void* f,
                               void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Top-k cut of a draft step's output (Preliminaries, last paragraph: the output of every draft
 * step is cut to its k most probable tokens, and the joint probabilities of the tree follow from
 * their probabilities). Per row:
 *
 *   tokens[r,0..k-1] = the k entries with the largest logit, best first (equal logits: lower
 *                      token first; NaN counts as -infinity; -0 == +0)
 *   logp[r,j]        = logits[r,tokens[r,j]] - log(sum_v exp(logits[r,v]))      (log-softmax)
 *
 *   rows        1..65535 (one per node expanded in this draft step, over all sequences)
 *   logits      dev [rows] rows of V fp32, row_stride elements apart (>= V); finite, -infinity
 *               or NaN (+infinity is not supported)
 *   k           1..min(V, FSPAD_MAX_TOPK)
 *   tokens      dev [rows,k] i32 out;  logp dev [rows,k] f32 out -- what fspad_tree_build takes as
 *               cand_token / cand_logp of the new candidates
 *   workspace   dev, 16-byte aligned, >= fspad_draft_topk_workspace_bytes(rows,V,k)
 * The sum is formed from fp32 exponentials accumulated in fp64 (logp agrees with an fp64
 * evaluation to about 1e-6); the tokens are exact. A row without a finite entry yields tokens
 * 0..k-1 and logp -infinity. V * k <= 2^24 is required. Never synchronises, allocates nothing.
 */
#define FSPAD_MAX_TOPK 16
size_t fspad_draft_topk_workspace_bytes(int32_t rows, int32_t V, int32_t k);
fspad_status fspad_draft_topk(int32_t rows, int32_t V, int32_t k, const float* logits, int64_t row_stride,
                              int32_t* tokens, float* logp,
                              void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Dynamic draft tree from its candidates (Preliminaries, last paragraph: the output of every
 * draft step is cut to its top-k, joint probabilities follow from the dependencies between the
 * tokens, and one more top-k over all tokens yields a valid tree of bounded size; the
 * paragraph before it: the tokens are then organised into a tree and the attention mask is
 * derived from it). This call covers everything after the per-step top-k: it accumulates the
 * joint scores, picks the tree, flattens it and emits the arrays the verification calls consume.
 *
 *   joint[0] = 0;  joint[c] = joint[cand_parent[c]] + cand_logp[c]    (one fp32 addition per edge)
 *   kept = root + the n_keep-1 non-root candidates with the highest joint (ties: lower index);
 *          a kept candidate whose parent is not kept is dropped with its descendants (cannot
 *          happen when all cand_logp <= 0)
 *   nodes = kept candidates in candidate order (parents precede children, siblings keep their
 *          order); parent / draft_tokens / anc_mask as every other call here expects them
 *
 *   cand_parent dev [B,M] i32: candidate index of the parent, < own index; [b,0] = -1 (root)
 *   cand_token  dev [B,M] i32
 *   cand_logp   dev [B,M] f32: conditional log-probability given the parent's path; [b,0] is
 *               ignored; NaN counts as -infinity
 *   n_cand      dev [B] i32, 1..M;  M <= FSPAD_MAX_CANDIDATES
 *   n_keep      nodes to keep, root included, 1..Nmax (Nmax <= 64)
 *   parent, draft_tokens, node_cand dev [B,Nmax] i32 out (-1 in unused slots); node_cand[b,i] is
 *               the candidate node i came from; n_nodes dev [B] i32 out; anc_mask dev [B,Nmax] u64 out
 * A parent index outside [0, own index) makes that candidate (and its descendants) unreachable:
 * it is never kept. No workspace.
 */
#define FSPAD_MAX_CANDIDATES 1024
fspad_status fspad_tree_build(int32_t B, int32_t M, int32_t Nmax, const int32_t* cand_parent,
                              const int32_t* cand_token, const float* cand_logp, const int32_t* n_cand,
                              int32_t n_keep, int32_t* parent, int32_t* draft_tokens, int32_t* n_nodes,
                              uint64_t* anc_mask, int32_t* node_cand, void* hip_stream);

/*
 * Host helpers for the tree (Preliminaries: tokens organised into a tree by
 * their dependencies, then the mask derived from the tree).
 *
 * fspad_tree_build_mask: mask_host[b,i] = bit i | mask_host[b,parent[b,i]] for
 *   i < n_nodes_host[b]; words of nodes >= n_nodes_host[b] are 0. All arrays on the
 *   host, [B,Nmax] / [B]. Returns FSPAD_ERR_TREE for an ill-formed parent array.
 * fspad_tree_validate: checks parent order, token range (tokens_host may be
 *   NULL to skip the token checks) and that no two siblings carry the same token.
 */
fspad_status fspad_tree_build_mask(int32_t B, int32_t Nmax, const int32_t* parent_host,
                                   const int32_t* n_nodes_host, uint64_t* mask_host);
fspad_status fspad_tree_validate(int32_t B, int32_t Nmax, int32_t V, const int32_t* parent_host,
                                 const int32_t* tokens_host, const int32_t* n_nodes_host);

/* Static, NUL-terminated description of a status code. */
const char* fspad_status_string(fspad_status status);

#ifdef __cplusplus
}
#endif
#endif /* FSPAD_H */
