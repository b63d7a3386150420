/*
 * cascade.h -- C ABI of the B200 (sm_100a) library for Cascade's sequence-sharded attention.
 *
 * The paper (Cascade: Token-Sharded Private LLM Inference) splits the tokens of a layer into disjoint
 * index sets -- query shards S_j and key/value shards T_k (Section 5.1) -- lets one "AttnNode" per pair
 * (j, k) compute a partial attention output u with per-row statistics m (row max) and e (sum of
 * exponentials) (the Attention-Pass algorithm), and combines the partials over k with a log-sum-exp weighted average
 * (Section 5.2.3, the Post-Pass algorithm), which reproduces unsharded softmax attention exactly.
 * This library runs all parties on one GPU.
 *
 * Conventions
 *  - Every function returns a cascade_status_t; CASCADE_OK is 0.  Nothing throws or aborts across the ABI.
 *    cascade_last_error() returns a thread-local, NUL-terminated description of the last failure.
 *  - Pointers named *_dev / q / k / v / o_* / m_* / l_* / workspace are DEVICE pointers owned by the
 *    caller.  Token-to-shard maps and read-back buffers are HOST pointers.
 *  - All GPU work is enqueued on the caller's stream (a cudaStream_t passed as void*; NULL = default
 *    stream) without synchronising, except where a function says it synchronises.  Some kernels are launched as
 *    programmatic dependents, so that their set-up overlaps the end of earlier work on the stream; all of them
 *    are ordered after earlier work on the stream and before later work, as usual.
 *  - The library allocates device memory only inside cascade_shard_plan (released by
 *    cascade_plan_destroy).  Scratch memory is caller-provided after cascade_workspace_bytes.
 *  - Token ids, shard ids, rows and positions are 0-based.  Query row i of a sequence sits at position
 *    i + q_pos_offset; KV row y at position y.  With causal != 0 row i sees KV rows y <= i + q_pos_offset.
 *  - Tensors are token-major: element (b, token, head, c) lives at
 *    base + b*strides.batch + token*strides.token + head*strides.head + c   (units: elements, c contiguous).
 *    Row starts must be 16-byte aligned.
 *  - Query head h reads KV head h / (n_heads / n_kv_heads)  ("repeat_kv", the Attention-Pass algorithm).
 *  - "Shard-major row order": query rows listed shard 0 first, then shard 1, ..., ascending token id
 *    inside a shard (Section 5.2.2: rows are concatenated in sorted order).  Slot r of that order holds
 *    token Q_IDX[r].
 *  - Statistics: m is the true row maximum of the scaled, masked logits in natural-log units, l is
 *    sum exp(a - m) (the paper's e), both fp32.  A row that sees no key of a shard has m = -inf, l = 0 and
 *    an all-zero partial output.  The stored partial output is the paper's u: normalised inside its shard.
 */
#ifndef CASCADE_H_
#define CASCADE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t cascade_status_t;
enum {
  CASCADE_OK = 0,
  CASCADE_ERR_INVALID_ARG = 1,  /* null pointer, non-positive size, misaligned pointer or stride */
  CASCADE_ERR_BAD_MAP = 2,      /* shard id outside [0, n_shards) */
  CASCADE_ERR_UNSUPPORTED = 3,  /* head_dim not in {64,128}, n_heads % n_kv_heads != 0, unknown dtype */
  CASCADE_ERR_WORKSPACE = 4,    /* workspace missing or smaller than cascade_workspace_bytes reports */
  CASCADE_ERR_ALLOC = 5,        /* host or device allocation failed */
  CASCADE_ERR_CUDA = 6,         /* a CUDA runtime call or launch failed */
  CASCADE_ERR_TIMEOUT = 7       /* a bounded device-side wait gave up (see cascade_plan_device_status) */
};

typedef enum { CASCADE_F32 = 0, CASCADE_BF16 = 1 } cascade_dtype_t;

/* Strides in elements; the head_dim axis is contiguous. */
typedef struct {
  int64_t batch, token, head;
} cascade_strides_t;

typedef struct cascade_plan cascade_plan_t; /* opaque, library-owned */

/* Plan arrays readable with cascade_plan_get.  All int32 except PAIR_CLASS (uint8).
 * Leading dimension n_maps (1 when one map serves the whole batch). */
enum {
  CASCADE_PLAN_Q_OFF = 0,      /* [n_maps][n_q_shards+1]   first slot of each query shard            */
  CASCADE_PLAN_Q_IDX = 1,      /* [n_maps][n_q]            token id held by each shard-major slot     */
  CASCADE_PLAN_Q_INV = 2,      /* [n_maps][n_q]            slot of each token                         */
  CASCADE_PLAN_KV_OFF = 3,     /* [n_maps][n_kv_shards+1]                                             */
  CASCADE_PLAN_KV_IDX = 4,     /* [n_maps][n_kv]                                                      */
  CASCADE_PLAN_KV_INV = 5,     /* [n_maps][n_kv]                                                      */
  CASCADE_PLAN_VIS = 6,        /* [n_maps][n_q][n_kv_shards] visible-prefix length of slot r in T_k   */
  CASCADE_PLAN_PAIR_CLASS = 7  /* [n_maps][n_q_shards][n_kv_shards]  0 EMPTY, 1 PARTIAL, 2 FULL       */
};
enum { CASCADE_PAIR_EMPTY = 0, CASCADE_PAIR_PARTIAL = 1, CASCADE_PAIR_FULL = 2 };

int32_t cascade_version(void);
const char* cascade_last_error(void);

/* Number of kernels this library has launched in this process (monotone; for benchmark accounting). */
int64_t cascade_launch_count(void);

/*
 * Device-side timing of the attention kernel (for roofline accounting; not a step of the method).  Between
 * cascade_kernel_timing_begin() and cascade_kernel_timing_end() every launch of the tensor-core attention kernel or of
 * the decode kernel is bracketed by a pair of CUDA events recorded on the launch stream (at most 8192 launches; later
 * ones are not timed).  cascade_kernel_timing_end SYNCHRONISES the device, stops the recording and returns the summed
 * duration in milliseconds and the number of timed launches (either pointer may be NULL).  The shard-gather and merge
 * launches are not included.  Not thread-safe against concurrent attention calls.  Errors: CUDA.
 */
cascade_status_t cascade_kernel_timing_begin(void);
cascade_status_t cascade_kernel_timing_end(double* total_ms, int64_t* n_launches);

/*
 * cascade_shard_plan -- index maps and causal pair mask (Section 5.1 index sets; Section 5.2.2 sorted
 * concatenation; the sharded mask s^{S_j T_k} = s[:, S_j, T_k]).
 * Because each shard is kept in ascending token order and the mask is unidirectional, row r of pair
 * (j, k) sees exactly the first VIS[r][k] keys of T_k (each mask row is visible entries followed by
 * -inf, Appendix E), so the mask is stored as that prefix length.
 *   n_maps        1 (one map for every sequence) or the batch size (maps laid out [n_maps][n])
 *   q_shard_of    HOST int32 [n_maps][n_q],  values in [0, n_q_shards)
 *   kv_shard_of   HOST int32 [n_maps][n_kv], values in [0, n_kv_shards)
 *   q_pos_offset  position of query row 0 (0 for prefill, n_kv - n_q for decode with the new tokens
 *                 already in the cache)
 *   causal        1 unidirectional mask, 0 no mask
 * Copies the maps, builds the arrays on the host, uploads them on `stream` and SYNCHRONISES that stream.
 * Empty shards are allowed.  Errors: INVALID_ARG, BAD_MAP, ALLOC, CUDA.  *out_plan is set only on success.
 */
cascade_status_t cascade_shard_plan(int32_t n_maps, int32_t n_q, int32_t n_kv, const int32_t* q_shard_of,
                                    const int32_t* kv_shard_of, int32_t n_q_shards, int32_t n_kv_shards,
                                    int32_t q_pos_offset, int32_t causal, void* stream,
                                    cascade_plan_t** out_plan);

/*
 * cascade_shard_plan_resident -- a plan for a party that holds only SOME of the K/V rows: an AttnNode keeps the k, v
 * rows of its own KV shards and nothing else (Section 5.2: every AttnNode_{jk} receives k^{T_k}, v^{T_k}; "Caching" in
 * the appendix on cost optimizations: each node stores the rows of its shard).  The k/v tensors of the attention calls
 * then have n_kv = (number of resident rows) rows, and row y is the token at ORIGINAL position kv_pos[y]; the causal
 * mask compares that position with the query position, so VIS[r][k] = #{y in T_k : kv_pos[y] <= q_idx[r] + q_pos_offset}.
 *   kv_pos   HOST int32 [n_maps][n_kv], non-negative and strictly ascending inside a map (rows kept in token order)
 * Everything else as cascade_shard_plan (which is this call with kv_pos[y] = y).  The partials of such a plan are the
 * columns of the full problem's partials that belong to the resident shards; cascade_merge over the union of all
 * parties' columns gives the exact result (Section 5.2.3).  cascade_attn_sharded_rope refuses these plans (it takes a
 * key row's position from its index).  Errors as cascade_shard_plan; BAD_MAP also for a kv_pos that is not ascending.
 */
cascade_status_t cascade_shard_plan_resident(int32_t n_maps, int32_t n_q, int32_t n_kv, const int32_t* q_shard_of,
                                             const int32_t* kv_shard_of, const int32_t* kv_pos, int32_t n_q_shards,
                                             int32_t n_kv_shards, int32_t q_pos_offset, int32_t causal, void* stream,
                                             cascade_plan_t** out_plan);
/* The same, built on the host only (see cascade_shard_plan_host). */
cascade_status_t cascade_shard_plan_resident_host(int32_t n_maps, int32_t n_q, int32_t n_kv, const int32_t* q_shard_of,
                                                  const int32_t* kv_shard_of, const int32_t* kv_pos,
                                                  int32_t n_q_shards, int32_t n_kv_shards, int32_t q_pos_offset,
                                                  int32_t causal, cascade_plan_t** out_plan);

/* Same arrays as cascade_shard_plan, built on the host only: no CUDA call is made, so it works on a machine
 * without a GPU.  The plan can be read with cascade_plan_get / cascade_plan_dense_mask (device pointers are
 * NULL) and must be destroyed as usual; the attention calls reject it with INVALID_ARG. */
cascade_status_t cascade_shard_plan_host(int32_t n_maps, int32_t n_q, int32_t n_kv, const int32_t* q_shard_of,
                                         const int32_t* kv_shard_of, int32_t n_q_shards, int32_t n_kv_shards,
                                         int32_t q_pos_offset, int32_t causal, cascade_plan_t** out_plan);

/* Frees host and device memory of a plan (NULL is accepted).  Synchronises the device first. */
cascade_status_t cascade_plan_destroy(cascade_plan_t* plan);

/* Read-back of a plan array: host copy (library-owned, valid until destroy), device copy and element
 * count.  Any of the three outputs may be NULL. */
cascade_status_t cascade_plan_get(const cascade_plan_t* plan, int32_t field, const void** host_ptr,
                                  const void** dev_ptr, int64_t* n_elems);

/* Dense mask of pair (j, k) of map `map`: host_out[r * |T_k| + c] = 1 if row r of S_j sees key c of T_k.
 * capacity = bytes available at host_out; WORKSPACE error if smaller than |S_j| * |T_k|. */
cascade_status_t cascade_plan_dense_mask(const cascade_plan_t* plan, int32_t map, int32_t j, int32_t k,
                                         uint8_t* host_out, int64_t capacity);

/* Reads the plan's device status word (SYNCHRONISES the device): 0 = no kernel that used this plan hit a
 * bounded-wait limit; otherwise a code identifying the wait.  Returns TIMEOUT if non-zero.
 * The word is sticky: once a wait inside the tensor-core kernel has given up (2 s without progress), every later
 * tensor-core attention call on this plan returns CASCADE_OK from the host but its blocks write nothing.  A
 * non-zero status therefore invalidates the outputs of every call made on the plan since the last check that read 0;
 * destroy the plan and build a new one.  A caller that cannot afford stale outputs polls this after the calls whose
 * results it is about to use. */
cascade_status_t cascade_plan_device_status(const cascade_plan_t* plan, int32_t* out_code);

/*
 * cascade_attn_partials -- the attention-pass of every AttnNode_{jk} (the Attention-Pass algorithm) in one launch:
 * for each query shard j and KV shard k, a = scale * q^{S_j} (k^{T_k})^T + s^{S_j T_k}; m = row max;
 * l = row sum exp(a - m); u = softmax(a) v^{T_k}.  Rows of Q/K/V are gathered through the plan's maps.
 *   q  [batch][n_q][n_heads][head_dim], k, v [batch][n_kv][n_kv_heads][head_dim]  (strides given)
 *   o_part  [batch][n_kv_shards][n_q shard-major][n_heads][head_dim], same dtype as q, contiguous
 *   m_part, l_part  fp32 [batch][n_kv_shards][n_q shard-major][n_heads], contiguous
 * (Together these are the paper's stage-B payload: n_kv_shards * (head_dim + 2) * n_heads * n_q values
 * per sequence, Appendix D.)  batch must equal n_maps when the plan has per-sequence maps.
 * head_dim in {64,128}; bf16 runs on the tensor cores (tcgen05), and so does fp32 at head_dim 64, its operands split into
 * three bf16 parts each, where that is the faster way; fp32 at head_dim 128, more than 256 KV shards, and head_dim 64
 * without a sufficient workspace run on the fp32 ALU kernels; n_q == 1 with bf16 runs the KV-streaming decode kernel.
 * scale must be positive and finite (INVALID_ARG otherwise: the kernels take row maxima before scaling).
 * Only the k/v rows that some query row of the plan sees have to hold finite values: positions later than the last
 * query position (the unwritten tail of a preallocated cache) may hold anything, NaN bit patterns included; no route
 * lets them reach a result.  batch and n_heads may not exceed 65535 (and batch * n_kv_shards on the ALU route).
 * workspace: as reported by cascade_workspace_bytes(CASCADE_CALL_PARTIALS) (may be 0 -> NULL allowed).  The
 * tensor-core route first copies K and V into shard-major order there (the stage-A hand-over of each KV shard to
 * its AttnNodes, Appendix D): 2 * batch * n_kv_heads * n_kv * head_dim * 2 bytes, overwritten by every call.  fp32 at head_dim
 * 64 keeps the split keys and values there, three times as much and a byte per 64 rows; none is asked for where the ALU kernels
 * are the faster way, and without it they are taken.
 */
cascade_status_t cascade_attn_partials(const cascade_plan_t* plan, cascade_dtype_t dtype, int32_t batch,
                                       int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                                       const void* q, cascade_strides_t q_strides, const void* k,
                                       cascade_strides_t k_strides, const void* v,
                                       cascade_strides_t v_strides, void* o_part, float* m_part,
                                       float* l_part, void* workspace, size_t workspace_bytes,
                                       void* stream);

/*
 * cascade_merge -- the post-pass combine (the Post-Pass algorithm; derivation in Section 5.2.3):
 * n = max_p m_p;  w = sum_p exp(m_p - n) l_p;  o = sum_p exp(m_p - n) l_p u_p / w.
 * Needs no plan.  Inputs in the layout cascade_attn_partials writes, with n_parts = n_kv_shards.
 *   row_scatter  DEVICE int32 [n_rows] or NULL: output token row of partial row r (the plan's Q_IDX
 *                device array); NULL = identity.  With per-sequence maps pass row_scatter_batch_stride
 *                = n_rows, else 0.
 *   o_out        [batch][n_rows][n_heads][head_dim] with strides, dtype as the partials
 *   lse_out      optional fp32 [batch][n_rows][n_heads] (token order): n + ln w; -inf if all parts empty
 * Rows whose parts are all empty produce zeros.
 */
cascade_status_t cascade_merge(cascade_dtype_t dtype, int32_t batch, int32_t n_parts, int32_t n_rows,
                               int32_t n_heads, int32_t head_dim, const void* o_part, const float* m_part,
                               const float* l_part, const int32_t* row_scatter,
                               int64_t row_scatter_batch_stride, void* o_out, cascade_strides_t o_strides,
                               float* lse_out, void* stream);

/*
 * cascade_merge_peers -- stage B of the layer and the post-pass combine in one kernel (Single Layer Forward Pass
 * algorithm: "CompNode_i gets m, e, u" from the AttnNodes, then the Post-Pass algorithm; Section 5.2.3): the parts are
 * read where they were computed instead of being copied to the combining party first.  Source s is the set of
 * partial buffers one party wrote with cascade_attn_partials for ITS KV shards (cascade_shard_plan_resident):
 *   o_parts[s]  DEVICE [batch][parts_per_source[s]][n_source_rows][n_heads][head_dim] in `dtype`
 *   m_parts[s], l_parts[s]  DEVICE fp32 [batch][parts_per_source[s]][n_source_rows][n_heads]
 * The three pointer tables and parts_per_source are HOST arrays of n_sources entries (at most 16).  A source pointer
 * may address another GPU's memory that is mapped into this process (CUDA IPC, peer access): the kernel reads it
 * with plain loads, each 16-byte piece once; it uses no multicast and no TMA.  The caller orders this call after the
 * writers of every source (their streams, or a barrier between processes).
 *   row_gather  DEVICE int32 [n_rows] or NULL: the row of the source buffers (shard-major slot of the whole sequence)
 *               that output row r combines -- the rows of the query shards this party owns; NULL = row r
 *   o_out       [batch][n_rows][n_heads][head_dim] with strides;  lse_out optional fp32 [batch][n_rows][n_heads]
 * The result equals cascade_merge over the union of all sources' parts restricted to the gathered rows.
 * Errors: INVALID_ARG, UNSUPPORTED (dtype, head_dim, more than 16 sources), CUDA.
 */
cascade_status_t cascade_merge_peers(cascade_dtype_t dtype, int32_t batch, int32_t n_sources,
                                     const void* const* o_parts, const float* const* m_parts,
                                     const float* const* l_parts, const int32_t* parts_per_source,
                                     int32_t n_source_rows, const int32_t* row_gather, int32_t n_rows,
                                     int32_t n_heads, int32_t head_dim, void* o_out, cascade_strides_t o_strides,
                                     float* lse_out, void* stream);

/*
 * cascade_attn_sharded -- attention-pass and post-pass fused (the Attention-Pass algorithm followed by the Post-Pass
 * algorithm): carries (n, w, o) across the keys of all shards, so no partial is written to memory; by the identity of
 * Section 5.2.3 the result equals cascade_merge(cascade_attn_partials(...)).  Output in token order:
 *   o_out [batch][n_q][n_heads][head_dim] with strides; lse_out optional fp32 [batch][n_q][n_heads].
 * For n_q == 1 (decode, Appendix F "Caching") the KV shards are processed as independent partials that meet on chip, in
 * one launch (`workspace` is checked but not used).  The tensor-core route (bf16) reads K and V where they are and uses
 * `workspace` only for tensors whose strides its loads cannot take and for calls that are being captured into a graph; a
 * graph follows cascade_plan_advance when it is replayed.  Size: cascade_workspace_bytes(CASCADE_CALL_SHARDED), the size of
 * cascade_attn_partials' workspace on the tensor-core route; heads of 64 columns take the fp32 ALU kernel without it.  fp32 at
 * head_dim 64 as cascade_attn_partials.
 */
cascade_status_t cascade_attn_sharded(const cascade_plan_t* plan, cascade_dtype_t dtype, int32_t batch,
                                      int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                                      const void* q, cascade_strides_t q_strides, const void* k,
                                      cascade_strides_t k_strides, const void* v,
                                      cascade_strides_t v_strides, void* o_out,
                                      cascade_strides_t o_strides, float* lse_out, void* workspace,
                                      size_t workspace_bytes, void* stream);

/*
 * cascade_rope_table -- the positional table p of the rotary embedding (Section 5.1 lists p among the tensors set up
 * before inference and sharded with the tokens; the Pre-Pass algorithm consumes its rows p^{R_i}).  The paper does not print
 * the rotary formula; this library takes the rotate-half form with theta_i = base^(-2 i / head_dim):
 *   table[t][i] = (cos(t theta_i), sin(t theta_i)),  t = 0 .. n_positions-1,  i = 0 .. head_dim/2 - 1,
 * angles formed and evaluated in fp64, stored as fp32 pairs.
 *   table  DEVICE fp32 [n_positions][head_dim/2][2], 16-byte aligned, caller-owned; written on `stream`.
 * Errors: CASCADE_ERR_INVALID_ARG (null / misaligned table, n_positions < 1, odd head_dim, base <= 1),
 * CASCADE_ERR_CUDA (launch failure).
 */
cascade_status_t cascade_rope_table(int32_t n_positions, int32_t head_dim, double base, float* table,
                                    void* stream);

/*
 * cascade_attn_sharded_rope -- cascade_attn_sharded with the tail of the pre-pass fused in (the Pre-Pass algorithm:
 * q <- rotary_pos_emb(q, p^{R_i}), k <- rotary_pos_emb(k, p^{R_i})): q and k are given UNROTATED; every query row is
 * turned by the table row of its position (q_pos_offset + token index) and every key row by the row of its token
 * index while they are staged for the attention kernel, so no separate pass over q and k runs:
 *   y[i] = x[i] cos - x[i + d/2] sin,   y[i + d/2] = x[i + d/2] cos + x[i] sin,   (cos, sin) = table[pos][i],
 * computed in fp32 and rounded once to bf16, the type the pre-pass would hand q and k on in.  Because a row's angle
 * depends on its original index only, the result equals rotating the whole sequence first and calling
 * cascade_attn_sharded.
 *   rope_table   DEVICE table written by cascade_rope_table for head_dim 128, 16-byte aligned, read-only
 *   n_positions  its row count; must cover max(q_pos_offset + n_q, n_kv).  A negative q_pos_offset is taken with the causal
 *                mask only (a row before position 0 sees nothing and yields zeros); INVALID_ARG without
 * All other arguments, the workspace (used here: copies of the rotated keys and of the values) and the outputs are those of
 * cascade_attn_sharded.  A graph that holds the call keeps the positions of its query rows.
 * Supported on the tensor-core route only (bf16, head_dim 128, n_q > 1, at most 256 KV shards); other shapes return
 * CASCADE_ERR_UNSUPPORTED and the caller rotates q and k beforehand.
 */
cascade_status_t cascade_attn_sharded_rope(const cascade_plan_t* plan, cascade_dtype_t dtype, int32_t batch,
                                           int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                                           const void* q, cascade_strides_t q_strides, const void* k,
                                           cascade_strides_t k_strides, const void* v,
                                           cascade_strides_t v_strides, const float* rope_table,
                                           int32_t n_positions, void* o_out, cascade_strides_t o_strides,
                                           float* lse_out, void* workspace, size_t workspace_bytes,
                                           void* stream);

/*
 * Shard-map generators and shard-safety measures.  HOST arrays only, integer only, no device work; the maps they
 * write are what cascade_shard_plan takes.  Token indices are 0-based (the paper prints 1-based ones).
 *
 * cascade_cdelta_shard_map -- (c, delta)-sharding (Section 6, definition of a (c, delta)-sequence): sequence i holds
 * the tokens i c .. i c + c - 1 of every period of delta tokens, shard_of[t] = (t mod delta) / c; the number of
 * sequences that covers [N] is alpha = ceil(delta / c), written to *n_shards_out (optional).  If c does not divide
 * delta the last sequence has clusters of delta mod c tokens.
 *   shard_of  HOST int32 [n_tokens], written.   Errors: INVALID_ARG unless 1 <= c <= delta, n_tokens >= 0.
 */
cascade_status_t cascade_cdelta_shard_map(int32_t n_tokens, int32_t c, int32_t delta, int32_t* shard_of,
                                          int32_t* n_shards_out);

/*
 * cascade_msplit_shard_map -- the m-split of AttnNodes (Section 6.4): every hidden shard R_i is cut into m pieces,
 * R_{i,x} taking the members of sorted R_i at ranks x, x + m, x + 2m, ... (the rule the section's worked example
 * with N = 18, c = 2, delta = 6, m = 2 follows), and the query/KV shards are S_{m i + x} = R_{i,x}; beta = m alpha.
 *   r_shard_of  HOST int32 [n_tokens], values in [0, n_r_shards)     s_shard_of  HOST int32 [n_tokens], written
 * Errors: INVALID_ARG (sizes, null arrays), BAD_MAP (an id outside [0, n_r_shards); the message names the token).
 */
cascade_status_t cascade_msplit_shard_map(int32_t n_tokens, const int32_t* r_shard_of, int32_t n_r_shards, int32_t m,
                                          int32_t* s_shard_of);

/*
 * cascade_index_set_gaps -- clusters and gaps of the index set a node holds, or of the union a colluding set of nodes
 * pools (CompNode_i: R_i; AttnNode_jk: S_j u T_k; appendix on collusion).  A cluster is a maximal run of consecutive
 * held indices; the gap between neighbouring clusters is the number of indices strictly between them, i.e. the
 * unknown tokens a generalized vocab-matching attack must enumerate (V^gap candidates).  For a (c, delta)-sequence
 * every gap is delta - c (Section 6.2 states it as the cluster-to-cluster distance delta - c + 1).  Criteria:
 *   Section 6.2 (leakage from the node's own hidden states):  min_gap + 1 >= rho
 *   Theorem of Section 6.3 and the collusion appendix:         min_gap     >= rho
 *   held  HOST uint8 [n_tokens], non-zero = the index is held.
 *   n_indices, n_clusters, min_gap, max_gap: optional outputs; min_gap = max_gap = -1 with fewer than two clusters.
 */
cascade_status_t cascade_index_set_gaps(int32_t n_tokens, const uint8_t* held, int32_t* n_indices,
                                        int32_t* n_clusters, int32_t* min_gap, int32_t* max_gap);

/*
 * cascade_kl_gaps -- the (k, l)-gaps from the proof of the Section 6.3 theorem: for the node's sorted indices
 * r_1 < r_2 < ... and KV shard S_k, gap (k, l) = { s in S_k : r_l < s < r_{l+1} } without the node's own indices.
 * The attack of the proof needs a NON-EMPTY gap with fewer than rho members, so the call reports, per KV shard, the
 * size of the smallest non-empty gap over l (-1 if every gap of that shard is empty).
 *   r_held  HOST uint8 [n_tokens]      s_shard_of  HOST int32 [n_tokens], values in [0, n_s_shards)
 *   min_gap_per_shard  HOST int32 [n_s_shards], written.   Errors: INVALID_ARG, BAD_MAP.
 */
cascade_status_t cascade_kl_gaps(int32_t n_tokens, const uint8_t* r_held, const int32_t* s_shard_of,
                                 int32_t n_s_shards, int32_t* min_gap_per_shard);

/*
 * cascade_attn_sharded_host -- cascade_attn_sharded for callers whose tensors live in HOST memory (the paper's nodes
 * exchange q, k, v and the outputs over a network; here the host side of the PCIe link stands in for it).  The call
 * copies k and v to the device, then works through the KV heads one at a time: the G = n_heads / n_kv_heads query
 * heads of KV head g are uploaded on one copy stream while the fused attention of head g - 1 runs on the caller's
 * stream and the output of head g - 2 travels back on a second copy stream, so the transfers in both directions
 * overlap each other and the compute.  Results are those of cascade_attn_sharded.
 *   q_host, o_host  HOST, dense [batch][n_q][n_heads][head_dim]; k_host, v_host  HOST, dense
 *                   [batch][n_kv][n_kv_heads][head_dim].  Pinned memory is needed for the copies to be asynchronous.
 *   workspace       DEVICE, 256-byte aligned, cascade_workspace_bytes(CASCADE_CALL_SHARDED_HOST) bytes: staging for
 *                   q, k, v, o and the scratch of one head group.  Overwritten by every call.  Heads of 64 columns take any
 *                   size from the staging alone on (each of the four rounded up to 256 bytes), and the ALU kernels without
 *                   the rest.
 * All work is ordered after what `stream` holds at the time of the call, and `stream` waits for the last output
 * copy: synchronising `stream` makes o_host valid.  The first call on a device creates two internal copy streams and
 * their events (no device memory); all calls on a device share them, so calls from several host threads for the same
 * device must be serialised by the caller.  Errors as cascade_attn_sharded, plus CASCADE_ERR_INVALID_ARG for more than 128 KV
 * heads.
 */
cascade_status_t cascade_attn_sharded_host(const cascade_plan_t* plan, cascade_dtype_t dtype, int32_t batch,
                                           int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                                           const void* q_host, const void* k_host, const void* v_host,
                                           void* o_host, void* workspace, size_t workspace_bytes, void* stream);

/*
 * cascade_plan_advance -- moves the query block of a plan to a new position: token-sharded KV caching (Appendix F,
 * "Caching").  Under a (c, delta)-style scheme the shard of every future token is known in advance, so a decode loop
 * builds ONE plan over the whole cache capacity (n_kv = capacity, every slot already mapped to its KV shard, n_q = 1)
 * and, for each generated token, writes that token's k and v rows at its index of the caller's cache tensors and
 * calls this function with the token's position: the causal mask (key token <= query position) then admits exactly
 * the cache rows written so far, and the new row belongs to its shard's list without any list being rebuilt.
 * Recomputes VIS and PAIR_CLASS for query position q_pos_offset + token index; the index lists do not change.  On a
 * device plan with more than 256 (query row, KV shard) entries a small kernel rewrites the device arrays in stream
 * order from the plan's own index lists (no host computation, no upload; the host copies that cascade_plan_get and
 * cascade_plan_dense_mask return are brought up to date when they are next asked for).  Smaller plans (a decode
 * step), host-only plans and plans over resident K/V rows (kv_pos) recompute on the host and update the device in stream order.  Works for any n_q (a prefill chunk that slides along the sequence);
 * the work-sorted order of the plan's query tiles is left as it was built, which affects speed only.
 * Calls that use the plan before and after must be on `stream` or ordered with it.
 * Cache rows beyond the new position need not be initialised (see cascade_attn_partials); rows at or before it must be
 * written, and finite, before the attention call that follows.
 * Errors: CASCADE_ERR_INVALID_ARG (null plan), CASCADE_ERR_CUDA.
 */
cascade_status_t cascade_plan_advance(cascade_plan_t* plan, int32_t q_pos_offset, void* stream);

/*
 * cascade_attn_decode_static -- the decode case of cascade_attn_sharded (one query row per sequence, bf16,
 * head_dim 128, n_heads / n_kv_heads in {1,2,4,8}) without a workspace argument and without any allocation.
 * (The paper has no counterpart: this is a convenience of this library, not a step of the method.)
 *
 * Who it is for: callers that cannot hand over scratch memory and cannot allocate it either -- a server whose
 * cache manager already owns all free HBM, a decode loop that must not hit the device-wide synchronisation of
 * cudaMalloc / cudaFree, a plug-in that only receives raw pointers.  The per-shard partials meet on chip, so the call needs
 * no scratch memory; it issues no cudaMalloc, cudaFree or other allocating routine.
 *
 *  - Limit: batch * n_kv_shards * n_heads * 264 bytes (rounded up per region to 256) must fit in 16 MiB,
 *    e.g. batch 64 x 16 shards x 32 heads = 8.3 MiB.  Larger problems return CASCADE_ERR_WORKSPACE with a
 *    message naming the sizes; use cascade_attn_sharded with a workspace for those.
 *  - Make the first call on each device during start-up, before any stream capture (it loads the kernel).
 *  - Inputs, outputs, strides, stream and results are exactly those of cascade_attn_sharded.
 */
cascade_status_t cascade_attn_decode_static(const cascade_plan_t* plan, int32_t batch, int32_t n_heads,
                                            int32_t n_kv_heads, float scale, const void* q,
                                            cascade_strides_t q_strides, const void* k,
                                            cascade_strides_t k_strides, const void* v,
                                            cascade_strides_t v_strides, void* o_out, cascade_strides_t o_strides,
                                            float* lse_out, void* stream);

/*
 * cascade_rope_apply -- the rotary steps of the Pre-Pass algorithm (q <- rotary_pos_emb(q, p^{R_i}), the same for k) as
 * a pass of its own, for rows that no fused call covers (fp32, head_dim 64, rows rotated once and then cached):
 *   y[b][r][h][i]       = x[..][i] cos - x[..][i + d/2] sin
 *   y[b][r][h][i + d/2] = x[..][i + d/2] cos + x[..][i] sin,      (cos, sin) = table[first_position + r][i]
 * in fp32, rounded once to `dtype`.  Row r of every sequence sits at position first_position + r.
 *   x, y         DEVICE [batch][n_rows][n_heads][head_dim] with strides (y may be x: in place); head_dim 64 or 128
 *   rope_table   DEVICE table of cascade_rope_table for this head_dim; n_positions its row count
 * Errors: INVALID_ARG (null, misaligned, positions outside the table), UNSUPPORTED (dtype, head_dim), CUDA.
 */
cascade_status_t cascade_rope_apply(cascade_dtype_t dtype, int32_t batch, int32_t n_rows, int32_t n_heads,
                                    int32_t head_dim, const void* x, cascade_strides_t x_strides,
                                    int32_t first_position, const float* rope_table, int32_t n_positions, void* y,
                                    cascade_strides_t y_strides, void* stream);

/*
 * cascade_decode_step_rope -- one generated token against a token-sharded KV cache ("Caching" in the appendix on cost
 * optimizations), with the tail of the Pre-Pass algorithm folded in: given the new token's UNROTATED q, k, v rows
 *   1. moves the plan's query block to `position` (cascade_plan_advance: the mask admits cache rows <= position),
 *   2. rotates the k row by the table row of `position` and writes it, and the v row as it is, at row `position` of the
 *      caches -- the node that holds the token's KV shard appends it; rows already cached are not touched again,
 *   3. rotates the q row and runs the decode route of cascade_attn_sharded on the caches (one partial per KV shard,
 *      then the post-pass combine).
 *   plan            built by cascade_shard_plan over the cache CAPACITY with n_q = 1 (see cascade_plan_advance)
 *   q_new           DEVICE bf16 [batch][1][n_heads][128];  k_new, v_new  DEVICE bf16 [batch][1][n_kv_heads][128]
 *   k_cache, v_cache  DEVICE bf16 [batch][capacity][n_kv_heads][128] with strides; row `position` is WRITTEN
 *   rope_table      DEVICE table of cascade_rope_table for head_dim 128 with more than `position` rows
 *   o_out, lse_out  as cascade_attn_sharded (one row per sequence)
 *   workspace       cascade_workspace_bytes(CASCADE_CALL_DECODE_STEP_ROPE) bytes
 * bf16, head_dim 128, n_heads / n_kv_heads in {1, 2, 4, 8}.  Errors as cascade_attn_sharded and cascade_plan_advance.
 */
cascade_status_t cascade_decode_step_rope(cascade_plan_t* plan, int32_t batch, int32_t n_heads, int32_t n_kv_heads,
                                          float scale, const void* q_new, cascade_strides_t q_strides,
                                          const void* k_new, cascade_strides_t k_new_strides, const void* v_new,
                                          cascade_strides_t v_new_strides, void* k_cache,
                                          cascade_strides_t k_cache_strides, void* v_cache,
                                          cascade_strides_t v_cache_strides, int32_t position, const float* rope_table,
                                          int32_t n_positions, void* o_out, cascade_strides_t o_strides, float* lse_out,
                                          void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------------------------------
 * Paged caches.  A server holds the K/V rows of many sequences, of lengths that nobody knows beforehand, in pages of one pool.
 * (The paper's nodes keep the rows of their shard, "Caching" in the appendix on cost optimizations; it does not say how they
 * lay them out.  A party's pool holds the rows of its own shards, and its calls below return partials like any other.)
 *
 * What the calls share:
 *  - k_pages, v_pages  DEVICE [n_pages][page_size][n_kv_heads][head_dim] with strides (batch: from page to page, token: from row to
 *                      row of a page, head), so pages may be laid out row by row or head by head; page_size a multiple of 16
 *  - page_table        DEVICE int32, row b (table_stride apart) the ids of the pages of sequence b, of which max_pages may be read;
 *                      row y of its cache is row y % page_size of page page_table[b][y / page_size].  Entries past the last page
 *                      that the length needs may hold anything
 *  - row_start         DEVICE int32 [batch + 1]: the new rows of sequence b are rows row_start[b] .. row_start[b + 1] - 1 of
 *                      tensors [n_rows][heads][head_dim] (strides.batch is not used).  Rows before the first and behind the last
 *                      sequence are padding: outputs leave them as they were
 *  - kv_len            DEVICE int32 [batch]: rows in the cache of sequence b, its new rows counted
 * Lengths, row starts and tables are read on the device when the call runs, so a captured graph follows them.  What they say is
 * checked there before it forms an address.  A bad row_start counts as no rows, a bad length as the nearest good one, a bad page
 * id as page 0 (nothing is written to it); the first is kept for cascade_paged_status, and the outputs of its sequence are then
 * not to be used.
 * New rows may only go to pages that one sequence holds (cascade_pages_fork sees to that).  Two calls that write the same pages, or
 * pages that the other reads, have to be ordered by the caller.  Make a first paged call on each device before one is captured (it
 * loads the kernels).  No sequence may have room for more than 2^30 rows, and in attention all of them together for 2^35 or more.
 */

/* Reads and clears what the paged calls on the current device have reported (SYNCHRONISES the device).  *out_code: 0, a code of
 * 121 on for a bad index (BAD_MAP; the message names it and where it stood), or that of a bounded wait that gave up (TIMEOUT).
 * After a wait has given up, later bf16 calls of cascade_attn_paged may write nothing until this has been called. */
cascade_status_t cascade_paged_status(int32_t* out_code);

/*
 * cascade_rope_table_scaled -- cascade_rope_table for angles stretched to longer contexts: theta_i = base^(-2 i / rot_dim), i <
 * rot_dim / 2, then by `kind`
 *   CASCADE_ROPE_NONE    as it is
 *   CASCADE_ROPE_LINEAR  theta / factor
 *   CASCADE_ROPE_BASE    base * factor^(rot_dim / (rot_dim - 2)) in the place of base (rot_dim above 2)
 *   CASCADE_ROPE_BANDS   by the turns t = original_positions theta / (2 pi): theta for t >= high, theta / factor for t <= low, and
 *                        between them mixed with weight (t - low) / (high - low) of theta
 *   CASCADE_ROPE_RAMP    by the dimension: D(t) = rot_dim ln(original_positions / (2 pi t)) / (2 ln base) turns t times; theta up
 *                        to a = max(0, floor D(high)), theta / factor from b = min(rot_dim - 1, ceil D(low)) on, mixed with
 *                        weight (i - a) / (b - a) of the latter between them
 * cos and sin are multiplied by `attention`; 0 stands for 0.1 ln(factor) + 1 with RAMP and 1 otherwise.
 *   table  DEVICE fp32 [n_positions][rot_dim / 2][2], 16-byte aligned.  Angles are formed in fp64.
 * Errors: INVALID_ARG (sizes, an odd rot_dim, base <= 1, factor < 1, not 0 < low < high or original_positions <= 0 where they are
 * used), CUDA.
 */
enum { CASCADE_ROPE_NONE = 0, CASCADE_ROPE_LINEAR = 1, CASCADE_ROPE_BASE = 2, CASCADE_ROPE_BANDS = 3, CASCADE_ROPE_RAMP = 4 };
cascade_status_t cascade_rope_table_scaled(int32_t n_positions, int32_t rot_dim, double base, int32_t kind, double factor,
                                           double original_positions, double low, double high, double attention,
                                           float* table, void* stream);

/*
 * cascade_rope_rows -- the rotary step of the Pre-Pass algorithm for rows that stand anywhere: row r by the table row of
 * positions[r].  Only the first rot_dim columns are turned, the others pass through:
 *   interleaved = 0   pairs (i, i + rot_dim / 2)        interleaved = 1   pairs (2 i, 2 i + 1)         i < rot_dim / 2
 * in fp32, rounded once to `dtype`.
 *   x, y        DEVICE [n_rows][n_heads][head_dim] with strides (batch unused); y may be x.  head_dim 64 or 128
 *   positions   DEVICE int32 [n_rows]; a negative one marks a padded row, whose y stays as it was
 *   rope_table  DEVICE fp32 [n_positions][rot_dim / 2][2]; rot_dim a multiple of 16, at most head_dim
 * A position past the table is reported to cascade_paged_status and its row left as it was.
 * Errors: INVALID_ARG, UNSUPPORTED (dtype, head_dim, rot_dim), CUDA.
 */
cascade_status_t cascade_rope_rows(cascade_dtype_t dtype, int32_t n_rows, int32_t n_heads, int32_t head_dim, int32_t rot_dim,
                                   int32_t interleaved, const void* x, cascade_strides_t x_strides, const int32_t* positions,
                                   const float* rope_table, int32_t n_positions, void* y, cascade_strides_t y_strides,
                                   void* stream);

/*
 * cascade_paged_append -- the new rows of a batch go to the pages of their sequences, in one launch: row i of the n of sequence b
 * becomes row y = kv_len[b] - n + i of its cache.  With rope_table k is turned on the way as by cascade_rope_rows (rot_dim,
 * interleaved), and so are the queries: q_out = R q.
 *   k, v       DEVICE [n_rows][n_kv_heads][head_dim] with strides;  q, q_out  DEVICE [n_rows][n_heads][head_dim] or both NULL;
 *              q_out may be q
 *   positions  DEVICE int32 [n_rows] or NULL: y itself.  (A party that holds some of the tokens gives the original ones.)
 *   rope_table NULL: rows are taken as they are
 * A row whose place, page or position is bad is reported and not written, and so are all rows of a sequence whose kv_len is negative or
 * more than its row of the table has room for.  Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
cascade_status_t cascade_paged_append(cascade_dtype_t dtype, int32_t batch, int32_t n_rows, int32_t n_heads,
                                      int32_t n_kv_heads, int32_t head_dim, const void* q, cascade_strides_t q_strides,
                                      void* q_out, cascade_strides_t q_out_strides, const void* k,
                                      cascade_strides_t k_strides, const void* v, cascade_strides_t v_strides,
                                      const int32_t* positions, const float* rope_table, int32_t n_positions,
                                      int32_t rot_dim, int32_t interleaved, void* k_pages, cascade_strides_t k_page_strides,
                                      void* v_pages, cascade_strides_t v_page_strides, int32_t n_pages, int32_t page_size,
                                      const int32_t* page_table, int64_t table_stride, int32_t max_pages,
                                      const int32_t* row_start, const int32_t* kv_len, void* stream);

/*
 * cascade_attn_paged -- the Attention-Pass and Post-Pass algorithms for the new rows of a ragged batch over their paged caches:
 * chunks of prompts, single tokens and drafts side by side, or the rows of a decoder over an encoder's states of another length.
 *   q, o_out   DEVICE [n_rows][n_heads][head_dim] with strides;  lse_out  optional fp32 [n_rows][n_heads]
 *   causal     1: row i of the n of sequence b sees the cache rows y <= kv_len[b] - n + i;  0: all kv_len[b]
 *   visible    DEVICE int32 [n_rows] or NULL: the number of cache rows that a row sees instead (at most kv_len[b]); for a party
 *              whose pool holds the rows of a shard, VIS of its plan (cascade_shard_plan_resident)
 *   max_rows   no sequence has more rows; goes into the choice of kernels only.  A sequence with more is either reported and left as it
 *              was (where the kernel for few rows is alone) or worked out like any other, and then not reported
 * A row that sees nothing yields zeros and lse = -inf.  (o_out, lse_out, 1) of one party is a partial (u, m, l) for cascade_merge
 * with those of others.  A query that holds a NaN yields NaN in its row and head of o_out and lse_out, and nowhere else.  Rows of the
 * cache that no length reaches, and those that `visible` lets no row of their sequence see, may hold anything, NaN included.
 * bf16 and fp32, head_dim 64 and 128, n_heads a multiple of n_kv_heads.  K and V row starts must be 16-byte aligned, and for bf16
 * the strides of pages positive and below 2^38 elements.  scale positive and finite.  Rows of the cache that are seen hold finite
 * values.  bf16: the weights keep 16 bits of mantissa in the product with V for single tokens and for drafts whose max_rows times the
 * heads of a KV head is at most 16, and with heads of 64 in longer chunks; elsewhere they are rounded to bf16, as in cascade_attn_sharded.
 * So the last bits of a row depend on how many rows stand beside it.  fp32 operands are taken apart into two tf32 parts each, and
 * products keep what lies above 2^-21 of themselves.
 *   workspace  cascade_attn_paged_workspace_bytes(...) bytes, 256-byte aligned; overwritten by every call, so calls that may run at
 *              the same time need one each
 * Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, CUDA.
 */
cascade_status_t cascade_attn_paged(cascade_dtype_t dtype, int32_t batch, int32_t n_rows, int32_t max_rows, int32_t n_heads,
                                    int32_t n_kv_heads, int32_t head_dim, float scale, int32_t causal, const void* q,
                                    cascade_strides_t q_strides, const void* k_pages, cascade_strides_t k_page_strides,
                                    const void* v_pages, cascade_strides_t v_page_strides, int32_t n_pages,
                                    int32_t page_size, const int32_t* page_table, int64_t table_stride, int32_t max_pages,
                                    const int32_t* row_start, const int32_t* kv_len, const int32_t* visible, void* o_out,
                                    cascade_strides_t o_strides, float* lse_out, void* workspace, size_t workspace_bytes,
                                    void* stream);
cascade_status_t cascade_attn_paged_workspace_bytes(cascade_dtype_t dtype, int32_t batch, int32_t n_rows, int32_t max_rows,
                                                    int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                                    int32_t page_size, int32_t max_pages, size_t* out_bytes);

/*
 * cascade_pages_fork -- one step of the page tables, on the device: sequence i of the new state continues sequence source[i] of the
 * old one (-1: none, the place is emptied; the same source any number of times) and gets room for add[i] more rows.
 * A page is held by every sequence whose length reaches it, and free when none holds it.  Pages are shared as they are; a sequence
 * that goes on writing a partly filled page which others hold, too, gets a copy of its own, except the first of them where all of
 * its holders do.  New pages are the free ones with the lowest ids, in the order of the sequences (the copy first).
 *   table_in, kv_len_in    DEVICE int32 [n_seqs][width], [n_seqs]: the old state;  source, add  DEVICE int32 [n_seqs]
 *   table_out, kv_len_out  the new one (kv_len = old + add); entries past the last page -1.  May not overlap the old one
 *   refs      DEVICE int32 [n_pages], written: holders of every page
 *   copies    DEVICE int32 [n_seqs][2], written: (from, to) for cascade_pages_copy, before the new rows are appended; or (-1, -1)
 *   report    DEVICE int32 [4], written: pages lacking; sequences that the table is too narrow for; bad entries (a source, a
 *             length, a page id, a negative add); pages left free.  Unless the first three are 0 nothing is done: the new state is
 *             the old one
 * One launch, no atomics whose order matters.  n_seqs at most 8192, n_pages at most 2^30, n_seqs * width below 2^31.
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
cascade_status_t cascade_pages_fork(int32_t n_seqs, int32_t width, int32_t n_pages, int32_t page_size,
                                    const int32_t* table_in, const int32_t* kv_len_in, const int32_t* source,
                                    const int32_t* add, int32_t* table_out, int32_t* kv_len_out, int32_t* refs,
                                    int32_t* copies, int32_t* report, void* stream);

/*
 * cascade_pages_compact -- moves the held pages together at the front of the pool: of n_live held pages, those from id n_live on go,
 * in order, to the free ids below it; the others stay.  (Fewest moves, and no page is both moved and moved to.)
 *   table_out  the table with the new ids, entries past the last page -1; may not overlap table_in
 *   refs       as cascade_pages_fork, by the new ids
 *   moves      DEVICE int32 [n_pages / 2][2], written: (from, to) for cascade_pages_copy, then (-1, -1)
 *   report     DEVICE int32 [4], written: n_live; moves; bad entries (then nothing is moved); free pages
 * n_pages at most 2^30, n_seqs * width below 2^31.  Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
cascade_status_t cascade_pages_compact(int32_t n_seqs, int32_t width, int32_t n_pages, int32_t page_size,
                                       const int32_t* table_in, const int32_t* kv_len, int32_t* table_out, int32_t* refs,
                                       int32_t* moves, int32_t* report, void* stream);

/*
 * cascade_pages_copy -- copies page pairs[j][0] over page pairs[j][1] in every pool (K and V of every layer), in one launch; pairs
 * with a -1 are skipped, ids past n_pages reported to cascade_paged_status.  No page may be copied to twice, or both from and to
 * (what it then holds is not defined).
 *   pools        HOST array of n_pools (at most 256) DEVICE pointers, 16-byte aligned
 *   page_strides HOST int64 [n_pools]: bytes from page to page, at least page_bytes
 *   page_bytes   bytes of a page, which is contiguous; a multiple of 16
 *   pairs        DEVICE int32 [n_pairs][2], at most 2^30 of them
 * Errors: INVALID_ARG, UNSUPPORTED (more pools or pairs), CUDA.
 */
cascade_status_t cascade_pages_copy(int32_t n_pools, void* const* pools, const int64_t* page_strides, int64_t page_bytes,
                                    int32_t n_pages, const int32_t* pairs, int32_t n_pairs, void* stream);

enum {
  CASCADE_CALL_PARTIALS = 0,
  CASCADE_CALL_SHARDED = 1,
  CASCADE_CALL_SHARDED_HOST = 2,
  CASCADE_CALL_DECODE_STEP_ROPE = 3
};

/* Scratch bytes the given call needs for this plan and shape (0 if none).  The workspace must be
 * 256-byte aligned. */
cascade_status_t cascade_workspace_bytes(const cascade_plan_t* plan, int32_t which_call,
                                         cascade_dtype_t dtype, int32_t batch, int32_t n_heads,
                                         int32_t n_kv_heads, int32_t head_dim, size_t* out_bytes);

#ifdef __cplusplus
}
#endif
#endif /* CASCADE_H_ */
