/*
 * kvs.h -- C ABI of the MI355X (gfx950) library for the DHD KV-reuse hot path of KVShare
 * (Dual-Stage High Deviation token selection, Alg. 1 / Eq. (3); partial recomputation,
 * App. A; decode-stage re-check, Sec. 4.2).
 *
 * Conventions shared by every call
 * --------------------------------
 * Pointers marked [dev] are device (HBM) addresses, pointers marked [host] are ordinary host
 * memory that is read before the call returns.  The caller owns every buffer; the library
 * allocates nothing, reads no environment variable, and never synchronises.  The only state it
 * keeps between calls is, per device, which kernels have had their launch attributes set and the
 * device's compute-unit count (both written once, safely from several host threads).  Each call checks
 * its arguments on the host, enqueues its kernels on `stream` (a hipStream_t passed as
 * void*, NULL = the default stream) and returns.  Outputs are valid in stream order.
 *
 * Layouts are row-major and contiguous:
 *   K, V        [rows, n_kv_heads, head_dim]   element type given by kvs_shape.dtype
 *   Q           [rows, n_q_heads,  head_dim]
 *   dev_k/dev_v [n_kv_heads, rows] fp32        per-token, per-KV-head L1 deviation
 *   alpha       [n_kv_heads, rows] fp32        attention column mass, summed over the query
 *                                              heads that share the KV head
 *   score       [rows] fp32                    -inf for tokens that are not candidates
 * Query head h reads KV head h / (n_q_heads / n_kv_heads).  K/V/Q base addresses must be
 * 16-byte aligned.
 *
 * Errors: every function returns a kvs_status.  Argument errors are detected on the host
 * before anything is enqueued (KVS_EINVAL: NULL required pointer, negative size, k larger
 * than its row, n_q_heads not a multiple of n_kv_heads, unsorted offsets; KVS_EUNSUPPORTED:
 * head_dim/dtype combination that has no kernel; KVS_EWORKSPACE: workspace too small;
 * KVS_EHIP: the HIP runtime refused a launch).  kvs_last_error() returns a thread-local
 * description of the most recent failure.  Nothing throws or aborts across this boundary.
 *
 * Supported shapes: dtype KVS_BF16 or KVS_F32; head_dim 64 or 128; any n_q_heads that is a
 * multiple of n_kv_heads (n_kv_heads <= 64).
 */
#ifndef KVS_H
#define KVS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KVS_API __attribute__((visibility("default")))

typedef enum {
    KVS_OK = 0,
    KVS_EINVAL = 1,
    KVS_EUNSUPPORTED = 2,
    KVS_EWORKSPACE = 3,
    KVS_EHIP = 4
} kvs_status;

typedef enum { KVS_F32 = 0, KVS_BF16 = 1 } kvs_dtype;

/* KVS_SCORE_V is the paper's score (value deviation only, Sec. 4.1 drops the key term);
 * KVS_SCORE_KV adds the key deviation's L1 norm under the same weight. */
typedef enum { KVS_SCORE_V = 0, KVS_SCORE_KV = 1 } kvs_score_mode;

typedef struct {
    int32_t n_q_heads;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t dtype; /* kvs_dtype */
} kvs_shape;

/*
 * kvs_deviation -- Alg. 1 step 3 / Eq. (3): the deviation impact score of every token.
 *
 *   dev_v[g,i] = sum_c | v_fresh[i,g,c] - v_cache[i,g,c] |        (L1 norm of Delta V_i on head g)
 *   dev_k[g,i] likewise on K (computed when mode == KVS_SCORE_KV or dev_k != NULL)
 *   score[i]   = sum_g alpha[g,i] * dev_v[g,i]                    mode KVS_SCORE_V
 *              = sum_g alpha[g,i] * (dev_k[g,i] + dev_v[g,i])     mode KVS_SCORE_KV
 *   score[i]   = -inf where reused[i] == 0 (the token was computed fresh, nothing to repair)
 *
 * n_tokens            rows of every tensor (0 is allowed: nothing is launched)
 * k_fresh, k_cache    [dev] may be NULL in mode KVS_SCORE_V with dev_k == NULL
 * v_fresh, v_cache    [dev] required
 * reused              [dev] uint8[n_tokens], NULL = every token is a candidate
 * alpha               [dev] fp32[n_kv_heads, n_tokens], NULL = 1 (magnitude-only ranking)
 * dev_k, dev_v, score [dev] outputs; each may be NULL if not wanted
 * All arithmetic is fp32 on exactly widened inputs, in a fixed order (bit-reproducible).
 */
KVS_API kvs_status kvs_deviation(const kvs_shape *shape, int64_t n_tokens,
                         const void *k_fresh, const void *v_fresh,
                         const void *k_cache, const void *v_cache,
                         const uint8_t *reused, const float *alpha, int32_t mode,
                         float *dev_k, float *dev_v, float *score, void *stream);

/*
 * kvs_deviation_topk -- Alg. 1 steps 3 and 4 in one call: the scores of kvs_deviation and, from
 * them, the k highest-scoring tokens of the one row of n_tokens scores, exactly as
 * kvs_select_topk(score, 1, {0, n_tokens}, {k}, idx_out) would return them (order (score
 * descending, index ascending), -0 equal to +0, -inf last, ascending indices out; bit-identical
 * to the two separate calls).  All arguments up to `score` are those of kvs_deviation.
 *
 * k        0 <= k <= n_tokens           idx_out [dev] int32[k]
 * score    [dev] fp32[n_tokens]; may be NULL only for rows of 12289 to 262144 tokens (outside that
 *          range the ranking reads the scores back from it)
 * workspace [dev] optional, as for kvs_select_topk: only used by rows above 262144 tokens
 *
 * Rows of up to 12288 tokens (one workgroup ranks them as fast) and above 262144 run as the two
 * separate calls.  Rows in between take three launches: the scoring kernel also stores every token's
 * order-preserving key and counts the keys' leading 13 bits into a histogram (integer atomics, so
 * the counts do not depend on arrival order and the result stays deterministic); then, with one
 * workgroup per 1024 keys, a launch that reads the threshold's bin off the histogram and sets the
 * few hundred keys of that bin aside, and a launch that resolves the other 19 bits on those and
 * writes the list.  Keys, histogram (32 KiB) and the records the launches exchange live in
 * device memory that belongs to the library (2.1 MB per device); the histogram is all zero
 * whenever no such call is in flight.  Calls that overlap in time on one device (two streams, two
 * host threads) would mix their counts: the caller serialises them.
 */
KVS_API kvs_status kvs_deviation_topk(const kvs_shape *shape, int64_t n_tokens,
                              const void *k_fresh, const void *v_fresh,
                              const void *k_cache, const void *v_cache,
                              const uint8_t *reused, const float *alpha, int32_t mode,
                              float *dev_k, float *dev_v, float *score,
                              int32_t k, int32_t *idx_out,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * kvs_select_topk -- Alg. 1 step 4: the k highest-scoring entries of each row.
 *
 * Row r of the ragged matrix is scores[row_off[r] .. row_off[r+1]).  The k_row[r] entries
 * that come first in the order (score descending, index ascending) are written as row-local
 * int32 indices, in ascending index order, at idx_out + sum(k_row[0..r)).  Scores compare as
 * real numbers (-0 equals +0); -inf entries rank last (still by index); NaN scores are a
 * caller error with unspecified (but memory-safe) results.  The result is exact and
 * deterministic.
 *
 * scores   [dev] fp32            row_off [host] int64[n_rows+1], non-decreasing
 * k_row    [host] int32[n_rows], 0 <= k_row[r] <= row length; rows longer than 2^31-1 are
 *          rejected
 * idx_out  [dev] int32[sum k_row]
 * workspace [dev] optional (NULL / 0 is valid), 256-byte aligned, kvs_workspace_size("select_topk",
 *          any valid shape, n_rows, total scores) bytes: rows longer than 49152 entries are then
 *          cut into parts of 32768 that run on workgroups of their own (four launches, 41 us
 *          instead of 105 us for 131072 entries); without it, or for a row of more than 64
 *          parts, such a row is handled by one workgroup.  The result is the same either way.
 */
KVS_API kvs_status kvs_select_topk(const float *scores, int32_t n_rows, const int64_t *row_off,
                           const int32_t *k_row, int32_t *idx_out,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * kvs_select_topk_static -- kvs_select_topk for callers that cannot allocate device memory (code
 * under stream capture, serving loops and harnesses that forbid hipMalloc): same arguments without
 * the workspace, same results.  Rows longer than 49152 scores, which kvs_select_topk spreads over
 * several workgroups only when given a workspace, here use a scratch buffer that belongs to the
 * library: a file-scope device array of 4.3 MB (each device the library runs on holds it until
 * the process ends).  The call allocates and frees nothing; on its first call on a device it asks
 * the runtime once for that device's address of the array (a call with n_rows = 0 does just
 * that and may be made ahead of time, e.g. before a stream capture begins).
 *
 * Limit: every row at most 1048576 (2^20) scores; a longer row returns KVS_EINVAL before anything
 * is launched.  All calls on one device share that device's scratch and the kernels overwrite what
 * they use before reading it, so nothing has to be cleared between calls; calls that overlap in
 * time on one device (different streams, or host threads) race on it and must be serialised by
 * the caller.
 */
KVS_API kvs_status kvs_select_topk_static(const float *scores, int32_t n_rows, const int64_t *row_off,
                                  const int32_t *k_row, int32_t *idx_out, void *stream);

/*
 * kvs_scatter_kv -- the KV Writer of App. A: recomputed K/V replace the reused entries.
 *
 *   k_cache[sel_pos[s]] = k_new[s],  v_cache[sel_pos[s]] = v_new[s]      for s in [0, n_sel)
 *   reused[sel_pos[s]] = 0           (if reused != NULL)  the token is no longer a candidate
 *   dev_v[g, sel_pos[s]] = 0         (if dev_v  != NULL)  its stored deviation is repaired
 *
 * n_rows     rows of the cache (and row stride of dev_v)
 * k_new,v_new [dev] [n_sel, n_kv_heads, head_dim]
 * sel_pos    [dev] int32[n_sel], global cache rows in [0, n_rows), all distinct (duplicates
 *            race: one of the writers wins per 16-byte piece)
 */
KVS_API kvs_status kvs_scatter_kv(const kvs_shape *shape, int64_t n_rows,
                          const void *k_new, const void *v_new,
                          const int32_t *sel_pos, int64_t n_sel,
                          void *k_cache, void *v_cache, uint8_t *reused, float *dev_v,
                          void *stream);

/*
 * kvs_partial_attention -- Eq. (1) restricted to the rows of the selected tokens (App. A:
 * only the selected tokens are computed, the others' KV is reused).
 *
 * Request b owns cache rows [ctx_off[b], ctx_off[b] + ctx_len[b]) and the selected tokens
 * [cu_sel[b], cu_sel[b+1]).  Selected token s sits at request-local position p = sel_pos[s]
 * and its query head h attends causally, by that original position, over the cache as it
 * stands (recomputed rows already scattered in):
 *
 *   out[s,h,:] = sum_{i <= p} softmax_i( scale * q_sel[s,h,:] . K[ctx_off[b]+i, g(h), :] )
 *                             * V[ctx_off[b]+i, g(h), :]
 *   lse[s,h]   = log sum_{i <= p} exp( scale * q . K_i )          (natural log; optional)
 *
 * ctx_off, ctx_len [host] int64[batch];  cu_sel [host] int64[batch+1], non-decreasing
 * q_sel   [dev] [n_sel, n_q_heads, head_dim]         sel_pos [dev] int32[n_sel], ascending
 *         within each request, each in [0, ctx_len[b])
 * out     [dev] [n_sel, n_q_heads, head_dim] in the shape's dtype
 * lse_out [dev] fp32[n_sel, n_q_heads] or NULL
 * workspace [dev] optional (NULL / 0 is valid), 256-byte aligned.  With at least
 *         kvs_workspace_size("partial_attention", ...) bytes, launches too small to fill the chip
 *         (few selected tokens over long contexts, e.g. the decode-stage recompute) cut each row tile's
 *         key range into up to 16 pieces handled by separate workgroups and merge them; results are the
 *         same up to fp32 summation order.  With less, such launches take fewer pieces or keep whole key
 *         ranges.  Launches that fill the chip keep whole key ranges; where they hold several requests
 *         their workgroups draw work from counters in it (without it they take it in a fixed order).  As
 *         every workspace it is one call's until that call has ended on its stream.  The size
 *         asked for stays below 0.56 GB for one request (528 bytes a row and piece).
 * bf16 inputs (head_dim 128, scale > 0) are contracted on the matrix cores with fp32 accumulation
 * and an fp32 softmax, the softmax weights entering the second product as bf16; every other case
 * is computed in fp32 throughout, on the fp32 matrix instruction.  In bf16 launches of many rows weights lie around 2^-60 while a row's
 * first logits are its largest: values below 2^-60 may lose bits there, and sums of values beyond 2^27 may become infinite.
 */
KVS_API kvs_status kvs_partial_attention(const kvs_shape *shape, int32_t batch,
                                 const int64_t *ctx_off, const int64_t *ctx_len,
                                 const int64_t *cu_sel,
                                 const void *q_sel, const int32_t *sel_pos,
                                 const void *k_cache, const void *v_cache, float scale,
                                 void *out, float *lse_out,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * kvs_decode_check -- Sec. 4.2: Alg. 1 re-run in the decode stage with alpha replaced by the
 * decoding token's current attention over the cache.
 *
 * For request b (its new token's K/V already appended, context ctx_len[b] rows):
 *   a[h,i]   = softmax_{i in [0, ctx_len[b])}( scale * q_new[b,h,:] . K[ctx_off[b]+i, g(h), :] )
 *   score[i] = sum_g ( sum_{h in group g} a[h,i] ) * dev_v[g, ctx_off[b]+i]   if reused, else -inf
 * and the k_req[b] best candidates (same order and tie rule as kvs_select_topk) are written
 * as ascending request-local indices at idx_out + sum(k_req[0..b)).
 *
 * n_rows    rows of the packed cache (row stride of dev_v, length of reused / score_out)
 * ctx_off, ctx_len [host] int64[batch]; every context lies inside [0, n_rows) and no two contexts
 *           share a cache row (KVS_EINVAL otherwise: scores and logits are kept per cache row)
 * q_new     [dev] [batch, n_q_heads, head_dim]
 * v_cache   [dev] only read when attn_out != NULL
 * dev_v     [dev] fp32[n_kv_heads, n_rows] as left by kvs_deviation / kvs_scatter_kv
 * reused    [dev] uint8[n_rows] or NULL (all candidates)
 * k_req     [host] int32[batch], 0 <= k_req[b] <= ctx_len[b]
 * score_out [dev] fp32[n_rows] or NULL; rows outside the contexts are not written
 * attn_out  [dev] [batch, n_q_heads, head_dim] (shape dtype) or NULL: sum_i a[h,i] * V_i
 * A call with one context of 12289..262144 rows selects the way kvs_deviation_topk does (keys and their
 * histogram from the scoring launch, two short selecting launches, same index list bit for bit) and, like it,
 * uses 2.1 MB of device memory that belongs to the library: such calls and kvs_deviation_topk calls on one
 * device must not overlap (one stream, or ordered by events).
 */
KVS_API kvs_status kvs_decode_check(const kvs_shape *shape, int32_t batch, int64_t n_rows,
                            const int64_t *ctx_off, const int64_t *ctx_len,
                            const void *q_new, const void *k_cache, const void *v_cache,
                            const float *dev_v, const uint8_t *reused, float scale,
                            const int32_t *k_req, int32_t *idx_out, float *score_out,
                            void *attn_out,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * kvs_attn_colsum -- Alg. 1 steps 1-2: the attention column mass of a whole prefill,
 *     alpha[g, i] = sum over the query heads h of KV head g, and over the rows j >= i, of A_h[j, i],
 *     A_h = row softmax over the keys i <= j of scale * q[j, h] . k[i, g]      (Eq. (3), causal),
 * i.e. the alpha that kvs_deviation takes.  Every row of A sums to 1, so sum_i alpha[g, i] =
 * n_tokens * n_q_heads / n_kv_heads.  The score matrix is never stored: one sweep leaves each
 * row's log-sum-exp in the workspace, a second one sums exp(score - lse) down the columns.
 * Cost: two passes of n_tokens^2 / 2 * head_dim * n_q_heads multiply-adds on the matrix cores
 * (fp32 layers of up to 2048 tokens, with the workspace asked for: one).
 *
 * bf16 with head_dim 128 and a positive scale runs on the matrix cores (tensors below 4 GiB);
 * every other supported shape, fp32 included, takes an fp32 kernel that is only meant for
 * small problems.  Q and K as for the other calls: [n_tokens, heads, head_dim], 16-byte aligned.
 *
 * q         [dev] [n_tokens, n_q_heads, head_dim]
 * k         [dev] [n_tokens, n_kv_heads, head_dim] (the fresh keys)
 * alpha     [dev] fp32[n_kv_heads, n_tokens], written
 * workspace [dev] kvs_workspace_size("attn_colsum", shape, 1, n_tokens, 0) bytes, 256-byte
 *           aligned, required; contents on return are unspecified.  It holds every row's softmax statistics and the
 *           results of the pieces into which short sweeps, and sweeps of uneven blocks, are cut (short fp32 layers also
 *           run, in two passes, with 8 * n_tokens * n_q_heads bytes rounded up to 512, and 256)
 */
KVS_API kvs_status kvs_attn_colsum(const kvs_shape *shape, int64_t n_tokens, const void *q, const void *k,
                           float scale, float *alpha,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * kvs_first_order_impact -- Sec. 4.1, Eq. (2): the first-order expansion of the attention output's
 * deviation, dH ~ (dH/dK) dK + (dH/dV) dV, rated token by token.  With H = A V the correct (fresh,
 * causal) attention, dK = k_cache - k_fresh and dV = v_cache - v_fresh, reusing token i's cache
 * entry moves output row j >= i of query head h (KV head g) by
 *     A[h,j,i] * dV[g,i]  +  A[h,j,i] * scale * (q[j,h] . dK[g,i]) * (V[g,i] - H[h,j])
 * (value direction: dH/dV = A; key direction: the softmax Jacobian), and
 *     impact_v[i]  = sum over h, j of the L1 norm of the first term  (= Eq. (3): alpha * |dV|_1)
 *     impact_k[i]  = ... of the second term
 *     impact_kv[i] = ... of their sum
 * with -inf where reused[i] == 0.  The key direction is what the paper leaves out of Alg. 1 to save
 * work (it costs n_tokens^2 / 2 * n_q_heads * head_dim vector operations and is no matrix product);
 * this call exists to rank by it on check layers and to compare the two rankings (App. D.2).
 *
 * q        [dev] [n_tokens, n_q_heads, head_dim]
 * h_fresh  [dev] [n_tokens, n_q_heads, head_dim] (shape dtype): the causal attention of every row over
 *          the fresh K/V, e.g. from kvs_partial_attention with every token selected
 * lse      [dev] fp32[n_tokens, n_q_heads]: that attention's log-sum-exp (natural log), same call
 * reused   [dev] uint8[n_tokens] or NULL (every token is rated)
 * impact_* [dev] fp32[n_tokens], each may be NULL
 * workspace [dev] kvs_workspace_size("first_order_impact", shape, 1, n_tokens, 0) bytes, 256-byte aligned
 * All arithmetic is fp32 on exactly widened inputs in a fixed order (bit-reproducible); up to 2^20 tokens.
 */
KVS_API kvs_status kvs_first_order_impact(const kvs_shape *shape, int64_t n_tokens, const void *q,
                                  const void *k_fresh, const void *v_fresh,
                                  const void *k_cache, const void *v_cache,
                                  const void *h_fresh, const float *lse,
                                  const uint8_t *reused, float scale,
                                  float *impact_v, float *impact_k, float *impact_kv,
                                  void *workspace, size_t workspace_bytes, void *stream);

/*
 * Token-sequence matching of the KV Retriever (Sec. 5.1; App. E Alg. 3 with the polynomial window
 * hash of Eq. (7)): which tokens of a new request (the target) also stand, in stretches that start
 * with a whole window of `window` equal-hash tokens, in an earlier request (the candidate), and where.
 * The result is the one the algorithm's sequential scan produces: a target position is matched once,
 * by the first pair of window starts (candidate window ascending, then target window ascending)
 * whose stretch of equal tokens reaches it; windows are compared by hash only, then token by
 * token, so two different windows with one hash contribute the equal tokens they begin with.
 * The paper names neither the base, the modulus nor the window: all three are arguments.
 *
 * target, candidate [dev] int32 token ids, non-negative (an id is hashed as an unsigned 32-bit number)
 * window            > 0; sequences shorter than the window match nothing
 * hash_base         b of Eq. (7), any 32-bit value
 * hash_modulus      m of Eq. (7), 1 .. 2^32-1
 * match_cand        [dev] int32[n_target] out: candidate position matched to each target position, -1: none
 * target_matches, candidate_matches
 *                   [dev] int32[n_target] out, each may be NULL: the matched pairs in the algorithm's
 *                   order of discovery (its two output lists); entries from *n_matches on are not written
 * n_matches         [dev] int64 out: number of matched target positions (hit rate = n_matches / n_target)
 * workspace         [dev] kvs_workspace_size("match_tokens", NULL, 1, n_target, n_candidate) bytes,
 *                   256-byte aligned (not needed when a sequence is shorter than the window)
 * Up to 2^26 tokens per sequence.  Integer work: the outputs are exact and do not depend on the
 * order in which the device's atomics arrive.  Five launches, no host synchronisation.  Cost grows
 * with the matched tokens, except for degenerate inputs (one token repeated throughout both
 * sequences makes every pair of windows a candidate: n_target x n_candidate steps).
 * Several earlier requests are matched in one call by concatenating them into one candidate with a token id
 * that occurs nowhere else between them (no window then spans two requests); partners index the concatenation.
 * The scheduler of Sec. 4.3 Alg. 2 needs no call of its own: the batch it sends on is
 * kvs_select_topk over the requests' hit rates (ties to the request that arrived first).
 */
KVS_API kvs_status kvs_match_tokens(const int32_t *target, int64_t n_target,
                                    const int32_t *candidate, int64_t n_candidate,
                                    int32_t window, uint32_t hash_base, uint32_t hash_modulus,
                                    int32_t *match_cand, int32_t *target_matches, int32_t *candidate_matches,
                                    int64_t *n_matches, void *workspace, size_t workspace_bytes, void *stream);

/*
 * A later layer's Q, K and V of the selected tokens (App. D.1: the tokens picked in an early layer are
 * the ones recomputed in the layers after it; their index list is simply passed on to this call,
 * kvs_scatter_kv and kvs_partial_attention of those layers).  Recomputing a token in a layer starts with
 * the layer's projection of its hidden state:
 *     y[m, f] = sum_c x[x_rows[m], c] * w_qkv[f, c],   f over (n_q_heads + 2 n_kv_heads) * head_dim features
 * in the order all Q heads, all K heads, all V heads.  With a rotary table, channel pair
 * (c, c + head_dim/2) of every Q and K head is turned by the table's angle for position sel_pos[m]:
 *     out[c] = y[c] cos - y[c + head_dim/2] sin,   out[c + head_dim/2] = y[c + head_dim/2] cos + y[c] sin
 * (the convention of the Llama / Qwen / Yi families the paper evaluates; the paper itself takes Q, K, V
 * as given).  One launch: gather, bf16 matrix product with fp32 accumulation, rotation in fp32, one
 * rounding to bf16 on the way out.
 *
 * x        [dev] bf16 [n_tokens, hidden] hidden states
 * x_rows   [dev] int32[n_sel] row of x for each selected token, or NULL (row m of x is selected token m:
 *          from the second recomputed layer on only the selected tokens have hidden states)
 * sel_pos  [dev] int32[n_sel] positions of the selected tokens (read only with a rotary table)
 * w_qkv    [dev] bf16 [(n_q_heads + 2 n_kv_heads) * head_dim, hidden], one row per output feature
 * rope     [dev] fp32 [rope_positions, head_dim/2, 2] = (cos, sin) per position and channel pair, or NULL
 * q_out    [dev] bf16 [n_sel, n_q_heads, head_dim]; k_out, v_out [dev] bf16 [n_sel, n_kv_heads, head_dim]:
 *          the layouts kvs_partial_attention and kvs_scatter_kv take
 * Built for bf16, head_dim 128, hidden a multiple of 64, an even number of heads in all, x and w below
 * 4 GiB each, a rotary table below 4 GiB (KVS_EUNSUPPORTED otherwise).  Tensors 16-byte aligned.  No workspace.  Row indices and
 * positions outside their ranges are clamped (memory safety only).
 */
KVS_API kvs_status kvs_project_qkv(const kvs_shape *shape, int32_t hidden, const void *x, int64_t n_tokens,
                                   const int32_t *x_rows, const int32_t *sel_pos, int64_t n_sel,
                                   const void *w_qkv, const float *rope, int64_t rope_positions,
                                   void *q_out, void *k_out, void *v_out, void *stream);

/*
 * kvs_rotary -- rotary positions of Q and K rows: what a layer applies to fresh rows, and what a reused key needs when it
 * takes another position in the new request than it had in the one it was computed for (its K then has to be turned by the
 * difference; V carries no position).
 *
 * The first rotary_dim channels of every head form rotary_dim/2 pairs, pair j = channels (j, j + rotary_dim/2) in the
 * KVS_ROTARY_HALF layout and (2j, 2j + 1) in the KVS_ROTARY_INTERLEAVED one; the other channels pass through.  With
 * a = (pos[i] - pos_from[i]) * f_j a pair (u, v) of row i becomes
 *     magnitude * (u cos a - v sin a),   magnitude * (v cos a + u sin a)
 * in fp32, rounded once.  Angles are formed in fp64 (a position of 10^6 keeps them to 1e-7).  f_j, before scaling, is
 * base^(-2j / rotary_dim); the scalings for contexts longer than `original`, the length that a model was trained on, are
 *     KVS_ROTARY_PLAIN       f_j
 *     KVS_ROTARY_LINEAR      f_j / factor                         (position interpolation)
 *     KVS_ROTARY_NTK         base * factor^(rotary_dim / (rotary_dim - 2)) in place of base; rotary_dim > 2
 *     KVS_ROTARY_RAMP        f_j (1 - w) + f_j / factor * w, w rising from 0 to 1 over the pairs from floor(at(high)), at least 0,
 *                            to ceil(at(low)), at most rotary_dim - 1, at(t) = rotary_dim * ln(original / (2 pi t)) / (2 ln base): pairs that turn more
 *                            than `high` times within the original length keep their frequency, those under `low` turns are
 *                            interpolated (YaRN, arXiv 2309.00071; its magnitude 0.1 ln(factor) + 1 is the caller's)
 *     KVS_ROTARY_WAVELENGTH  f_j w + f_j / factor * (1 - w), w rising from 0 to 1 with the turns original * f_j / (2 pi)
 *                            from `low` to `high`
 * factor, original, low and high are only read by the scalings that use them (0 < low < high).  A magnitude other than 1
 * belongs to fresh rows: moved ones have it already.
 *
 * n_tokens        rows; 0 is allowed
 * pos             [dev] int32[n_tokens], any value        pos_from [dev] int32[n_tokens] or NULL (0: fresh rows)
 * q, q_out        [dev] n_tokens rows of n_q_heads * head_dim elements, q_stride and q_out_stride elements apart, each at
 *                 least a row long and a multiple of 16 bytes: a slice of a fused projection's buffer will do
 * k, k_out        the same with n_kv_heads.  q or k may be NULL (with its output), not both; up to 4095 heads together
 * In place (the same pointer and stride) is allowed; an output may not overlap an input or output in any other way.  Rows may lie
 * beside each other in one buffer, slices of its columns, where their strides are the same; rows of another stride between a buffer's first
 * and last are refused.
 */
typedef enum { KVS_ROTARY_HALF = 0, KVS_ROTARY_INTERLEAVED = 1 } kvs_rotary_layout;
typedef enum {
    KVS_ROTARY_PLAIN = 0, KVS_ROTARY_LINEAR = 1, KVS_ROTARY_NTK = 2, KVS_ROTARY_RAMP = 3, KVS_ROTARY_WAVELENGTH = 4
} kvs_rotary_scaling;

typedef struct {
    int32_t rotary_dim; /* channels of a head that are turned: even, 2 .. head_dim */
    int32_t layout;     /* kvs_rotary_layout */
    int32_t scaling;    /* kvs_rotary_scaling */
    int32_t original;   /* context length that the unscaled frequencies belong to */
    double base;        /* > 1 */
    double factor;      /* > 0 */
    double low, high;   /* turns */
    double magnitude;
} kvs_rotary_spec;

KVS_API kvs_status kvs_rotary(const kvs_shape *shape, const kvs_rotary_spec *spec, int64_t n_tokens,
                              const int32_t *pos, const int32_t *pos_from,
                              const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                              void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, void *stream);

/*
 * A KV cache held in 8 bits, with a scale for each block of tokens and KV head.  K and V are kept apart: element c of
 * row i and head g stands for  code[i, g, c] * scale[i / block, g].  Blocks are counted over the cache's rows, so
 * requests that begin with a block of their own share no scale with another request.  No scale is negative.  A scale of 0
 * marks a block that holds nothing but zeros (whatever its codes): set the scales of a block to 0 before its first use and
 * before another request takes it over.  A scale that is NaN marks a block that a NaN or infinity was stored into: rows that
 * see one of its keys become NaN, their log-sum-exps too, no others.
 *
 * KVS_E4M3 codes are OCP 8-bit floats with 3 mantissa bits (largest 448), KVS_INT8 codes whole numbers from -127 to 127.
 * A store writes no other codes; e4m3's two NaN codes, where memory that was never stored to holds them, do not reach
 * rows that do not see their key.
 *
 * Everything else stays in the shape's dtype (Q, outputs, rows to store, fresh rows), bf16 or fp32.  head_dim 64 or 128,
 * up to 64 KV heads.
 */
typedef enum { KVS_E4M3 = 0, KVS_INT8 = 1 } kvs_code;

typedef struct {
    void *k, *v;             /* [dev] [n_rows, n_kv_heads, head_dim] codes, one byte each, 16-byte aligned */
    float *k_scale, *v_scale; /* [dev] fp32 [(n_rows + block - 1) / block, n_kv_heads] */
    int64_t n_rows;
    int32_t block;           /* 16, 32, 64 or 128 tokens */
    int32_t code;            /* kvs_code */
} kvs_cache8;

/*
 * kvs_store_kv8 -- the KV Writer (App. A) for a cache in 8 bits: a prompt's rows, a decode step's new ones, or recomputed
 * rows in place of reused ones.
 *
 * sel_pos == NULL  row row0 + s takes k_new[s], v_new[s]           for s in [0, n_sel)
 * sel_pos != NULL  row sel_pos[s] takes them (row0 is not read).  Entries outside [0, n_rows) are skipped, wherever they stand (the
 *                  places of a padded batch that hold no token).  The others of one block have to stand together in the list: an
 *                  ascending list does that, and one that keeps every request's rows together in any order of the
 *                  requests if no two requests share a block (requests that do are stored in ascending order of their
 *                  rows, or by a call each).  The call cannot see a list that breaks this: the codes and scales of a block
 *                  whose entries stand apart are then not to be used.  Inside a block any order goes, and of equal
 *                  entries the last one counts.
 *
 * For each block that takes a row, each KV head, K and V apart, with top = 448 (KVS_E4M3) or 127 (KVS_INT8), in fp32:
 *     need  = max |x| over the rows that the block takes * (1 / top), at least 2^-126 (0 if they are all zero)
 *     scale = max(need, old scale), or need alone if all of the block's rows in the cache are taken
 *     code  = nearest code (ties to even) to x * (1 / scale)      for the rows taken
 *     code  = nearest code to code * (old scale / scale)          for the other rows, where the scale has changed
 * Kept rows are therefore rounded again only when a larger value comes into their block, by half a step at most each time: a block of
 * normal values that is filled a row at a time ends 1.1 to 1.4 times as far from its rows, in norm, as one stored at once (2 to 5
 * growths), one whose rows grow 17-fold over it 2.4 times (28).  If one of the rows taken holds a NaN or infinity, or a row is kept
 * and the old scale is NaN, the scale becomes NaN.
 *
 * k_new, v_new  [dev] [n_sel, n_kv_heads, head_dim] in the shape's dtype
 * reused, dev_v [dev] uint8[n_rows], fp32[n_kv_heads, n_rows], each may be NULL: cleared for the rows taken, as in
 *               kvs_scatter_kv
 * Nothing is accumulated out of order: the result does not depend on timing.  Calls on one cache that could touch the
 * same block have to be ordered (one stream, or events).
 */
KVS_API kvs_status kvs_store_kv8(const kvs_shape *shape, const kvs_cache8 *cache, const void *k_new, const void *v_new,
                                 const int32_t *sel_pos, int64_t row0, int64_t n_sel,
                                 uint8_t *reused, float *dev_v, void *stream);

/*
 * kvs_deviation_kv8 -- kvs_deviation against a cache in 8 bits: what the cache rows row0 .. row0 + n_tokens - 1 stand for
 * against freshly computed rows.
 *
 *   dev_v[g,i] = sum_c | v_fresh[i,g,c] - v_code[row0+i,g,c] * v_scale[(row0+i) / block, g] |,   dev_k likewise
 *
 * score, alpha, reused and mode as in kvs_deviation, all of n_tokens entries: scores go on to kvs_select_topk.  k_fresh
 * may be NULL in mode KVS_SCORE_V with dev_k == NULL.  fp32 in a fixed order (bit-reproducible).
 */
KVS_API kvs_status kvs_deviation_kv8(const kvs_shape *shape, const kvs_cache8 *cache, int64_t row0, int64_t n_tokens,
                                     const void *k_fresh, const void *v_fresh,
                                     const uint8_t *reused, const float *alpha, int32_t mode,
                                     float *dev_k, float *dev_v, float *score, void *stream);

/*
 * kvs_attention_kv8 -- kvs_partial_attention over a cache in 8 bits; a decode step is the call with one selected token a
 * request, at position ctx_len - 1.
 *
 * Request b owns cache rows [ctx_off[b], ctx_off[b] + ctx_len[b]) and the selected tokens [cu_sel[b], cu_sel[b+1]); token
 * s at request-local position p = sel_pos[s] sees its request's rows 0 .. p.  A negative position sees nothing (a place
 * of a padded batch that holds no token): its out rows are 0 and its lse -inf; a position past the context sees all of
 * it.  Positions may come in any order (ascending is fastest); contexts may overlap, begin anywhere in a block, and lie
 * inside [0, n_rows).
 *
 * q_sel, out [dev] [n_sel, n_q_heads, head_dim]      lse_out [dev] fp32[n_sel, n_q_heads] or NULL (natural log)
 * scale      any finite number
 * workspace  [dev] optional (NULL / 0 is valid), 256-byte aligned, kvs_workspace_size("attention_kv8", shape, batch, rows, n_sel)
 *            bytes, rows being those of its contexts together, or the cache's if they are fewer.  Launches that would leave units
 *            idle cut their key ranges into pieces and merge them.
 *            Launches of so many rows that it pays (bf16, head_dim 128, scale > 0, contexts that begin at multiples of
 *            16 rows) widen the rows that their contexts hold to bf16 in it, once where contexts share them, 4 bytes an
 *            element of K, and go on as kvs_partial_attention; the size asked for has room for that from 7373 rows (tokens
 *            times query heads) on; what a key adds to an output there is lost below 2^-65.  Less workspace means fewer pieces and no
 *            widening.  One call's until that call has ended on its stream.
 * Codes enter the matrix cores as the bf16 numbers that they are, exactly; K's scales multiply the scores in fp32.
 * bf16: softmax weights enter the second product times V's scales, as two bf16 numbers that hold 16 of their bits where no
 * request has more than 32 rows a KV head (tokens times the query heads that share it), rounded to one elsewhere.
 * fp32: Q and these products enter as three bf16 numbers each, which together hold all their bits, and everything else is
 * fp32.  Sums of values beyond 2^110 may become infinite; in bf16 launches of many rows beyond 2^27, and values below 2^-60 may lose bits.
 */
KVS_API kvs_status kvs_attention_kv8(const kvs_shape *shape, const kvs_cache8 *cache, int32_t batch,
                                     const int64_t *ctx_off, const int64_t *ctx_len, const int64_t *cu_sel,
                                     const void *q_sel, const int32_t *sel_pos, float scale,
                                     void *out, float *lse_out,
                                     void *workspace, size_t workspace_bytes, void *stream);

/*
 * A KV cache in pages.  The pool holds n_pages pages of `page` rows; row i of request b is row i % page of page
 * table[b, i / page].  A page is laid out as the rows of the other calls are, so the pool is also a cache of n_pages * page rows
 * that kvs_scatter_kv and the others take.  Requests may share pages (a prefix, or whatever else was reused).
 *
 * The page table and the lengths are read on the device, when the kernels run: a captured call can be replayed after they have
 * changed.  max_ctx is what the host promises about them: no context is longer.  Launches are sized by it, so it should not be
 * far above; of a longer context the first max_ctx rows are taken, and of one longer than the table is wide what the table
 * names (its last tokens then stand behind those: they overwrite no row, and see what the last one taken sees).  A negative length is 0.  An entry of the table outside [0, n_pages) names no page: its rows are not stored to, seen or
 * copied.  Entries behind a context's last page are not used.
 *
 * Tokens of a call belong to the requests in order: those of request b are [cu_new[b], cu_new[b+1]) (device memory, at
 * least 0, non-decreasing, at most n_new; offsets that break this give unspecified results, and no access outside the tensors).
 * Tokens outside [cu_new[0], cu_new[batch]) belong to none: nothing of theirs is written, and what their rows hold reaches nothing (the rows
 * may be read), so a captured call may hold more places than tokens.  cu_new == NULL: one token a request (n_new == batch).  Token i of a request's n stands at position
 * sel_pos[cu_new[b] + i], or, with sel_pos == NULL, at ctx_len[b] - n + i: the context's last rows.  A negative position sees
 * nothing; one behind the context sees what its last row sees.
 *
 * Everything is in the shape's dtype, bf16 or fp32; head_dim 64 or 128, up to 64 KV heads and 4096 query heads.
 */
typedef struct {
    void *k, *v;            /* [dev] [n_pages, page, n_kv_heads, head_dim], 16-byte aligned */
    int64_t n_pages;
    int32_t page;           /* 16, 32, 64, 128 or 256 rows */
} kvs_paged_cache;

typedef struct {
    const int32_t *table;   /* [dev] [batch, width] page ids */
    const int32_t *ctx_len; /* [dev] [batch] rows of each request, new tokens' among them */
    int64_t max_ctx;
    int32_t batch, width;
} kvs_page_table;

/*
 * kvs_store_paged -- rows of K and V into the pages of their requests: a chunk of a prompt, a decode step's new rows, or
 * recomputed rows in place of reused ones.
 *
 * Token s goes to its position (above); tokens whose position is negative or behind the context are skipped.  Where neighbouring
 * tokens of a request have the same position the last one counts (an ascending list may repeat itself); the same position further
 * apart, and one row of the pool reached through two requests, are a race.
 *
 * k_new, v_new [dev] [n_new, n_kv_heads, head_dim], not in the cache
 * mass         [dev] fp32 [batch, n_kv_heads, mass_stride] or NULL: set to 0 at the positions stored to (kvs_mass_paged;
 *              mass_stride at least max_ctx).  No overlap
 */
KVS_API kvs_status kvs_store_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages,
                                   const int32_t *cu_new, const int32_t *sel_pos, int64_t n_new,
                                   const void *k_new, const void *v_new, float *mass, int64_t mass_stride, void *stream);

/*
 * kvs_attention_paged -- kvs_partial_attention over a cache in pages: a chunk of new tokens, selected ones, or a decode
 * step's single ones, all in one call if they come together.
 *
 * The row of a token at position p sees row i of its request if i <= p and (window == 0 or i > p - window or i < n_first): all
 * that is before it, or a window that ends with it beside the first n_first rows.  Rows that a window leaves out are not read.
 *   out[s,h,:] = sum_i softmax_i( scale * q_new[s,h,:] . K[i, g(h), :] ) * V[i, g(h), :]
 *   lse[s,h]   = log sum_i exp( scale * q . K_i )                 (natural log; optional)
 * A token that sees nothing gets 0 and -inf.  What a row does not see does not reach it, whatever it holds (NaN and
 * infinities too).
 *
 * q_new, out [dev] [n_new, n_q_heads, head_dim]      lse_out [dev] fp32[n_new, n_q_heads] or NULL      no overlap
 * scale      any number up to 2^127 in magnitude
 * workspace  [dev] optional (NULL / 0 is valid), 256-byte aligned, kvs_workspace_size("attention_paged", shape, batch,
 *            max_ctx, n_new) bytes: launches that would leave units idle cut their key ranges into pieces and merge them, and those
 *            of many tokens go to a kernel of larger tiles.  Less means fewer pieces and smaller tiles.  One call's until that
 *            call has ended on its stream.
 * bf16: fp32 accumulation and softmax; the weights enter the second product as two bf16 numbers that hold 16 of their bits where
 * there are no more than 32 rows (tokens times query heads of a KV head) a request on average, rounded to one elsewhere.  fp32
 * throughout otherwise.  Sums of values beyond 2^110 may become infinite, values below 2^-100 may lose bits.  Equal calls give equal bits.
 */
KVS_API kvs_status kvs_attention_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages,
                                       const int32_t *cu_new, const int32_t *sel_pos, int64_t n_new, const void *q_new, float scale,
                                       int32_t window, int32_t n_first, void *out, float *lse_out,
                                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * kvs_mass_paged -- the attention that every cached row receives, added up over calls: what Alg. 1 takes as alpha
 * (kvs_attn_colsum), for a cache that is filled in chunks and read by decode steps.
 *
 *   mass_out[b,g,i] = decay * mass[b,g,i] + sum over the tokens s of request b that see row i (window and n_first as above) and the
 *                     query heads h of KV head g of exp( scale * q_new[s,h,:] . K[i,g,:] - lse[s,h] )
 *
 * for every row i of the contexts; entries behind them stay as they are.  lse is what kvs_attention_paged has given for the
 * same tokens: then every token adds 1 for each query head, spread over the rows it saw.
 *
 * lse            [dev] fp32[n_new, n_q_heads]
 * decay          finite, at least 0
 * mass, mass_out [dev] fp32 [batch, n_kv_heads, mass_stride], mass_stride at least max_ctx.  mass may be mass_out, or NULL (zeros);
 *                mass_out may not overlap it otherwise, nor anything else that is read
 * workspace      [dev] optional, 256-byte aligned, kvs_workspace_size("mass_paged", shape, batch, max_ctx, n_new) bytes:
 *                chunks over short contexts cut their rows into pieces and add them up
 * fp32 sums in a fixed order (bit-reproducible for equal workspaces); bf16 products are accumulated in fp32.
 */
KVS_API kvs_status kvs_mass_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages,
                                  const int32_t *cu_new, const int32_t *sel_pos, int64_t n_new, const void *q_new, const float *lse, float scale,
                                  int32_t window, int32_t n_first, float decay, const float *mass, float *mass_out, int64_t mass_stride,
                                  void *workspace, size_t workspace_bytes, void *stream);

/*
 * kvs_evict_paged -- contexts that have grown too long, cut down to the rows that received most attention.
 *
 * Request b keeps m = min(ctx_len[b], keep[b], max_keep) rows (none for a negative keep[b]):
 *   the first f = min(n_first, m), the last r = min(n_recent, m - f), and of the others the m - f - r with the largest
 *   mass[b,0,i] + mass[b,1,i] + ... (fp32, in the order of the KV heads), ties to the lower index; NaN ranks below all numbers, -0 equals 0.
 * They are copied, in order, to the pages of new_table: row j of them to row j % page of page new_table[b, j / page].  Pages that
 * requests share stay as they are: a request takes pages of its own for what it keeps, and gives back its old ones.  The two
 * tables' pages in use may not overlap (rows would be overwritten before they are read).  The rest of a last page stays as it was.
 *
 * keep      [dev] int32[batch]
 * max_keep  what the host promises about keep, as max_ctx
 * mass      [dev] fp32 [batch, n_kv_heads, mass_stride], mass_stride at least max_ctx
 * new_table [dev] int32[batch, new_width], new_width pages holding at least max_keep rows; NULL: nothing is copied.  Entries outside
 *           [0, n_pages) take nothing
 * kept      [dev] int32[batch, max_keep] or NULL: the kept rows' positions, ascending; entries from m on stay as they are
 * new_len   [dev] int32[batch] or NULL: m.  May be ctx_len
 * new_mass  [dev] fp32 [batch, n_kv_heads, max_keep] or NULL: the kept rows' mass; entries from m on stay as they are.  Nothing that is written
 *           may overlap anything else
 * workspace [dev] kvs_workspace_size("evict_paged", shape, batch, max_ctx, 0) bytes, 256-byte aligned, required
 * Exact and deterministic.
 */
KVS_API kvs_status kvs_evict_paged(const kvs_shape *shape, const kvs_paged_cache *cache, const kvs_page_table *pages,
                                   const int32_t *keep, int64_t max_keep, int32_t n_first, int32_t n_recent, const float *mass, int64_t mass_stride,
                                   const int32_t *new_table, int32_t new_width, int32_t *kept, int32_t *new_len, float *new_mass,
                                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * Workspace a call needs, in bytes, for the given problem.  `call` is "select_topk",
 * "partial_attention", "decode_check", "attn_colsum", "first_order_impact", "match_tokens", "attention_kv8", "attention_paged", "mass_paged" or
 * "evict_paged" (anything else returns 0).  n_rows_total is the total number of score / cache rows the call will see (match_tokens: the
 * target's tokens), n_sel_total the total number of selected tokens (partial_attention, attention_kv8) or the candidate's
 * tokens (match_tokens, which ignores shape: it may be NULL there).  The paged calls take max_ctx as n_rows_total and n_new as n_sel_total.  The answer is an upper bound valid for any split of the
 * totals over `batch` requests, and does not shrink as the totals grow.
 */
KVS_API size_t kvs_workspace_size(const char *call, const kvs_shape *shape, int32_t batch,
                          int64_t n_rows_total, int64_t n_sel_total);

KVS_API const char *kvs_strerror(kvs_status status);
KVS_API const char *kvs_last_error(void);

/* Library build identification: "kvshare-hip gfx950 <n>" */
KVS_API const char *kvs_version(void);

#ifdef __cplusplus
}
#endif
#endif /* KVS_H */
