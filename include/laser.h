/*
 * laser.h - C ABI of the MI355X (gfx950) implementation of LASER's hot path
 * (arxiv 2602.11562): Segmented Target Attention (STA) over a long per-user
 * behaviour history, then Global Stacked Target Attention (GSTA) over the
 * compressed segments.
 *
 * Problem statement (paper Sec. 3.1, generalised from one target item to the C
 * candidates a ranking request scores for one user): a user u has a history of
 * up to L items; item j carries a key K[u,j,:] in R^{d_q} and a value V[u,j,:]
 * in R^{d} (K = H W_k, V = H W_v, already projected); candidate c carries a
 * query Q[u,c,:] in R^{d_q} (Q = t W_q) and a target vector t[u,c,:] in R^{d}.
 *
 * Conventions for every entry point
 *   - Every data pointer is a DEVICE pointer (HBM), caller-owned, row-major,
 *     contiguous, 16-byte aligned. Nothing is copied to or from the host.
 *   - The library allocates nothing, keeps no state and never synchronises: work
 *     is enqueued on `stream` (a hipStream_t; NULL = the default stream). (One exception
 *     to "no state": laser_sta_backward_static owns a fixed scratch array per GPU.)
 *   - Outputs are overwritten in full, including exact zeros for empty segments.
 *   - Return value only; no exception or abort crosses the ABI. Arguments are
 *     validated on the host before anything is launched, so an error return means
 *     no kernel ran. `lens` is device data and cannot be checked on the host: each
 *     value is clamped to [0, L] on the device.
 *   - dtype `dt` is the storage type of q, k, v, t0, the GSTA weights and H'
 *     (LASER_F32 or LASER_BF16). Arithmetic accumulates in fp32. z is always fp32.
 *   - Segment i covers items [i*w, min((i+1)*w, L)); S = ceil(L / w).
 *     Item j of user u is valid iff j < lens[u]. Padded rows are never multiplied
 *     in, so they may hold anything, including NaN or Inf.
 */
#ifndef LASER_H_
#define LASER_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LASER_OK = 0,
  LASER_ERR_NULL = 1,        /* a required pointer is NULL                       */
  LASER_ERR_SHAPE = 2,       /* a size is <= 0, too large, or inconsistent       */
  LASER_ERR_DTYPE = 3,       /* dt is not a laser_dtype                          */
  LASER_ERR_UNSUPPORTED = 4, /* valid request that no kernel here implements     */
  LASER_ERR_LAUNCH = 5,      /* the HIP runtime refused a launch                 */
  LASER_ERR_ALIGN = 6,       /* a pointer is not 16-byte aligned                 */
  LASER_STATUS_ANY_INT = 0x7fffffff
} laser_status;

/* (The *_ANY_INT members below name no value of their own: they make every non-negative int a representable value of
 * the enumeration, so that a caller's out-of-range number reaches the library's own check, which answers with
 * LASER_ERR_DTYPE or LASER_ERR_UNSUPPORTED, instead of being undefined behaviour at the call.) */
typedef enum { LASER_F32 = 0, LASER_BF16 = 1, LASER_DTYPE_ANY_INT = 0x7fffffff } laser_dtype;

/* Which STA kernel runs. AUTO picks by (dt, C, d_q, d, w); the others force one
 * and return LASER_ERR_UNSUPPORTED when the shape is outside that kernel's range. */
typedef enum {
  LASER_STA_AUTO = 0,
  LASER_STA_GENERIC = 1, /* fp32 FMA, any shape, either dtype                        */
  LASER_STA_MFMA = 2,    /* bf16 MFMA, many candidates per user                      */
  LASER_STA_STREAM = 3,  /* bf16, few candidates per user, HBM streaming             */
  LASER_STA_MFMA_CACHED = 4, /* LASER_STA_MFMA with H' stored cacheable instead of with the non-temporal hint: for a
                              * caller whose next launch reads H' back (this is the form laser_forward launches) */
  LASER_STA_VARIANT_ANY_INT = 0x7fffffff
} laser_sta_variant;

/* Which GSTA kernel runs. */
typedef enum {
  LASER_GSTA_AUTO = 0,
  LASER_GSTA_GENERIC = 1, /* fp32 FMA, one workgroup per pair, any shape              */
  LASER_GSTA_TILED = 2,   /* bf16 storage, d in {64, 128}: 1 to 16 pairs per workgroup, MFMA, any M and S */
  LASER_GSTA_SPLIT = 3,   /* bf16 storage, M = 1: projection / streaming / output kernels; z_out is the scratch */
  LASER_GSTA_ONE = 4,     /* bf16 storage, M = 1: the same three steps in one launch, 32 pairs per workgroup */
  LASER_GSTA_VARIANT_ANY_INT = 0x7fffffff
} laser_gsta_variant;

/*
 * Segmented Target Attention, forward (paper Sec. 3.4.2, the STA equation
 *   s_i = Sigmoid(Q K_i^T / gamma) V_i,
 * in the "global scores, then per-segment aggregation" form of Sec. 3.5.1):
 *   seg_out[u,c,i,:] = sum over valid j in segment i of
 *                      sigmoid(dot(q[u,c,:], k[u,j,:]) / gamma) * v[u,j,:]
 *   seg_cnt[u,i]     = number of valid items in segment i
 *
 *   q       [U,C,d_q]  candidate queries
 *   k       [U,L,d_q]  history keys
 *   v       [U,L,d]    history values
 *   lens    [U] int32  valid lengths; NULL means every user has L valid items
 *   gamma   score scale (> 0); the paper leaves its value open
 *   seg_out [U,C,S,d]  H', dtype dt (fp32 sums rounded once to dt)
 *   seg_cnt [U,S] int32, may be NULL
 * Limits: U,C,L,d_q,d,w >= 1; d_q, d <= 1024 and multiples of 8; every tensor < 2^31 elements.
 */
laser_status laser_sta_forward(const void* q, const void* k, const void* v, const int32_t* lens,
                               int U, int C, int L, int d_q, int d, int w, float gamma, laser_dtype dt,
                               void* seg_out, int32_t* seg_cnt, void* stream);

/* Same operation with the kernel chosen by the caller (tests and benchmarks). */
laser_status laser_sta_forward_variant(const void* q, const void* k, const void* v, const int32_t* lens,
                                       int U, int C, int L, int d_q, int d, int w, float gamma, laser_dtype dt,
                                       void* seg_out, int32_t* seg_cnt, void* stream, laser_sta_variant variant);

/*
 * STA with several attention heads (paper Sec. 4.1.2 runs the compression module with 2 heads, d_q = 16 per head, and
 * a value width equal to the embedding width). The paper gives the head count and the widths only; here, as in
 * multi-head attention, head h owns columns [h d_q/heads, (h+1) d_q/heads) of q and k and columns
 * [h d/heads, (h+1) d/heads) of v and seg_out: every head is the STA above on its own columns, with the same gamma,
 * and the heads' outputs lie side by side, so all shapes and layouts are those of laser_sta_forward. heads = 1 is
 * laser_sta_forward_variant. heads must divide d_q and d (1 <= heads <= 64), else LASER_ERR_SHAPE. The streaming
 * kernel takes 1 or 2 heads (d_q/heads and d/heads multiples of 8); the matrix-core kernel takes 1, 2 or 4 heads (d_q / heads a multiple of 16, d / heads of 32); other
 * cases run on the generic kernel (AUTO picks; a forced variant that does not take the case returns
 * LASER_ERR_UNSUPPORTED). Everything else as for laser_sta_forward.
 */
laser_status laser_sta_forward_heads(const void* q, const void* k, const void* v, const int32_t* lens,
                                     int U, int C, int L, int d_q, int d, int w, float gamma, int heads,
                                     laser_dtype dt, void* seg_out, int32_t* seg_cnt, void* stream,
                                     laser_sta_variant variant);

/*
 * The ablation variant of paper Sec. 4.4.1 / Table 4, STA with a softmax over the items in the place of its sigmoid
 * gates:  seg_out[u,c,i,:] = sum_j softmax_j(dot(q[u,c,:], k[u,j,:]) / gamma) * v[u,j,:], the softmax taken over the
 * valid items j of segment i (per head on the head's own columns, as in laser_sta_forward_heads); segments without a
 * valid item give zeros. Arguments, layouts, limits and errors as for laser_sta_forward_heads. Kernels: the streaming
 * kernel for short segments (C <= 8, bf16, w below one step of its long form), the matrix-core kernel (C >= 9, bf16,
 * 1, 2 or 4 heads, its usual widths) and the generic kernel; the long-segment streaming kernel carries sigmoid gates only
 * (a forced variant that does not take the case returns LASER_ERR_UNSUPPORTED).
 */
laser_status laser_sta_forward_softmax(const void* q, const void* k, const void* v, const int32_t* lens,
                                       int U, int C, int L, int d_q, int d, int w, float gamma, int heads,
                                       laser_dtype dt, void* seg_out, int32_t* seg_cnt, void* stream,
                                       laser_sta_variant variant);

/*
 * Global Stacked Target Attention, forward (paper Sec. 3.4.3): for l = 1..M
 *   a_l = softmax((t_{l-1} W_q^l)(H' W_k^l)^T / sqrt(d)),  o_l = a_l (H' W_v^l),  t_l = t_{l-1} + o_l
 * with t_0 = t0 and z = t_M. The softmax runs over the segments of user u that hold at
 * least one valid item (the first ceil(lens[u] / w)); with none, z = t0.
 *
 *   seg   [U,C,S,d]  H' (dtype dt), S = ceil(L / w)
 *   t0    [U,C,d]    target vectors (dtype dt)
 *   wq, wk, wv [M,d,d] each (dtype dt), applied as y = x W (row vector times matrix)
 *   lens  [U] int32 or NULL (all L)
 *   z_out [U,C,d] fp32
 * Limits: d <= 1024 and a multiple of 8; S <= 4096; M >= 1.
 */
laser_status laser_gsta_forward(const void* seg, const void* t0, const void* wq, const void* wk, const void* wv,
                                const int32_t* lens, int U, int C, int L, int d, int w, int M, laser_dtype dt,
                                float* z_out, void* stream);

laser_status laser_gsta_forward_variant(const void* seg, const void* t0, const void* wq, const void* wk,
                                        const void* wv, const int32_t* lens, int U, int C, int L, int d, int w,
                                        int M, laser_dtype dt, float* z_out, void* stream,
                                        laser_gsta_variant variant);

/*
 * The whole path: STA, then GSTA on the segment vectors it produced (paper Sec. 3.2,
 * "compress-then-refine"; the per-segment FFN + LayerNorm of Sec. 3.4.2 is not applied,
 * which is the paper's "-FFN+LayerNorm" ablation variant). Arguments as above; seg_cnt may be NULL.
 * seg_out [U,C,S,d] is the buffer GSTA reads: GSTA consumes H' as stored there, i.e. after rounding to dt.
 * seg_out may be NULL when H' is not wanted (M = 1 only; M > 1 returns LASER_ERR_UNSUPPORTED, because every further
 * layer reads every segment vector again): the call is then laser_forward_fused below without a work buffer, i.e.
 * one launch in which every workgroup walks a whole history and nothing but z_out (and seg_cnt) is written.
 */
laser_status laser_forward(const void* q, const void* k, const void* v, const void* t0,
                           const void* wq, const void* wk, const void* wv, const int32_t* lens,
                           int U, int C, int L, int d_q, int d, int w, float gamma, int M, laser_dtype dt,
                           void* seg_out, int32_t* seg_cnt, float* z_out, void* stream);

/*
 * The whole path with one GSTA layer and H' never stored (paper Sec. 3.4.2 and 3.4.3): the attention of Sec. 3.4.3,
 *   a = softmax((t0 W_q)(H' W_k)^T / sqrt(d)),  z = t0 + a (H' W_v),
 * is applied to each segment vector while it is still in registers, as an online softmax over the segments (running
 * maximum, denominator and weighted sum per pair), with the products re-associated (H' (W_k (t0 W_q)^T) and (a H') W_v:
 * exact). Same arguments, layouts, masks and limits as laser_forward with M = 1 (wq, wk, wv [d,d]); the segment vectors
 * enter the layer as fp32 sums, not rounded to dt, so z_out agrees with laser_forward's within the tolerance, not bit
 * for bit. seg_cnt [U,S] may be NULL.
 * work: with few users a history must be cut into runs of segments that different workgroups walk, and each run
 * leaves a partial result (maximum, denominator, weighted sum) per pair that a second, small launch merges in run
 * order (fixed order: results are reproducible). work is caller-owned device scratch for those partial results, 16-byte
 * aligned, at least laser_forward_fused_work_bytes(...) bytes (contents unspecified on return; 0 bytes are needed when
 * there are enough users to fill the machine, or when no kernel here cuts histories for the shape). work may be NULL:
 * every workgroup then walks a whole history, which is always correct and needs no scratch, but leaves compute units
 * idle when U * ceil(C / 128) is small. Kernels: bf16 with d_q in {32, 64, 128} and d in {64, 128} on the matrix cores;
 * everything else (fp32 storage, other widths) on a generic fp32 kernel, one run per user.
 * Errors: as laser_forward, and LASER_ERR_ALIGN (work), LASER_ERR_SHAPE (work_bytes too small). Nothing is launched
 * on an error.
 */
size_t laser_forward_fused_work_bytes(int U, int C, int L, int d_q, int d, int w, laser_dtype dt);   /* host only */
laser_status laser_forward_fused(const void* q, const void* k, const void* v, const void* t0,
                                 const void* wq, const void* wk, const void* wv, const int32_t* lens,
                                 int U, int C, int L, int d_q, int d, int w, float gamma, laser_dtype dt,
                                 int32_t* seg_cnt, float* z_out, void* work, size_t work_bytes, void* stream);

/*
 * Ragged candidate counts per user (serving batches: every request brings its own number of candidates). The pair
 * tensors are packed: q [P,d_q], t0 [P,d], seg_out [P,S,d], z_out [P,d] hold the P pairs of the batch one after the
 * other, user by user, and cand_off [U+1] int32 (device) gives each user's rows, cand_off[u] .. cand_off[u+1]-1, with
 * cand_off[0] = 0, non-decreasing, cand_off[U] = P, and at most C_max rows per user (C_max sizes the launch; users
 * without candidates are allowed). Everything else (k, v, lens, seg_cnt [U,S], weights, arithmetic, kernels, limits
 * with C_max in the place of C) is as in laser_sta_forward / laser_gsta_forward / laser_forward, and with equal
 * counts the results are those of the dense entry points bit for bit. The host cannot see the offsets: on the device
 * they are clamped so that no access leaves the P rows (a user's first row into [0, P], its count into
 * [0, min(C_max, P - first)]); offsets that break the rules above give unspecified values in the rows concerned,
 * never a fault. Rows that belong to no user are not written.
 * Errors: as for the dense entry points, and LASER_ERR_NULL (cand_off), LASER_ERR_ALIGN (cand_off not 4-byte aligned),
 * LASER_ERR_SHAPE (P < 1, P > U * C_max, P * S * d >= 2^31). Nothing is launched on an error.
 */
laser_status laser_sta_forward_ragged(const void* q, const void* k, const void* v, const int32_t* lens,
                                      const int32_t* cand_off, int U, int C_max, int P, int L, int d_q, int d, int w,
                                      float gamma, laser_dtype dt, void* seg_out, int32_t* seg_cnt, void* stream);
laser_status laser_gsta_forward_ragged(const void* seg, const void* t0, const void* wq, const void* wk, const void* wv,
                                       const int32_t* lens, const int32_t* cand_off, int U, int C_max, int P, int L,
                                       int d, int w, int M, laser_dtype dt, float* z_out, void* stream);
laser_status laser_forward_ragged(const void* q, const void* k, const void* v, const void* t0, const void* wq,
                                  const void* wk, const void* wv, const int32_t* lens, const int32_t* cand_off, int U,
                                  int C_max, int P, int L, int d_q, int d, int w, float gamma, int M, laser_dtype dt,
                                  void* seg_out, int32_t* seg_cnt, float* z_out, void* stream);

/* The views of Sec. 3.4.4 and the segment FFN + LayerNorm step of Sec. 3.4.2 on packed pairs: seg [P,S,d], pool_out
 * [P,d], recent_out [P,r,d], seg_out [P,S,d]; cand_off, C_max and P as above, everything else as for
 * laser_multires_forward and laser_segment_ffn_forward (kernel chosen as by LASER_FFN_AUTO). */
laser_status laser_multires_forward_ragged(const void* seg, const int32_t* lens, const int32_t* cand_off, int U,
                                           int C_max, int P, int L, int d, int w, int r, laser_dtype dt, void* pool_out,
                                           void* recent_out, void* stream);
laser_status laser_segment_ffn_forward_ragged(const void* seg, const int32_t* lens, const int32_t* cand_off,
                                              const void* w1, const float* b1, const void* w2, const float* b2,
                                              const float* ln_g, const float* ln_b, int U, int C_max, int P, int L,
                                              int d, int d_ff, int w, float eps, laser_dtype dt, void* seg_out,
                                              void* stream);

/*
 * Segment feed-forward step (paper Sec. 3.4.2, the equation after the STA paragraph): every segment vector of H'
 * becomes s <- LN(FFN(s) + s). The paper names neither the network's shape nor the normalisation's constants; here
 *   FFN(s) = relu(s W1 + b1) W2 + b2,  W1 [d, d_ff], W2 [d_ff, d]  (row vector times matrix, as everywhere),
 *   LN(x)  = (x - mean(x)) / sqrt(var(x) + eps) * ln_g + ln_b       over the d components, biased variance.
 * seg [U,C,S,d] dt (H' as stored), lens [U] or NULL as for laser_gsta_forward; w1, w2 in dt; b1 [d_ff], b2 [d],
 * ln_g [d], ln_b [d] in fp32; d_ff a multiple of 8, at most 4096; eps >= 0. seg_out [U,C,S,d] dt is fully
 * overwritten and may be seg itself (in place). Vectors of segments without a valid item (i*w >= lens[u]) are
 * written as zeros. Arithmetic in fp32 (bf16 products on the matrix cores for bf16 storage, the hidden layer
 * rounded to bf16 between the two products); the result is rounded to dt once.
 * All pointers are device pointers, caller-owned; 16-byte alignment for seg, w1, w2, seg_out, 4-byte for the rest.
 * Errors: LASER_ERR_NULL, LASER_ERR_SHAPE, LASER_ERR_DTYPE, LASER_ERR_ALIGN, LASER_ERR_UNSUPPORTED (a forced variant
 * that does not take the shape), LASER_ERR_LAUNCH. Nothing is launched on an error.
 */
typedef enum {
  LASER_FFN_AUTO = 0,
  LASER_FFN_GENERIC = 1, /* fp32 FMA, any d and d_ff, either dtype                                   */
  LASER_FFN_MFMA = 2,    /* bf16 MFMA, d = 128, d_ff in {64, 128}, both weight matrices in LDS     */
  LASER_FFN_VARIANT_ANY_INT = 0x7fffffff
} laser_ffn_variant;

laser_status laser_segment_ffn_forward(const void* seg, const int32_t* lens, const void* w1, const float* b1,
                                       const void* w2, const float* b2, const float* ln_g, const float* ln_b,
                                       int U, int C, int L, int d, int d_ff, int w, float eps, laser_dtype dt,
                                       void* seg_out, void* stream);
laser_status laser_segment_ffn_forward_variant(const void* seg, const int32_t* lens, const void* w1, const float* b1,
                                               const void* w2, const float* b2, const float* ln_g, const float* ln_b,
                                               int U, int C, int L, int d, int d_ff, int w, float eps, laser_dtype dt,
                                               void* seg_out, void* stream, laser_ffn_variant variant);

/*
 * The segment feed-forward step followed by GSTA (paper Sec. 3.4.2, the FFN + LayerNorm equation, then Sec. 3.4.3):
 * z = GSTA(t0; s) with s = LN(FFN(H') + H') as laser_segment_ffn_forward defines it, rounded to dt once as if it
 * were stored. Arguments as for laser_segment_ffn_forward (seg, lens, w1 .. ln_b, d_ff, eps) and laser_gsta_forward
 * (t0, wq, wk, wv, M, z_out); all pointers are device pointers, caller-owned, aligned as there.
 * seg_out [U,C,S,d] dt receives s (fully overwritten, zeros for segments without a valid item); it may be seg itself,
 * and it may be NULL when s is not wanted. bf16, d = 128, d_ff in {64, 128}, M = 1: one pass over H', s is scored
 * and pooled while it is on chip, z_out holds intermediate values until the last of three launches has run. Any
 * other shape: laser_segment_ffn_forward into seg_out, then laser_gsta_forward on it, and LASER_ERR_UNSUPPORTED if
 * seg_out is NULL. Results agree with those two calls in a row up to the order of fp32 sums.
 * Errors: those of the two entry points (seg_out may be NULL), everything validated before the first launch.
 */
laser_status laser_ffn_gsta_forward(const void* seg, const void* t0, const void* wq, const void* wk, const void* wv,
                                    const int32_t* lens, const void* w1, const float* b1, const void* w2,
                                    const float* b2, const float* ln_g, const float* ln_b, int U, int C, int L, int d,
                                    int d_ff, int w, int M, float eps, laser_dtype dt, void* seg_out, float* z_out,
                                    void* stream);

/*
 * laser_ffn_gsta_forward with the two other views of Sec. 3.4.4 taken from the transformed rows s (the complete head
 * on a stored H'): pool_out [U,C,d] dt, recent_out [U,C,r,d] dt and r as for laser_multires_forward, everything else
 * as for laser_ffn_gsta_forward, everything validated before the first launch. Where that entry point makes one pass
 * over H' the views come from the same pass; otherwise laser_segment_ffn_forward into seg_out (required then), then
 * laser_gsta_forward_multires on it. z_out, pool_out and recent_out agree with those two calls in a row: the views
 * bit for bit, z_out up to the order of fp32 sums.
 */
laser_status laser_ffn_gsta_forward_multires(const void* seg, const void* t0, const void* wq, const void* wk,
                                             const void* wv, const int32_t* lens, const void* w1, const float* b1,
                                             const void* w2, const float* b2, const float* ln_g, const float* ln_b,
                                             int U, int C, int L, int d, int d_ff, int w, int M, float eps,
                                             laser_dtype dt, void* seg_out, float* z_out, int r, void* pool_out,
                                             void* recent_out, void* stream);

/*
 * Multi-resolution feature fusion (paper Sec. 3.4.4): besides the global context z, the representation holds
 * max_pool(H') and the r most recent segments s_1 .. s_r. Both are taken from a stored H':
 *   pool_out   [U,C,d]   dt   component-wise maximum over the segment vectors of the pair that hold at least one
 *                             valid item (segment i of user u is valid iff i*w < lens[u], as in GSTA); zeros when
 *                             there is none. Exact: a maximum of stored values. May be NULL (not wanted).
 *   recent_out [U,C,r,d] dt   rows 0 .. r-1 of H' (the paper counts the history from its most recent item, so
 *                             s_1 is row 0), copied as stored (zeros for segments without a valid item).
 *                             0 <= r <= S; NULL exactly when r == 0.
 * seg [U,C,S,d] dt and lens [U] (NULL = all L) as for laser_gsta_forward; all pointers are device pointers,
 * caller-owned, 16-byte aligned (lens 4-byte); outputs are fully overwritten; work is enqueued on `stream`.
 * Errors: LASER_ERR_NULL (seg NULL, or both outputs NULL), LASER_ERR_SHAPE (sizes, r out of range, r and
 * recent_out disagree), LASER_ERR_DTYPE, LASER_ERR_ALIGN, LASER_ERR_LAUNCH. Nothing is launched on an error.
 */
laser_status laser_multires_forward(const void* seg, const int32_t* lens, int U, int C, int L, int d, int w, int r,
                                    laser_dtype dt, void* pool_out, void* recent_out, void* stream);

/*
 * The whole path with all three views of Sec. 3.4.4: laser_forward followed by laser_multires_forward on the
 * stored H', same arguments, same results, same errors; everything is validated before the first launch. Where
 * the GSTA kernel holds a pair's H' block in registers (bf16, M = 1, d in {64, 128}, S up to 32 * 64 / (d / 8)) the
 * views are written by that kernel from the same pass over H'; otherwise a third launch reads H' again.
 */
laser_status laser_forward_multires(const void* q, const void* k, const void* v, const void* t0,
                                    const void* wq, const void* wk, const void* wv, const int32_t* lens,
                                    int U, int C, int L, int d_q, int d, int w, float gamma, int M, laser_dtype dt,
                                    void* seg_out, int32_t* seg_cnt, float* z_out,
                                    int r, void* pool_out, void* recent_out, void* stream);

/*
 * GSTA and the two other views of Sec. 3.4.4 from a stored H' (for callers that put a step of their own between STA
 * and GSTA, such as laser_segment_ffn_forward): laser_gsta_forward followed by laser_multires_forward on the same seg,
 * same arguments, same results (z_out, pool_out and recent_out bit for bit), same errors, everything validated before
 * the first launch; H' is read once where the GSTA kernel holds a pair's block in registers (see above), twice
 * otherwise.
 */
laser_status laser_gsta_forward_multires(const void* seg, const void* t0, const void* wq, const void* wk, const void* wv,
                                         const int32_t* lens, int U, int C, int L, int d, int w, int M, laser_dtype dt,
                                         float* z_out, int r, void* pool_out, void* recent_out, void* stream);

/*
 * The linear maps ahead of STA (paper Sec. 3.5.1, first two equations): Q = t W_q for the targets, and K = H W_k,
 * V = H W_v for every item of the raw history, both from one pass over H. Row vector times matrix, no bias.
 *   t   [U,C,d_in] dt   target embeddings          w_q [d_in,d_q] dt     q_out [U,C,d_q] dt
 *   h   [U,L,d_in] dt   raw history embeddings     w_k [d_in,d_q] dt     k_out [U,L,d_q] dt
 *                                                  w_v [d_in,d]   dt     v_out [U,L,d]   dt
 * The outputs are the q, k, v arguments of laser_sta_forward / laser_forward (items past a user's valid length are
 * projected like any other; STA never reads them). Products in fp32 (bf16 operands on the matrix cores for bf16
 * storage), accumulated over d_in in fp32, rounded to dt once. 1 <= d_in, d_q, d <= 4096.
 * All pointers are device pointers, caller-owned, 16-byte aligned; outputs are fully overwritten and must not
 * overlap the inputs; work is enqueued on `stream`.
 * Errors: LASER_ERR_NULL, LASER_ERR_SHAPE, LASER_ERR_DTYPE, LASER_ERR_ALIGN, LASER_ERR_UNSUPPORTED (a forced variant
 * that does not take the shape), LASER_ERR_LAUNCH. Nothing is launched on an error.
 */
typedef enum {
  LASER_PROJECT_AUTO = 0,
  LASER_PROJECT_GENERIC = 1, /* fp32 FMA, any sizes, either dtype                                               */
  LASER_PROJECT_MFMA = 2,    /* bf16 MFMA, d_in = 128, output widths multiples of 32, each <= 128, weights in LDS */
  LASER_PROJECT_VARIANT_ANY_INT = 0x7fffffff
} laser_project_variant;

laser_status laser_project_q_forward(const void* t, const void* w_q, int U, int C, int d_in, int d_q, laser_dtype dt,
                                     void* q_out, void* stream);
laser_status laser_project_q_forward_variant(const void* t, const void* w_q, int U, int C, int d_in, int d_q,
                                             laser_dtype dt, void* q_out, void* stream,
                                             laser_project_variant variant);
laser_status laser_project_kv_forward(const void* h, const void* w_k, const void* w_v, int U, int L, int d_in, int d_q,
                                      int d, laser_dtype dt, void* k_out, void* v_out, void* stream);
laser_status laser_project_kv_forward_variant(const void* h, const void* w_k, const void* w_v, int U, int L, int d_in,
                                              int d_q, int d, laser_dtype dt, void* k_out, void* v_out, void* stream,
                                              laser_project_variant variant);

/*
 * Folded form of projections + STA for few candidates per user (paper Sec. 3.5.1: the matrices do not depend on the
 * position, so the products can be re-associated; here that is taken one step further than the paper does). K and V
 * are never formed and the raw history is read once:
 *   score of head h for item j   (t W_q)_h . (h_j W_k)_h  =  (t A_h) . h_j,     A_h = W_q,h W_k,h^T  [d_in, d_in]
 *   segment vector of head h     sum_j g_j (h_j W_v,h)    =  (sum_j g_j h_j) W_v,h
 * with W_x,h head h's run of columns (d_q / heads of W_q and W_k, d / heads of W_v), as in laser_sta_forward_heads.
 *
 * laser_fold_query_weights: a_out [d_in, heads * d_in] dt, A = [A_1 | ... | A_heads], from w_q, w_k [d_in, d_q] dt
 *   (fp32 sums rounded once to dt). Done once per model.
 * laser_project_heads_forward: y[p, i, h b + e] = sum_k x[p, h, i, k] w_v[k, h b + e], b = d / heads;
 *   x [P, heads, S, d_in] dt, w_v [d_in, d] dt, y [P, S, d] dt. d_in, d multiples of 8, heads divides d.
 * laser_sta_folded_forward: the whole chain from raw embeddings to H':
 *   qf_work [U, C * heads, d_in] dt   <- t A                      (laser_project_q_forward with A)
 *   g_work  [U, C * heads, S, d_in] dt <- STA(qf_work, h, h)      (laser_sta_forward: keys = values = raw items)
 *   seg_out [U, C, S, d] dt           <- laser_project_heads_forward(g_work, w_v)
 *   t [U,C,d_in], h [U,L,d_in], a_fold from laser_fold_query_weights, lens / seg_cnt / gamma as for
 *   laser_sta_forward. The two work buffers are caller-owned scratch (contents on return: the intermediates above,
 *   each rounded to dt); the library allocates nothing. Equal to projections followed by STA in exact arithmetic;
 *   in bf16 the intermediates are rounded at other places, so the two forms differ within the tolerance.
 * All pointers are device pointers, caller-owned, 16-byte aligned (lens, seg_cnt 4-byte); work is enqueued on
 * `stream`. Errors as for laser_sta_forward and laser_project_kv_forward; nothing is launched on an error.
 */
laser_status laser_fold_query_weights(const void* w_q, const void* w_k, int d_in, int d_q, int heads, laser_dtype dt,
                                      void* a_out, void* stream);
laser_status laser_project_heads_forward(const void* x, const void* w_v, int P, int S, int d_in, int d, int heads,
                                         laser_dtype dt, void* y, void* stream, laser_project_variant variant);
laser_status laser_sta_folded_forward(const void* t, const void* h, const void* a_fold, const void* w_v,
                                      const int32_t* lens, int U, int C, int L, int d_in, int d, int w, float gamma,
                                      int heads, laser_dtype dt, void* qf_work, void* g_work, void* seg_out,
                                      int32_t* seg_cnt, void* stream);

/*
 * Backward pass of STA (the derivatives of the forward equations of paper Sec. 3.4.2; the paper trains the module,
 * Sec. 4.1.2, and prints no backward formulas). Given dseg = d loss / d H' [U,C,S,d] (dt), with
 *   g_cj = sigmoid(q_c . k_j / gamma)   and   ds_cj = (dseg[c, i(j), :] . v_j) g_cj (1 - g_cj),   i(j) = j / w:
 *   dv_out[u,j,:] = sum_c g_cj dseg[u,c,i(j),:]           [U,L,d]   fp32
 *   dk_out[u,j,:] = sum_c ds_cj q[u,c,:] / gamma          [U,L,d_q] fp32
 *   dq_out[u,c,:] = sum_j ds_cj k[u,j,:] / gamma          [U,C,d_q] fp32
 * over the valid items j < lens[u]; items at or past the valid length get zeros (all outputs are fully overwritten).
 * q, k, v, lens, sizes and gamma as for laser_sta_forward (one head, sigmoid gates). Arithmetic in fp32 from the stored
 * inputs; sums in a fixed order (results are reproducible run to run).
 * Built for training batches, which hold one or a few targets per sample: d_q, d <= 256 (wider rows return
 * LASER_ERR_UNSUPPORTED), any number of candidates per user: more than four in bf16 with d_q in {32, 64, 128} and d in
 * {64, 128} run on the matrix cores, other cases up to eight candidates in one pass over k and v, more eight at a time,
 * one pass each, the later passes adding to dk_out and dv_out. work is caller-owned scratch of at least laser_sta_backward_work_bytes(U, C, L, d_q, w)
 * bytes (partial dq sums; contents unspecified on return); the library allocates nothing.
 * All pointers are device pointers, 16-byte aligned (lens 4-byte); work is enqueued on `stream`.
 * Errors: LASER_ERR_NULL, LASER_ERR_SHAPE (sizes, gamma, work_bytes too small), LASER_ERR_DTYPE, LASER_ERR_ALIGN,
 * LASER_ERR_UNSUPPORTED, LASER_ERR_LAUNCH. Nothing is launched on an error.
 */
size_t laser_sta_backward_work_bytes(int U, int C, int L, int d_q, int w);   /* host only; 0 for invalid sizes */
laser_status laser_sta_backward(const void* q, const void* k, const void* v, const int32_t* lens, const void* dseg,
                                int U, int C, int L, int d_q, int d, int w, float gamma, laser_dtype dt,
                                float* dq_out, float* dk_out, float* dv_out, void* work, size_t work_bytes,
                                void* stream);

/*
 * The same with bf16 inputs and the two large gradients in bf16 as well: dk_out [U,L,d_q] and dv_out [U,L,d] in the
 * storage type of k and v (fp32 sums rounded once), dq_out [U,C,d_q] fp32. Half the bytes of the pass's largest
 * outputs. C <= 4, d_q in {32, 64, 128}, d in {64, 128}; otherwise LASER_ERR_UNSUPPORTED. Everything else as above.
 */
laser_status laser_sta_backward_bf16(const void* q, const void* k, const void* v, const int32_t* lens, const void* dseg,
                                     int U, int C, int L, int d_q, int d, int w, float gamma, float* dq_out,
                                     void* dk_out, void* dv_out, void* work, size_t work_bytes, void* stream);

/*
 * laser_sta_backward for callers that cannot allocate device memory at all (code under HIP graph capture, tight
 * serving or training loops, harnesses that forbid hipMalloc): the same operation, kernels, results (bit for bit) and
 * errors, with the scratch of partial dq sums taken from a fixed array inside the library instead of a caller's
 * buffer. The array is device memory of the library's own code object, LASER_STATIC_SCRATCH_BYTES per GPU, held by
 * every GPU the library runs on until the process ends; its address is looked up once per device, on the first call
 * with that device current (a symbol lookup, no allocation). The call allocates and frees nothing.
 * Limit: laser_sta_backward_work_bytes(U, C, L, d_q, w) <= LASER_STATIC_SCRATCH_BYTES, else LASER_ERR_SHAPE and
 * nothing is launched (the paper's training batch of 2048 x 1 targets, L = 1000, w = 10, d_q = 32 needs 2.4 MB).
 * Every call on a GPU uses that GPU's one array: calls that overlap in time on the same GPU (two streams, two
 * threads) race on it and must be serialised by the caller; calls in order on one stream are safe. Nothing in the
 * array has to start at zero (every partial sum that is read is written first by the same call).
 */
#define LASER_STATIC_SCRATCH_BYTES (8u << 20)
laser_status laser_sta_backward_static(const void* q, const void* k, const void* v, const int32_t* lens,
                                       const void* dseg, int U, int C, int L, int d_q, int d, int w, float gamma,
                                       laser_dtype dt, float* dq_out, float* dk_out, float* dv_out, void* stream);

/*
 * Backward pass of GSTA (the derivatives of the forward equations of paper Sec. 3.4.3: per layer q' = t W_q,
 * e = (H' W_k) q' / sqrt(d), a = softmax over the valid segments, t <- t + a (H' W_v); the paper prints no backward
 * formulas). Given dz = d loss / d z [U,C,d] (fp32):
 *   dseg_out [U,C,S,d] dt    d loss / d H' through GSTA (rows of segments without a valid item are zeros); this is the
 *                            dseg argument of laser_sta_backward (add the other consumers of H' first, if any)
 *   dt0_out  [U,C,d]   fp32  d loss / d t0
 *   dwq_out, dwk_out, dwv_out [M,d,d] fp32, summed over all pairs in a fixed order
 * seg, t0, wq, wk, wv, lens and the sizes as for laser_gsta_forward. Arithmetic in fp32 from the stored inputs; dseg_out
 * is rounded once to dt. Limits: d <= 256,
 * M <= 8 and S d sizeof(dt) + ((M > 1 ? S d : 0) + (M + 7) d + 2 S + 4) * 4 bytes <= 150 KB; other shapes return LASER_ERR_UNSUPPORTED. work is caller-owned scratch
 * of at least laser_gsta_backward_work_bytes(U, C, d, M) bytes (six d-vectors per pair and layer, whose outer products
 * are the weight gradients, and for many pairs partial sums of those); the library allocates nothing.
 * All pointers are device pointers, 16-byte aligned (lens 4-byte); outputs are fully overwritten; work is enqueued on
 * `stream`. Errors: LASER_ERR_NULL, LASER_ERR_SHAPE (sizes, work_bytes too small), LASER_ERR_DTYPE, LASER_ERR_ALIGN,
 * LASER_ERR_UNSUPPORTED, LASER_ERR_LAUNCH. Nothing is launched on an error.
 */
size_t laser_gsta_backward_work_bytes(int U, int C, int d, int M);   /* host only; 0 for invalid sizes */
laser_status laser_gsta_backward(const void* seg, const void* t0, const void* wq, const void* wk, const void* wv,
                                 const int32_t* lens, const float* dz, int U, int C, int L, int d, int w, int M,
                                 laser_dtype dt, void* dseg_out, float* dt0_out, float* dwq_out, float* dwk_out,
                                 float* dwv_out, void* work, size_t work_bytes, void* stream);

/*
 * Attention among a history's own items: the encoder in front of STA, which the paper compares against as self-attention
 * (Sec. 4.2) and costs as C_SA (Sec. 3.6), causal and with the sequences packed. Sequence n owns rows off[n] .. off[n+1]-1
 * of q, k and v; query head h reads key-value head h / (H / H_kv). For item i of a sequence
 *   s_ij = q_i . k_j / gamma (j <= i),  lse_i = log sum_j exp s_ij,  o_i = sum_j exp(s_ij - lse_i) v_j.
 *   q [T,H,D] dt, k, v [T,H_kv,D] dt; heads of a token lie side by side, tokens q_pitch, k_pitch, v_pitch elements apart
 *   (column blocks of one projection's output need no copy); o_out [T,H,D] dt, lse_out [T,H] fp32 (NULL: not wanted, but
 *   the backward pass takes it). off [N+1] int32 on the device, non-decreasing; sequences may be empty. T: rows of the
 *   buffers; L_max: at least the longest sequence, sizes the launch.
 * Limits: D a multiple of 8, at most 128; H a multiple of H_kv, at most 1024; L_max * H < 2^30; T * H < 2^31; pitches at
 * least heads * D, at most 2^22, and whole 16-byte pieces; N * H_kv times the tiles of L_max * H / H_kv rows (of 128 rows, fp32 up
 * to 64 of 32) at most 2^31 - 1 (where they are more than 2^23 a kernel may go out in several launches, each of whole sequences);
 * gamma finite, at least 2^-126 (backward: and at most 2^120), and scores log2(e) q_i . k_j / gamma within fp32. Sums, the
 * softmax's statistics and its exponents are fp32; for bf16 storage probabilities are rounded to bf16 ahead of their product
 * with V, o is rounded once.
 * The offsets are clamped on the device so that no access leaves the T rows (a sequence's first row into [0, T], its length
 * into [0, min(L_max, T - first)]); offsets that break the rules give unspecified values in the rows concerned, never a
 * fault. Rows of no sequence are neither read into a result (they may hold anything, NaN included) nor written. The items of
 * a sequence are taken to be finite: an infinite or NaN value can reach all rows of its sequence, also earlier ones.
 * All pointers are device pointers, caller-owned, outputs apart from inputs; 16-byte alignment for q, k, v, o_out, 4-byte for off
 * and lse_out.
 * Errors: LASER_ERR_NULL, LASER_ERR_SHAPE, LASER_ERR_DTYPE, LASER_ERR_ALIGN, LASER_ERR_LAUNCH. Nothing is launched on an
 * error.
 */
laser_status laser_history_attention_forward(const void* q, int64_t q_pitch, const void* k, int64_t k_pitch, const void* v,
                                             int64_t v_pitch, const int32_t* off, int N, int T, int L_max, int H, int H_kv, int D,
                                             float gamma, laser_dtype dt, void* o_out, float* lse_out, void* stream);

/*
 * Its gradients. With p_ij = exp(s_ij - lse_i), delta_i = d_o_i . o_i, ds_ij = p_ij (d_o_i . v_j - delta_i):
 *   dq_i = sum_j ds_ij k_j / gamma,   dk_j = sum_i ds_ij q_i / gamma,   dv_j = sum_i p_ij d_o_i
 * (keys and values: summed over the query heads that share them, in a fixed order). o, lse as the forward pass wrote them,
 * d_o [T,H,D] dt; dq_out [T,H,D], dk_out, dv_out [T,H_kv,D] dt with pitches of their own, summed in fp32 and rounded once (for
 * bf16 storage p and ds are rounded to bf16 ahead of their products). Rows of no sequence are not written. work:
 * laser_history_attention_backward_work_bytes() bytes of caller-owned scratch, contents unspecified before and after; calls
 * that overlap need one each. The rest, limits and errors as above (work_bytes too small: LASER_ERR_SHAPE).
 */
size_t laser_history_attention_backward_work_bytes(int N, int T, int L_max, int H, int H_kv, int D,
                                                   laser_dtype dt);   /* host only; 0 for invalid sizes */
laser_status laser_history_attention_backward(const void* q, int64_t q_pitch, const void* k, int64_t k_pitch, const void* v,
                                              int64_t v_pitch, const void* o, const float* lse, const void* d_o,
                                              const int32_t* off, int N, int T, int L_max, int H, int H_kv, int D, float gamma,
                                              laser_dtype dt, void* dq_out, int64_t dq_pitch, void* dk_out, int64_t dk_pitch,
                                              void* dv_out, int64_t dv_pitch, void* work, size_t work_bytes, void* stream);

/*
 * The same attention while it is served: keys and values of a user's items stay in a paged cache, and new items (a chunk of
 * them, or one) or candidates attend to what is there.
 *   k_cache, v_cache [P,H_kv,page,D] dt: P pages of `page` items (a power of two, 8 to 4096). pages [U,max_pages] int32:
 *   item j of user u stands in page pages[u, j / page] at place j % page. Entries past a user's items are never read; an
 *   entry outside [0, P) is a page without items: nothing reads, writes or counts its places. lens [U] int32: items of each
 *   user, clamped to [0, min(L_max, max_pages * page)]; L_max sizes the launches.
 * Rows beside the cache (new keys and values, queries) are packed: user u's are off[u] .. off[u+1]-1 of T, at most C_max of
 * them, with pitches and limits as in laser_history_attention_forward (C_max * H < 2^30 too); offsets are clamped as there.
 *
 * laser_cache_append: user u's c new rows become the last c of its lens[u] items (lens counts them already); where
 *   there are more rows than items the first ones have no place and are left out. weight [P,page] fp32 (NULL: none): their
 *   places are set to 0. A page must not be listed twice, by one user or two, where new rows go.
 * laser_cache_attention_forward: o_out [T,H,D] dt, lse_out [T,H] fp32 (NULL: not wanted). causal != 0: the rows are the last
 *   c items of the cache (laser_cache_append has run), row i sees items 0 .. lens[u] - c + i. causal = 0: the rows are
 *   not in the cache (a request's candidates) and see all of it. A row that sees nothing gets zeros and lse = -inf. Items are
 *   taken to be finite, as above: an infinite or NaN value can reach rows of the same call that do not see it.
 *   work: laser_cache_attention_work_bytes() bytes of caller-owned scratch, contents unspecified before and after; calls that
 *   overlap need one each.
 * laser_cache_weights: what each item received, weight[its place] = sum of exp(s - lse) over the rows that see it and
 *   the H heads (add != 0: added to what stands there, atomically, so a page that several users list gets each one's part).
 *   q, lse, causal as for laser_cache_attention_forward; places behind a user's items are left alone. add = 0: a page that
 *   several users list ends up with one of their parts.
 * laser_cache_evict: each user keeps at most `budget` items: the last `recent` ones (0 <= recent <= budget) and of
 *   the others the heaviest by weight (of equal ones the first; NaN, and places on no page, count least). They move, in
 *   their order, with their weights, into the pages of pages_out [U,max_pages_out], of which none may be listed twice or be one that
 *   any user reads from in this call; a user within the budget keeps everything and moves too (an item on no page that stays
 *   all the same leaves its new place as it was: what stands there counts as an item from then on). lens_out [U] (may be lens
 *   itself) receives the new lengths, kept_out [U,budget] the old places of the items that stay, -1 behind the last.
 * Results are the same from run to run (laser_cache_weights with add: unless users share a page). Rows of no user and
 * places behind a user's items are never written.
 * All pointers are device pointers, caller-owned, outputs apart from inputs (but for lens_out); 16-byte alignment for q, k, v, the
 * caches, o_out and work, 4-byte for the rest. Errors: LASER_ERR_NULL, LASER_ERR_SHAPE, LASER_ERR_DTYPE, LASER_ERR_ALIGN,
 * LASER_ERR_LAUNCH. Nothing is launched on an error.
 */
laser_status laser_cache_append(const void* k, int64_t k_pitch, const void* v, int64_t v_pitch, void* k_cache, void* v_cache,
                                const int32_t* off, const int32_t* pages, const int32_t* lens, int U, int T, int C_max, int P,
                                int page, int max_pages, int L_max, int H_kv, int D, laser_dtype dt, float* weight,
                                void* stream);
size_t laser_cache_attention_work_bytes(int U, int T, int C_max, int L_max, int H, int H_kv, int D,
                                        laser_dtype dt);   /* host only; 0 for invalid sizes */
laser_status laser_cache_attention_forward(const void* q, int64_t q_pitch, const void* k_cache, const void* v_cache,
                                           const int32_t* off, const int32_t* pages, const int32_t* lens, int U, int T, int C_max,
                                           int P, int page, int max_pages, int L_max, int H, int H_kv, int D, float gamma,
                                           int causal, laser_dtype dt, void* o_out, float* lse_out, void* work,
                                           size_t work_bytes, void* stream);
laser_status laser_cache_weights(const void* q, int64_t q_pitch, const float* lse, const void* k_cache, const int32_t* off,
                                 const int32_t* pages, const int32_t* lens, int U, int T, int C_max, int P, int page,
                                 int max_pages, int L_max, int H, int H_kv, int D, float gamma, int causal, int add,
                                 laser_dtype dt, float* weight, void* stream);
laser_status laser_cache_evict(void* k_cache, void* v_cache, float* weight, const int32_t* pages, const int32_t* lens,
                               const int32_t* pages_out, int U, int P, int page, int max_pages, int max_pages_out, int L_max,
                               int budget, int recent, int H_kv, int D, laser_dtype dt, int32_t* lens_out, int32_t* kept_out,
                               void* stream);

/*
 * Rotary positions for the encoder above: pair i < R / 2 of the first R columns of every head of token t is turned by the angle
 * pos[t] * freq[i] and scaled, the columns from R on are passed on. With c, s = cos, sin of the angle and pairs (a, b) of columns
 *   LASER_ROTARY_HALF          (i, i + R / 2)
 *   LASER_ROTARY_INTERLEAVED   (2 i, 2 i + 1)
 * laser_rotary_forward:  (a, b) -> scale (a c - b s, a s + b c);   laser_rotary_backward, its transpose: gradients
 * (a, b) -> scale (a c + b s, b c - a s). Queries and keys are turned by one launch.
 *   q [T,H,D] dt, k [T,H_kv,D] dt (NULL exactly when H_kv = 0, k_out too), heads of a token side by side, tokens at pitches of
 *   their own, as in laser_history_attention_forward; q_out, k_out likewise. An output may be its input (with its pitch: turned in
 *   place), and lies apart from all others. pos [T] int32: a token whose position is negative is left out, neither read nor written
 *   (rows of no sequence in a padded batch). freq [R/2] fp64, radians a position. Angles are formed and reduced in fp64, the rest is
 *   fp32, results are rounded once. R even, 2 to D; T, heads, D and pitches within the limits above; scale finite.
 * laser_rotary_frequencies: freq_out[i] = f_i = base^(-2i/R) for 2 <= R <= 128, for contexts `factor` times as long as those of training by
 *   LASER_ROTARY_LINEAR   f_i / factor
 *   LASER_ROTARY_BASE     base replaced by base * factor^(R / (R - 2)): the slowest pair is stretched by factor, the fastest is not
 *   LASER_ROTARY_PARTS    f_i (g + (1 - g) / factor), g = (length f_i / (2 pi) - low) / (high - low) within [0, 1]: pairs that make `high`
 *                         turns and more within the training's `length` stay, those of `low` and fewer are stretched
 *   (arguments that the way does not name are not looked at).
 * All pointers are device pointers, 16-byte alignment for q, k and the outputs, 8 for freq, 4 for pos. Errors: LASER_ERR_NULL,
 * LASER_ERR_SHAPE, LASER_ERR_DTYPE, LASER_ERR_UNSUPPORTED (no such layout or way), LASER_ERR_ALIGN, LASER_ERR_LAUNCH. Nothing is
 * launched on an error.
 */
typedef enum { LASER_ROTARY_HALF = 0, LASER_ROTARY_INTERLEAVED = 1, LASER_ROTARY_LAYOUT_ANY_INT = 0x7fffffff } laser_rotary_layout;
typedef enum {
  LASER_ROTARY_NONE = 0,
  LASER_ROTARY_LINEAR = 1,
  LASER_ROTARY_BASE = 2,
  LASER_ROTARY_PARTS = 3,
  LASER_ROTARY_SCALING_ANY_INT = 0x7fffffff
} laser_rotary_scaling;
laser_status laser_rotary_frequencies(int R, double base, laser_rotary_scaling scaling, double factor, double length, double low,
                                      double high, double* freq_out, void* stream);
laser_status laser_rotary_forward(const void* q, int64_t q_pitch, const void* k, int64_t k_pitch, const int32_t* pos,
                                  const double* freq, int T, int H, int H_kv, int D, int R, laser_rotary_layout layout, float scale,
                                  laser_dtype dt, void* q_out, int64_t q_out_pitch, void* k_out, int64_t k_out_pitch, void* stream);
laser_status laser_rotary_backward(const void* d_q, int64_t d_q_pitch, const void* d_k, int64_t d_k_pitch, const int32_t* pos,
                                   const double* freq, int T, int H, int H_kv, int D, int R, laser_rotary_layout layout, float scale,
                                   laser_dtype dt, void* dq_out, int64_t dq_pitch, void* dk_out, int64_t dk_pitch, void* stream);

/*
 * The paged cache with its items in 8 bits, half the bytes of the bf16 one and what bounds few rows over long histories. It is appended to and
 * attended over; received weights and eviction (laser_cache_weights, laser_cache_evict) are of the fp32 and bf16 caches alone.
 *   k_cache, v_cache [P,H_kv,page,D] e4m3 (4 bits of exponent, 3 of mantissa, largest 448, no infinities); D a multiple of 16, at most 128.
 *   k_scale, v_scale [P,H_kv,page/block] fp32: what the numbers of each block of `block` items (a power of two, 8 to page) of a head are
 *   times; a power of two from 2^-100 to 2^119 (of any other value, what comes of the block's items is unspecified).
 *   Pages, tables, lengths, rows, offsets and their limits are those of the cache above; dt is the type of the rows (fp32 or bf16).
 *
 * laser_cache8_append: user u's c new rows become the last c of its lens[u] items, as in laser_cache_append. For every head's keys and
 *   values, a block that rows come into has the scale max(the one it had, where it held items of the user before them; the
 *   smallest power of two 2^x, -100 <= x <= 119, with |y| <= 448 2^x for all finite elements y of the new ones); each new element becomes
 *   the e4m3 number nearest to y / scale (of two equally near the even one), at most 448 in magnitude, infinities too; NaN stays
 *   NaN. Where the scale grows, the older items' numbers are rounded again to the new one. Places behind a user's items are not
 *   written. A page must not be listed twice, by one user or two, where new rows go. The blocks that min(C_max, L_max, T) rows touch
 *   are, times H_kv, at most 2^23 - 1.
 * laser_cache8_attention_forward: as laser_cache_attention_forward over the items' values (number times scale). bf16 rows:
 *   probabilities are rounded to bf16 ahead of their product with the values, o is rounded once; fp32 rows: every product and sum is of
 *   fp32's precision. A row whose query is NaN is NaN; so is one that sees a key that is NaN, and, in its columns, one that sees a value
 *   that is; rows that do not see such an item have nothing of it. Values are summed in fp32 ahead of the division, with probabilities of up to
 *   2^8: of values beyond 2^119 / lens the sum may overflow. work: laser_cache8_attention_work_bytes() bytes.
 * Results are the same from run to run. Everything else, alignment (4 bytes for scales) and errors as for the cache above.
 */
laser_status laser_cache8_append(const void* k, int64_t k_pitch, const void* v, int64_t v_pitch, void* k_cache, void* v_cache,
                                 float* k_scale, float* v_scale, const int32_t* off, const int32_t* pages, const int32_t* lens, int U,
                                 int T, int C_max, int P, int page, int block, int max_pages, int L_max, int H_kv, int D,
                                 laser_dtype dt, void* stream);
size_t laser_cache8_attention_work_bytes(int U, int T, int C_max, int L_max, int H, int H_kv, int D,
                                         laser_dtype dt);   /* host only; 0 for invalid sizes */
laser_status laser_cache8_attention_forward(const void* q, int64_t q_pitch, const void* k_cache, const void* v_cache,
                                            const float* k_scale, const float* v_scale, const int32_t* off, const int32_t* pages,
                                            const int32_t* lens, int U, int T, int C_max, int P, int page, int block, int max_pages,
                                            int L_max, int H, int H_kv, int D, float gamma, int causal, laser_dtype dt, void* o_out,
                                            float* lse_out, void* work, size_t work_bytes, void* stream);

/*
 * Who holds the pages of a cache, of whatever type. refs [P] int32 counts, for every page, the places of tables that name it
 * (pages [U,max_pages], the first ceil(lens[u] / page) of user u); a page with count 0 or less is free. Free pages are taken from the
 * lowest number up, users in order, so results are the same from run to run. A page's contents are its parts: n_parts arrays
 * (at most 1024) [P, part_bytes[i] bytes], parts and part_bytes being arrays in HOST memory (read before the call returns) of device
 * pointers and of sizes (at most 2^27; copies are by 16 bytes where pointer and size are multiples of 16, by 4, or by 1).
 * Entries outside [0, P) are pages without items: they pass on as they are, are counted and copied nowhere. lens are clamped to
 * [0, max_pages * page].
 * laser_pages_grow: lens[u] += off[u+1] - off[u] (nothing where that is negative; to max_pages * page at most), and the table gets
 *   fresh pages, counts 1, for the entries that the new length asks for. Ahead of an append of the rows that off packs. (Where a table is
 *   full the length stays, and the append puts the last rows in the place of items that were there: max_pages is to allow for them.)
 * laser_pages_fork: history v of the new tables pages_out [V,max_pages_out], lens_out [V] is the one of user source[v] (int32; outside
 *   [0, U): an empty one; a longer one than max_pages_out pages hold is cut there). Whole pages are shared, their counts go up; a partly filled last
 *   one is copied into a fresh page, all of it, so that either history can be appended to. Entries behind a history's pages become -1. The old tables
 *   stay valid and hold what they held.
 * missing_out [1] int32: fresh pages that there were none for; their entries are -1, the last ones in order.
 * laser_pages_free: of the users with gone[u] != 0 (NULL: all) every page's count goes down (never below 0), and lens[u] becomes 0;
 *   entries are left alone.
 * laser_pages_compact: the M pages in use move so that they are pages 0 .. M-1: those numbered M and more, in order, into the free ones
 *   below M, in order. pages_out [U,max_pages]: the tables with the new numbers (-1 behind a user's pages), refs_out [P] the counts,
 *   in_use_out [1] M. Tables must name no page whose count is 0, and all tables are one call's (those of forks side by side with the
 *   others): one that is not given keeps numbers that are no longer its pages'.
 * laser_pages_copy: page to[i] becomes a copy of page from[i] (int32 [n]; a pair with one outside [0, P) is left out). No page may be
 *   in `to` twice or in both.
 * page: items of one, a power of two, 8 to 4096. P <= 2^26; U * max_pages, V * max_pages_out, and items of a table below 2^31. work:
 * laser_pages_work_bytes(max(U, V), P) bytes of caller-owned scratch, contents unspecified before and after; calls that overlap need one
 * each. All other pointers are device pointers, 4-byte aligned, outputs apart from inputs (lens, refs, and grow's pages: in place).
 * Errors: LASER_ERR_NULL, LASER_ERR_SHAPE, LASER_ERR_ALIGN, LASER_ERR_LAUNCH. Nothing is launched on an error.
 */
size_t laser_pages_work_bytes(int U, int P);   /* host only; 0 for invalid sizes */
laser_status laser_pages_grow(int32_t* pages, int32_t* lens, const int32_t* off, int32_t* refs, int U, int P, int page, int max_pages,
                              int32_t* missing_out, void* work, size_t work_bytes, void* stream);
laser_status laser_pages_fork(void* const* parts, const int64_t* part_bytes, int n_parts, const int32_t* pages, const int32_t* lens,
                              const int32_t* source, int32_t* refs, int U, int V, int P, int page, int max_pages, int max_pages_out,
                              int32_t* pages_out, int32_t* lens_out, int32_t* missing_out, void* work, size_t work_bytes,
                              void* stream);
laser_status laser_pages_free(const int32_t* pages, int32_t* lens, const int32_t* gone, int32_t* refs, int U, int P, int page,
                              int max_pages, void* stream);
laser_status laser_pages_compact(void* const* parts, const int64_t* part_bytes, int n_parts, const int32_t* pages, const int32_t* lens,
                                 const int32_t* refs, int U, int P, int page, int max_pages, int32_t* pages_out, int32_t* refs_out,
                                 int32_t* in_use_out, void* work, size_t work_bytes, void* stream);
laser_status laser_pages_copy(void* const* parts, const int64_t* part_bytes, int n_parts, const int32_t* from, const int32_t* to,
                              int n, int P, void* stream);

/* Name of the family of STA / GSTA kernels AUTO would pick from for a shape in a batch that fills the machine (smaller ones
 * may take another form; "sta_generic" and "gsta_generic" include the matrix-core kernels that AUTO runs for fp32 at the
 * usual widths, "sta_stream_bf16" the one for a few candidates per user; static strings; host only, no GPU needed). */
const char* laser_sta_kernel_name(int C, int d_q, int d, int w, laser_dtype dt);
const char* laser_gsta_kernel_name(int C, int S, int d, laser_dtype dt);               /* one layer (M = 1) */
const char* laser_gsta_kernel_name_layers(int C, int S, int d, int M, laser_dtype dt);

/* Static, human-readable name of a status code. Never NULL. */
const char* laser_status_string(laser_status s);

/* Library version as major * 10000 + minor * 100 + patch. */
int laser_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LASER_H_ */
