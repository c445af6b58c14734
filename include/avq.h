/*
 * avq.h - C ABI of the MI355X (gfx950) AVQ-Attention forward pass.
 *
 * AVQ-Attention (Adaptive Vector-Quantized Attention) replaces keys by
 * codewords of a two-level codebook: M0 parents per head, each with Ch
 * children whose mean is the parent (Sec. 4.1, Eq. (parent_constraint)).
 * The forward pass is split into three calls, in this order:
 *
 *   avq_assign         keys -> nearest parent, then nearest child of that
 *                      parent (Sec. 4.2, Alg. 1)
 *   avq_aggregate      per-codeword key counts and value sums
 *                      (Eq. (aggregates), Alg. 1)
 *   avq_pack_aggregates  value sums and counts held by the caller, in the
 *                      operand layout of the attention kernel
 *   avq_attention_fwd  parent attention, per-query-tile importance, top-P
 *                      parent selection, child refinement with correcting
 *                      attention and normalisation (Sec. 4.3,
 *                      Eq. (vqflashattention), (importance),
 *                      (parent_recovery), (correcting_attention), Alg. 2)
 *   avq_attention_fwd_tiled  the same with the tiled-codeword importance of
 *                      App. B (Eq. (aproxdenom), (codewordimportance))
 *   avq_codebook_update  EMA codebook statistics and the constrained child
 *                      projection (App. A, Eq. (child_constraint_solve))
 *   avq_attention_fwd_ordered  attention with the queries in a given order
 *                      (the space-filling-curve reordering of Sec. 4)
 *   avq_gilbert_order  host helper: that order for a 2-D grid of tokens
 *
 * Beside it stand exact attention and the cache that a server keeps (their
 * conventions are given with them):
 *
 *   avq_prompt_attention_fwd  exact attention of packed prompts
 *   avq_cache_append   keys and values into a paged cache, with the rotation
 *   avq_cache_gather   cached positions read back
 *   avq_cache_attention_fwd  exact attention of the newest tokens over the cache
 *   avq_rotate_axes    rotary positions with several axes, and back
 *   avq_cross_attention_fwd, avq_cross_attention_bwd  exact attention over an
 *                      encoder's states, and its gradients
 *   avq_cache_prefix_attention_fwd  attention over the cache for groups of
 *                      sequences that share their first positions
 *
 * Conventions shared by every call:
 *   - Every array argument is a DEVICE pointer owned by the caller, contiguous,
 *     row-major and 16-byte aligned. Inputs are never written. Outputs are
 *     fully overwritten.
 *   - Tensors: Q, K, V, Y are [B][H][N][d]; the codebook is Cp [H][M0][d]
 *     (parents) and Cc [H][M0][Ch][d] (children of parent p in rows
 *     p*Ch .. p*Ch+Ch-1), shared across the batch (one codebook per head).
 *   - Codes: Mtot = M0*(1+Ch). Code p < M0 is parent p; code M0 + p*Ch + c is
 *     child c of parent p.
 *   - dtype selects the element type of Q, K, V, Cp, Cc and Y: AVQ_F32 (fp32)
 *     or AVQ_BF16 (bfloat16). Value sums are fp32, counts int32; the packed
 *     aggregates hold mean values in dtype.
 *   - Logits are exactly Q.C (the paper leaves the 1/sqrt(d) scale out of its
 *     formulas, Eq. (standardattention)); callers fold any scale into Q.
 *   - Calls are asynchronous on `stream` (a hipStream_t; NULL = the default
 *     stream). No call synchronises the device or allocates device memory:
 *     the device calls enqueue kernels only (no memset or copy), so after one
 *     call of an entry point on a device (it caches the device's attributes
 *     and kernel settings) its calls can be captured in a HIP graph.
 *   - Arguments are validated on the host before anything is launched; a
 *     non-OK status means nothing was enqueued (AVQ_ERR_DEVICE: a launch was
 *     rejected). avq_last_error() then returns a message for the calling
 *     thread. Inputs are not checked for NaN or infinity; the kernels are
 *     compiled without NaN semantics, so outputs for such inputs are
 *     unspecified (they need not be NaN).
 *   - Supported: d in {64, 128}; Ch in {0, 1, 2, 4, 8, 16}; 1 <= M0 <= 512;
 *     1 <= N <= 2^24, B >= 1, H >= 1 and B*H*N*d < 2^31. Other shapes return
 *     AVQ_ERR_UNSUPPORTED.
 *   - Ch = 0 is a flat codebook of M0 codewords (plain vector quantisation,
 *     Sec. 3.2): Cc may then be NULL, every code is a parent (Mtot = M0),
 *     and avq_attention_fwd needs P = 0, which is VQ attention (Sec. 3.2).
 */
#ifndef AVQ_H
#define AVQ_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  AVQ_OK = 0,
  AVQ_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, P outside [0, M0], ... */
  AVQ_ERR_UNSUPPORTED = 2, /* valid, but a shape/dtype this build has no kernel for */
  AVQ_ERR_DEVICE = 3       /* the HIP runtime rejected a launch */
} avq_status_t;

/* Element type of the dtype arguments. A plain 32-bit integer rather than an
 * enum type, so that any value a caller passes is well defined on arrival:
 * values other than these two are rejected with AVQ_ERR_INVALID_ARG. */
typedef int32_t avq_dtype_t;
enum { AVQ_F32 = 0, AVQ_BF16 = 1 };

/* Version of this ABI (major * 100 + minor). */
int avq_version(void);

/* Message for the last non-OK status returned to the calling thread
 * ("" if none). The pointer stays valid until the thread's next call. */
const char* avq_last_error(void);

/*
 * avq_assign - tree vector quantisation of the keys (Sec. 3.2 assignment with
 * squared Euclidean distance; Sec. 4.2 and Alg. 1 parent/child loops).
 *
 * For every key K[b][h][j]:
 *   parent_idx = p* = argmin_p ||K_j - Cp[h][p]||^2, lowest p on exact ties;
 *   c*            = argmin_c ||K_j - Cc[h][p*][c]||^2, lowest c on exact ties;
 *   code_idx      = M0 + p* * Ch + c* if that child distance is strictly below
 *                   the parent distance, else p* (always p* when Ch = 0).
 * Distances are evaluated in fp32 from the stored inputs.
 *
 *   K            [B][H][N][d]   dtype
 *   Cp           [H][M0][d]     dtype
 *   Cc           [H][M0][Ch][d] dtype (NULL allowed when Ch = 0)
 *   parent_idx   [B][H][N]      int32, out
 *   code_idx     [B][H][N]      int32, out
 */
avq_status_t avq_assign(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N, int32_t d,
                        int32_t M0, int32_t Ch, const void* K, const void* Cp,
                        const void* Cc, int32_t* parent_idx, int32_t* code_idx,
                        void* stream);

/*
 * Bytes of the packed aggregates of one (batch, head) (see avq_aggregate) for
 * the given dtype and sizes. Returns -1 for an unknown dtype or sizes outside
 * 1 <= M0 <= 512, 0 <= Ch <= 16, 1 <= d <= 128.
 */
int64_t avq_packed_bytes(avq_dtype_t dtype, int32_t M0, int32_t Ch, int32_t d);

/*
 * avq_aggregate - per-codeword counts and value sums (Eq. (aggregates)).
 *
 * Parent rows p < M0 cover the whole parent cell (every key whose nearest
 * parent is p, whether or not it moved to a child: Alg. 1 adds to the parent
 * unconditionally); child rows M0 + p*Ch + c cover the keys that moved to
 * that child. The parent of a key is code_idx itself when code_idx < M0 and
 * (code_idx - M0) / Ch otherwise.
 *
 *   V         [B][H][N][d]      dtype
 *   code_idx  [B][H][N]         int32, values in [0, Mtot) (as avq_assign writes;
 *                               other values are ignored)
 *   Vbar      [B][H][Mtot][d]   fp32, out, nullable (the sums)
 *   counts    [B][H][Mtot]      int32, out
 *   packed    [B][H][E] bytes, out, nullable; E = avq_packed_bytes(): the
 *             aggregates in the operand layout avq_attention_fwd reads. Codes
 *             are grouped in octets of 8; the octets are, in order, the parents
 *             (parents 8o .. 8o+7, padded with empty octets to a multiple of 8
 *             octets), then for every parent p its ceil(Ch/8) child octets
 *             (children 8j .. 8j+7 of p), then one empty octet. The buffer is
 *               means [n_oct][d][8] in dtype: mean value Vbar/n of each code
 *                     of the octet (0 for n = 0 and for padding slots),
 *                     rounded from fp32;
 *               info  [n_oct][16] fp32: n of each code (slots 0..7) and ln n
 *                     (slots 8..15; -inf for n = 0 and padding);
 *             means first, info right after it.
 * At least one of Vbar and packed must be given.
 *
 * Every sum is accumulated in fp32 by the one workgroup that owns the parent
 * family (matrix products with 0 and 1, in no fixed key order); counts are
 * exact.
 */
avq_status_t avq_aggregate(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N, int32_t d,
                           int32_t M0, int32_t Ch, const void* V, const int32_t* code_idx,
                           float* Vbar, int32_t* counts, void* packed, void* stream);

/*
 * avq_assign_aggregate - Alg. 1 as one precompute: the tree quantisation of
 * avq_assign and the counts and sums of avq_aggregate, with the child compare
 * and the value sums in one pass over each head's keys (Sec. 4.2: the
 * aggregates are formed in the same pass that assigns the keys).
 *
 * Outputs are those of avq_assign followed by avq_aggregate on its codes:
 * parent_idx and code_idx exactly (the same compare routine), counts exactly,
 * Vbar and packed within fp32 summation-order rounding. Two launches: the
 * parent assignment (it writes parent_idx, which the second launch reads),
 * then the child compare and aggregation per (batch, head, range of parent
 * families). Ch = 0, and fp32 with Ch = 16 at d = 128, run avq_assign's
 * kernels and then avq_aggregate's.
 *
 *   K, V         [B][H][N][d]   dtype
 *   Cp           [H][M0][d]     dtype
 *   Cc           [H][M0][Ch][d] dtype (NULL allowed when Ch = 0)
 *   parent_idx   [B][H][N]      int32, out
 *   code_idx     [B][H][N]      int32, out
 *   Vbar, counts, packed        as for avq_aggregate (Vbar or packed may be
 *                               NULL, not both)
 */
avq_status_t avq_assign_aggregate(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N,
                                  int32_t d, int32_t M0, int32_t Ch, const void* K,
                                  const void* V, const void* Cp, const void* Cc,
                                  int32_t* parent_idx, int32_t* code_idx, float* Vbar,
                                  int32_t* counts, void* packed, void* stream);

/*
 * avq_pack_aggregates - the aggregates in the form Alg. 2 takes them (its
 * input: the value sum Vbar and the count n of every code, Eq. (aggregates))
 * packed into the operand layout that avq_attention_fwd reads (the packed
 * buffer described under avq_aggregate). A caller that holds (Vbar, n) from
 * elsewhere reaches the attention kernel through this call.
 *
 * For every code x with n = max(counts[x], 0): mean = Vbar[x] * fl(1/n) in
 * fp32 (0 for n = 0), rounded once to dtype; info n (as a float) and
 * ln n = log2(n) ln 2 (-inf for n = 0); padding slots and the empty octet as
 * in avq_aggregate. This is the aggregation's own arithmetic: the Vbar and
 * counts that avq_aggregate writes pack into exactly its packed output.
 *
 *   Vbar     [B][H][Mtot][d]  fp32, rows as in avq_aggregate (parent rows the
 *                             whole cell, child rows the keys moved there)
 *   counts   [B][H][Mtot]     int32 (negative entries count as 0)
 *   packed   [B][H][E] bytes, out; E = avq_packed_bytes(dtype, M0, Ch, d)
 * Sizes as for avq_aggregate (N does not apply).
 */
avq_status_t avq_pack_aggregates(avq_dtype_t dtype, int32_t B, int32_t H, int32_t d,
                                 int32_t M0, int32_t Ch, const float* Vbar,
                                 const int32_t* counts, void* packed, void* stream);

/*
 * avq_attention_fwd - the fused refined-codebook attention (Alg. 2).
 *
 * Queries are taken in tiles of block_q consecutive tokens (the last tile may
 * be shorter). For each tile I and query i in I:
 *   parent pass  S_ip = Q_i . Cp_p; running max over non-empty parents
 *                (App. D); A_ip = exp(S_ip - m_i), zero for empty parents;
 *                Xbar_i = sum_p A_ip Vbar_p, Zbar_i = sum_p A_ip n_p
 *                (Eq. (vqflashattention));
 *   importance   w_p(I) = sum_{i in I} A_ip n_p / Zbar_i (Eq. (importance));
 *   top-P        the P parents of largest w (lowest index on ties);
 *   children     for every selected p and child c: T_ic = Q_i . Cc_pc; the
 *                running max is raised over non-empty children and Xbar, Zbar
 *                rescaled; the parent logit is recovered as the mean of all Ch
 *                child logits (Eq. (parent_recovery)); the correcting weight
 *                dA = exp(T_ic - m) - exp(Srec_ip - m), zero for empty children
 *                (Eq. (correcting_attention)), adds dA * Vbar_pc to Xbar and
 *                dA * n_pc to Zbar;
 *   output       Y_i = Xbar_i / Zbar_i.
 * P = 0 gives plain VQ attention over the parents (Sec. 3.2).
 *
 *   P            0 <= P <= M0; P = 0 when Ch = 0
 *   block_q      query tile size, 1 <= block_q <= 256 (semantic: importance
 *                and top-P are computed per tile of block_q tokens)
 *   Q            [B][H][N][d]    dtype
 *   Cp, Cc       as in avq_assign (Cc NULL allowed when Ch = 0)
 *   packed       the packed aggregates written by avq_aggregate or by
 *                avq_pack_aggregates (required)
 *   Y            [B][H][N][d]    dtype, out
 *   topp_idx     [B][H][T][P]    int32, out, nullable; T = ceil(N / block_q);
 *                the selected parents in the order importance descending,
 *                index ascending
 *   importance   [B][H][T][M0]   fp32, out, nullable; w_p(I) of every parent
 *
 * The kernel uses the log-count bias of App. D: a code's weight is
 * exp(S + ln n - m) applied to its mean value Vbar/n, which equals
 * exp(S - m) applied to Vbar; empty codes (n = 0) drop out without masks.
 *
 * Arithmetic: bf16 inputs use bf16 MFMA with fp32 accumulation (the weights
 * and the mean values are bf16 MFMA operands; softmax state, importance and
 * all sums stay fp32); fp32 inputs use fp32 MFMA throughout.
 */
avq_status_t avq_attention_fwd(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N,
                               int32_t d, int32_t M0, int32_t Ch, int32_t P,
                               int32_t block_q, const void* Q, const void* Cp,
                               const void* Cc, const void* packed, void* Y,
                               int32_t* topp_idx, float* importance,
                               void* stream);

/* Parents per codeword tile of avq_attention_fwd_tiled. */
#define AVQ_IMPORTANCE_TILE 64

/*
 * avq_attention_fwd_tiled - avq_attention_fwd with the importance of App. B
 * (computing importance with tiled codewords), in one parent sweep.
 *
 * The parents are visited in tiles of AVQ_IMPORTANCE_TILE (parents
 * 64t .. 64t+63). After tile J the partial denominator of query i, the sum of
 * A_ip n_p over the parents of tiles up to J, is extrapolated to all keys
 * (Eq. (aproxdenom)): Ztilde_i(J) = N / N_seen(J) * partial, N_seen(J) being
 * the number of keys whose parent lies in those tiles; the importance of each
 * parent p of tile J is w_p(I) = sum_{i in I} A_ip n_p / Ztilde_i(J)
 * (Eq. (codewordimportance)). A tile whose parents hold no key adds nothing.
 * The last tile has N_seen = N, so with M0 <= AVQ_IMPORTANCE_TILE this is
 * Eq. (importance) and the call equals avq_attention_fwd. Top-P, the child
 * pass and the output are as in avq_attention_fwd, on this importance.
 *
 * Arguments, layouts, ownership, arithmetic and errors as avq_attention_fwd
 * (importance, when given, receives this w).
 */
avq_status_t avq_attention_fwd_tiled(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N,
                                     int32_t d, int32_t M0, int32_t Ch, int32_t P,
                                     int32_t block_q, const void* Q, const void* Cp,
                                     const void* Cc, const void* packed, void* Y,
                                     int32_t* topp_idx, float* importance, void* stream);

/*
 * avq_attention_fwd_ordered - avq_attention_fwd (tiled_importance = 0) or
 * avq_attention_fwd_tiled (tiled_importance = 1) with the queries taken in
 * the order query_order instead of token order: query tile t is the tokens
 * query_order[t*block_q .. t*block_q + block_q - 1]. The result equals
 * permuting the rows of Q by query_order, calling the unordered entry point
 * and writing each output row back to its token: Y[b][h][query_order[k]] is
 * the output of query position k. The reordering is the one the paper
 * applies before tiling (Sec. 4, along a space-filling curve; see
 * avq_gilbert_order), so that the tokens of a tile, which share one top-P
 * selection, are spatial neighbours. Keys, values and the aggregates are
 * order-free (Sec. 3.2) and are not reordered.
 *
 *   query_order  [N] int32, device, a permutation of 0 .. N-1 shared by every
 *                batch entry and head. An entry outside [0, N) makes that
 *                query position take no part (no output row is written for
 *                it); a repeated entry writes that token's row more than once,
 *                in an unspecified order, and leaves some token unwritten.
 *   topp_idx, importance  per tile of the ORDERED queries.
 * Other arguments, layouts, ownership and errors as avq_attention_fwd.
 */
avq_status_t avq_attention_fwd_ordered(avq_dtype_t dtype, int32_t B, int32_t H, int32_t N,
                                       int32_t d, int32_t M0, int32_t Ch, int32_t P,
                                       int32_t block_q, const int32_t* query_order,
                                       int32_t tiled_importance, const void* Q, const void* Cp,
                                       const void* Cc, const void* packed, void* Y,
                                       int32_t* topp_idx, float* importance, void* stream);

/*
 * avq_gilbert_order - host helper: the cells of a width x height grid of
 * tokens (token y*width + x) in the order of a generalized Hilbert curve
 * (the Gilbert curve the paper reorders tokens along, Sec. 4,
 * Fig. per-tile adaptivity, App. spatial reordering ablation).
 *
 * The curve starts at cell (0, 0), visits every cell once, and each step
 * moves to a 4-neighbour, except for at most one diagonal step on some grids
 * with odd sides; on a 2^k x 2^k grid it is a Hilbert curve. Any run of
 * consecutive cells therefore covers a compact region, whatever the tile size.
 *
 *   width, height  grid sizes, >= 1, width*height <= 2^24
 *   order          [width*height] int32, HOST, out: order[k] = token of the
 *                  k-th cell (the query_order of avq_attention_fwd_ordered)
 *   rank           [width*height] int32, HOST, out, nullable: the inverse,
 *                  rank[order[k]] = k
 * Runs on the host only (no device call); copy order to the device once.
 */
avq_status_t avq_gilbert_order(int32_t width, int32_t height, int32_t* order, int32_t* rank);

/*
 * avq_codebook_update - one step of the codebook's exponential moving
 * averages under the parent-child constraint (App. A).
 *
 * The batch statistics are the aggregates of the KEYS (avq_aggregate called
 * with K in place of V, after avq_assign): sums[b][h][x] is the sum of the
 * keys with code x in batch entry b (a parent row covers its whole cell) and
 * counts[b][h][x] their number. For every head h (one codebook per head,
 * shared by the batch) and code x, summing over b in order:
 *   S_x <- lambda S_x + (1 - lambda) sum_b sums[b][h][x]
 *   N_x <- lambda N_x + (1 - lambda) sum_b counts[b][h][x]
 * Parents take the unconstrained mean C_p = S_p / N_p. The Ch children of p,
 * with means M_c = S_c / N_c, are projected onto the constraint that their
 * mean is C_p by the mass-weighted least-squares solution
 * (Eq. (child_constraint_solve)):
 *   delta = sum_c M_c - Ch C_p,  sigma = sum_c 1 / N_c,
 *   C_pc  = M_c - delta / (N_c sigma).
 *
 *   lambda   EMA decay, 0 < lambda <= 1 (else AVQ_ERR_INVALID_ARG)
 *   sums     [B][H][Mtot][d]  fp32 (the Vbar output of avq_aggregate on K)
 *   counts   [B][H][Mtot]     int32 (its counts)
 *   S        [H][Mtot][d]     fp32, in/out: the EMA key sums
 *   Nema     [H][Mtot]        fp32, in/out: the EMA counts; must be positive
 *                             on entry (then they stay positive); a
 *                             non-positive mass gives non-finite codewords
 *   Cp_out   [H][M0][d]       dtype, out: the new parents
 *   Cc_out   [H][M0][Ch][d]   dtype, out: the new children (NULL allowed
 *                             when Ch = 0)
 * Sizes as for the other calls (N does not apply). Arithmetic is fp32, one
 * thread per (family, dimension), batch entries summed in order; counts are
 * exact while the total count of a code stays below 2^24. The codewords are
 * rounded once to dtype.
 */
avq_status_t avq_codebook_update(avq_dtype_t dtype, int32_t B, int32_t H, int32_t d,
                                 int32_t M0, int32_t Ch, float lambda, const float* sums,
                                 const int32_t* counts, float* S, float* Nema, void* Cp_out,
                                 void* Cc_out, void* stream);

/* ---------------------------------------------------------------------------
 * Exact attention of packed prompts, and the paged cache (serving).
 *
 * These calls take tokens of several sequences packed one after the other:
 * rows of tokens, each row its heads [H][d] contiguous, q_stride / k_stride /
 * v_stride elements from one token's row to the next (at least H*d, a multiple
 * of 16 bytes, at most 2^22: slices of a fused projection need no copy).
 * cu [S + 1] (int32, device): sequence s owns rows cu[s] .. cu[s + 1] - 1; cu
 * must not decrease (if it does, outputs are unspecified) and may leave rows
 * behind cu[S], whose outputs are left as they were. Values outside [0, T] are
 * taken as the nearest of 0 and T.
 * Hq query heads share Hkv key-value heads: head h reads h / (Hq / Hkv).
 * Sizes: d in {64, 128}; Hq <= 1024, a multiple of Hkv; S <= 2^20; T <= 2^24
 * packed tokens, 0 included (nothing is then written). Element counts may pass
 * 2^31. An infinity or NaN in a sequence's inputs leaves the outputs of other
 * sequences as they are; the sequence's own are unspecified.
 * The attentions need |q_i . k_j| and |S_ij| log2(e) below 3e38, and values below
 * 2^120 / n in magnitude for n keys: numerators are fp32 sums of values times
 * weights of at most 2^8.
 */

/* Bytes of the workspace of avq_prompt_attention_fwd for these sizes: 0 where
 * it needs none (no query tile's keys are divided: enough tiles to fill the
 * device, or too few keys), -1 for unsupported sizes. Its contents need not be
 * set and mean nothing afterwards; calls that may run at the same time need one
 * each. */
int64_t avq_prompt_attention_workspace(avq_dtype_t dtype, int32_t S, int32_t Tq, int32_t Tk,
                                       int32_t Hq, int32_t d, int32_t causal);

/*
 * avq_prompt_attention_fwd - exact softmax attention (Eq. (standardattention))
 * of packed sequences.
 *
 * With Lq queries and Lk keys in sequence s, S_ij = scale q_i . k_j:
 *   lse_i = ln sum_j exp(S_ij),  Y_i = sum_j exp(S_ij - lse_i) v_j
 * over j < Lk, and with causal = 1 only j <= i + Lk - Lq: the queries are the
 * last Lq of the Lk positions (a whole prompt when Lq = Lk, a chunk behind
 * earlier keys when Lq < Lk). A query that sees no key (Lk = 0, or causal with
 * Lq > Lk + i) gets Y_i = 0 and lse_i = -inf.
 *
 *   scale  > 0, scale log2(e) finite in fp32 (2.35e38);  causal  0 or 1
 *   Q      [Tq] rows of [Hq][d], K, V [Tk] rows of [Hkv][d], dtype
 *   cu_q, cu_k  [S + 1] int32 (they may be one array)
 *   Y      [Tq][Hq][d] dtype, contiguous, out
 *   lse    [Tq][Hq] fp32, out, nullable
 *   workspace  avq_prompt_attention_workspace() bytes, NULL allowed for 0
 * (Tq / 128 + S) * Hq < 2^24. One launch, two with a workspace. Arithmetic as
 * avq_attention_fwd: bf16 products with fp32 accumulation and fp32 softmax
 * state, weights rounded to bf16 for the value product; fp32 throughout for
 * fp32.
 */
avq_status_t avq_prompt_attention_fwd(avq_dtype_t dtype, int32_t S, int32_t Tq, int32_t Tk,
                                      int32_t Hq, int32_t Hkv, int32_t d, float scale,
                                      int32_t causal, const void* Q, int64_t q_stride,
                                      const void* K, int64_t k_stride, const void* V,
                                      int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k,
                                      void* Y, float* lse, void* workspace,
                                      int64_t workspace_bytes, void* stream);

/* Element format of a paged cache: the calls' dtype, or 4 bits. */
typedef int32_t avq_cache_t;
enum { AVQ_CACHE_NATIVE = 0, AVQ_CACHE_FP4 = 1 };

/*
 * Bytes E of one (page, key-value head). The cache is one array
 * [n_pages][Hkv][E]; a page holds page_size (16, 32, 64, 128 or 256)
 * consecutive positions of a sequence:
 *   native  K [page_size][d], V [page_size/8][d][8], dtype
 *   fp4     K codes [page_size][d/2], V codes [page_size/8][d/2][8],
 *           K scales [page_size][d/32], V scales [page_size/8][d/32][8]: bytes.
 *           A code byte holds dimensions 2i (low 4 bits) and 2i+1 of one
 *           position as e2m1: sign, then 0, 0.5, 1, 1.5, 2, 3, 4, 6 for codes
 *           0 .. 7. A scale byte e in 1 .. 254 is 2^(e - 127), shared by 32
 *           dimensions of one position: 4.25 bits per element. Magnitudes of
 *           3.5 2^126 (2.97e38) and more become code 4 at 2^126, which is 2^128:
 *           infinite in avq_cache_attention_fwd.
 * block_table [S][max_pages] (int32, device) names the page of positions
 * i*page_size .. (i+1)*page_size - 1 of each sequence in column i; columns past
 * a sequence's length are not read. A position without a page (past max_pages,
 * or an entry outside [0, n_pages)) is not written by avq_cache_append, reads
 * as 0 in avq_cache_gather and takes no part in avq_cache_attention_fwd.
 * max_pages * page_size <= 2^30. Returns -1 for unsupported arguments.
 */
int64_t avq_cache_page_bytes(avq_dtype_t dtype, avq_cache_t format, int32_t page_size, int32_t d);

/*
 * avq_cache_append - appends new keys and values to the cache, with the keys
 * (and the queries of the same tokens) rotated to their positions.
 *
 * Token i of sequence s (packed row cu[s] + i) has position start[s] + i. The
 * first rot dimensions are rotated in pairs (a, b) = dimensions (i, i + rot/2),
 * or with interleaved = 1 (2i, 2i + 1), i < rot/2, by the angle whose cosine
 * and sine the caller gives for (position, i):
 *   a' = a cos - b sin,  b' = b cos + a sin      (fp32)
 * Rotated queries and keys are rounded once to dtype. In the 4-bit cache each
 * 32 dimensions of a rotated key (before that rounding) and of a value take
 * the smallest power-of-two scale that leaves no magnitude above 6, and every
 * element the nearest code (ties to the even code).
 *
 *   rot          0 (no rotation; cos, sin and n_pos are then not used) or a
 *                multiple of 16 up to d
 *   cos, sin     [n_pos][rot/2] fp32; nothing is written for a token whose
 *                position lies outside [0, n_pos)
 *   Q            [T] rows of [Hq][d], nullable with Q_out (Hq and q_stride are
 *                then not used)
 *   K, V         [T] rows of [Hkv][d], dtype
 *   cu           [S + 1]; NULL: one token per sequence, T = S
 *   start        [S] int32, tokens already cached; a negative one makes the
 *                sequence take no part
 *   block_table  [S][max_pages] int32; the pages of the call's positions must
 *                be pairwise different (shared pages are read only)
 *   cache        [n_pages][Hkv][E], in/out: only the new positions are written
 *   Q_out        [T][Hq][d] dtype, out (may be Q itself if Q is contiguous)
 *   K_out        [T][Hkv][d] dtype, out, nullable: the rotated keys (may be K
 *                itself if K is contiguous)
 * One launch. Otherwise outputs overlap no input.
 */
avq_status_t avq_cache_append(avq_dtype_t dtype, avq_cache_t format, int32_t S, int32_t T,
                              int32_t Hq, int32_t Hkv, int32_t d, int32_t n_pages,
                              int32_t page_size, int32_t max_pages, int32_t rot, int32_t n_pos,
                              int32_t interleaved, const void* Q, int64_t q_stride, const void* K,
                              int64_t k_stride, const void* V, int64_t v_stride,
                              const int32_t* cu, const int32_t* start, const int32_t* block_table,
                              const float* cos, const float* sin, void* cache, void* Q_out,
                              void* K_out, void* stream);

/*
 * avq_cache_gather - cached positions read back as packed rows: row cu[s] + i
 * is position start[s] + i of sequence s, in dtype (4-bit values are exact in
 * either type, but 2^128 is read as the type's largest finite value). Positions
 * below 0 read as 0, like those without a page. With start = 0 and cu the cached
 * lengths these are the K and V that avq_prompt_attention_fwd takes for a chunk
 * behind a cached prefix.
 *
 *   cu           [S + 1], start [S], block_table [S][max_pages]: int32
 *   K, V         [T][Hkv][d] dtype, contiguous, out
 */
avq_status_t avq_cache_gather(avq_dtype_t dtype, avq_cache_t format, int32_t S, int32_t T,
                              int32_t Hkv, int32_t d, int32_t n_pages, int32_t page_size,
                              int32_t max_pages, const void* cache, const int32_t* cu,
                              const int32_t* start, const int32_t* block_table, void* K, void* V,
                              void* stream);

/* Bytes of the workspace of avq_cache_attention_fwd (-1 for unsupported
 * sizes). Its contents need not be set and mean nothing afterwards; calls that
 * may run at the same time need one each. A cache with room for few positions
 * per sequence (max_pages * page_size <= AVQ_CACHE_UNDIVIDED) needs none. */
enum { AVQ_CACHE_UNDIVIDED = 512 };
int64_t avq_cache_attention_workspace(int32_t S, int32_t n_q, int32_t Hq, int32_t Hkv, int32_t d);

/*
 * avq_cache_attention_fwd - exact softmax attention of the n_q newest tokens of
 * every sequence over its cache (single tokens: n_q = 1).
 *
 * lens[s] positions of sequence s are cached, the n_q tokens' own keys and
 * values among them (appended before). Token i < n_q sees the positions
 * j < lens[s] - (n_q - 1 - i). Y and lse as in avq_prompt_attention_fwd; a
 * token that sees no position (lens[s] = 0: an idle entry of a padded batch)
 * gets 0 and -inf. lens is taken as at least 0 and at most
 * max_pages * page_size; S * max_pages * page_size <= 2^37 and
 * S * Hkv * ceil(n_q * Hq / Hkv / 16) < 2^24.
 *
 *   n_q          1 .. 16;  scale  as in avq_prompt_attention_fwd
 *   Q            [S * n_q] rows of [Hq][d], dtype, q_stride as above
 *   cache, block_table  as above; lens [S] int32
 *   Y            [S][n_q][Hq][d] dtype, out;  lse [S][n_q][Hq] fp32, nullable
 *   workspace    avq_cache_attention_workspace() bytes; NULL allowed (it is
 *                not used) if max_pages * page_size <= AVQ_CACHE_UNDIVIDED
 * Two launches, one where no workspace is needed. What lies in cache slots
 * behind a sequence's length has no effect, whatever it is.
 */
avq_status_t avq_cache_attention_fwd(avq_dtype_t dtype, avq_cache_t format, int32_t S, int32_t n_q,
                                     int32_t Hq, int32_t Hkv, int32_t d, int32_t n_pages,
                                     int32_t page_size, int32_t max_pages, float scale,
                                     const void* Q, int64_t q_stride, const void* cache,
                                     const int32_t* lens, const int32_t* block_table, void* Y,
                                     float* lse, void* workspace, int64_t workspace_bytes,
                                     void* stream);

/* ---------------------------------------------------------------------------
 * Rotary positions with several axes, and cross attention (serving and training).
 * Packed rows, strides and sizes as for avq_prompt_attention_fwd.
 */

/*
 * avq_rotate_axes - rotates the queries, and keys, of packed tokens by their
 * positions on several axes (time, height and width of a video's patches, say),
 * or back.
 *
 * Token t has n_axes positions pos[t][0 .. n_axes-1]. Pair i of every head, i <
 * rot/2, is dimensions (i, i + rot/2), or with interleaved = 1 (2i, 2i + 1), as
 * in avq_cache_append; it turns by the angle of column i of the tables at the
 * token's position on axis[i]: with p = pos[t][axis[i]],
 *   a' = a cos[p][i] - b sin[p][i],  b' = b cos[p][i] + a sin[p][i]   (fp32)
 * and with inverse = 1 by the opposite angle, -sin in place of sin: that takes
 * gradients of the rotated rows to gradients of the rows. Results are rounded once
 * to dtype; dimensions from rot on are copied. Nothing is written for a token that
 * has a position outside [0, n_pos).
 *
 *   rot          a multiple of 16 in [16, d]
 *   n_axes       1 .. AVQ_MAX_AXES
 *   axis         [rot/2] bytes, HOST, each below n_axes: any order of the axes
 *   Q            [T] rows of [Hq][d], dtype
 *   K            [T] rows of [Hkv][d], nullable with K_out (Hkv and k_stride are
 *                then not used)
 *   pos          [T][n_axes] int32
 *   cos, sin     [n_pos][rot/2] fp32
 *   Q_out, K_out [T][Hq][d], [T][Hkv][d] dtype, contiguous, out (may be Q and K
 *                themselves if these are contiguous; otherwise they overlap no input)
 * T <= 2^24, 0 included. One launch. axis has been read when the call returns.
 */
enum { AVQ_MAX_AXES = 4 };
avq_status_t avq_rotate_axes(avq_dtype_t dtype, int32_t T, int32_t Hq, int32_t Hkv, int32_t d,
                             int32_t rot, int32_t n_axes, const uint8_t* axis, int32_t n_pos,
                             int32_t interleaved, int32_t inverse, const void* Q, int64_t q_stride,
                             const void* K, int64_t k_stride, const int32_t* pos, const float* cos,
                             const float* sin, void* Q_out, void* K_out, void* stream);

/*
 * avq_cross_attention_fwd - exact softmax attention of packed queries over the
 * states of an encoder (or any others) of another length.
 *
 * Source s has queries cu_q[s] .. cu_q[s+1]-1 and states cu_k[s] .. cu_k[s+1]-1;
 * the queries of all sequences that read a source are simply packed together. With
 * S_ij = scale q_i . k_j over the states j of i's source that take part:
 *   lse_i = ln sum_j exp(S_ij),  Y_i = sum_j exp(S_ij - lse_i) v_j
 * A query that sees no state gets Y_i = 0 and lse_i = -inf. Query head h reads
 * key-value head h / (Hq / Hkv).
 *
 *   Q            [Tq] rows of [Hq][d], K, V [Tk] rows of [Hkv][d], dtype
 *   cu_q, cu_k   [S + 1] int32, as in avq_prompt_attention_fwd
 *   mask         [Tk] bytes, nullable, of any alignment: states with a 0 take no
 *                part, whatever their rows of K and V hold (infinities and NaN too)
 *   Y            [Tq][Hq][d] dtype, contiguous, out
 *   lse          [Tq][Hq] fp32, out, nullable (avq_cross_attention_bwd takes it)
 *   workspace    avq_cross_attention_workspace() bytes, NULL allowed for 0
 * Sizes: (Tq Hq / Hkv / 128 + S) Hkv and (Tk / 128 + S) Hkv below 2^24. One launch,
 * two with a workspace. Arithmetic and limits as avq_prompt_attention_fwd.
 */
avq_status_t avq_cross_attention_fwd(avq_dtype_t dtype, int32_t S, int32_t Tq, int32_t Tk,
                                     int32_t Hq, int32_t Hkv, int32_t d, float scale, const void* Q,
                                     int64_t q_stride, const void* K, int64_t k_stride,
                                     const void* V, int64_t v_stride, const int32_t* cu_q,
                                     const int32_t* cu_k, const uint8_t* mask, void* Y, float* lse,
                                     void* workspace, int64_t workspace_bytes, void* stream);

/* Bytes of the workspaces of the cross attention calls (0: none needed, -1:
 * unsupported sizes). Their contents need not be set and mean nothing afterwards;
 * calls that may run at the same time need one each. */
int64_t avq_cross_attention_workspace(avq_dtype_t dtype, int32_t S, int32_t Tq, int32_t Tk,
                                      int32_t Hq, int32_t Hkv, int32_t d);
int64_t avq_cross_attention_bwd_workspace(avq_dtype_t dtype, int32_t S, int32_t Tq, int32_t Tk,
                                          int32_t Hq, int32_t Hkv, int32_t d);

/*
 * avq_cross_attention_bwd - gradients of avq_cross_attention_fwd's Y with respect
 * to Q, K and V, from dY, that of the result with respect to Y. With P_ij =
 * exp(S_ij - lse_i) and dS_ij = P_ij (dY_i . v_j - dY_i . Y_i):
 *   dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i,  dV_j = sum_i P_ij dY_i
 * The sums over i take all queries of the source and all heads that share the
 * key-value head. Queries that see no state get dQ = 0, states that take no part or
 * are read by no query dK = dV = 0; rows that belong to no source are left as they
 * were. The same inputs give the same bits at every call.
 *
 *   dY           [Tq] rows of [Hq][d], dtype; dy_stride as the others
 *   Q, K, V, cu_q, cu_k, mask, scale  those of the forward call
 *   Y, lse       its results ([Tq][Hq][d], [Tq][Hq], contiguous)
 *   dQ           [Tq][Hq][d], dK, dV [Tk][Hkv][d], dtype, contiguous, out
 *   workspace    avq_cross_attention_bwd_workspace() bytes
 * Sizes as the forward call. Two to four launches. bf16: products with fp32
 * accumulation; P and dS, fp32, are rounded to bf16 for the products they enter, and
 * dY_i . Y_i, off by Y's rounding, is mended by the sum of dS, which is 0. fp32: fp32
 * throughout. P is taken from lse, whose rounding leaves a relative error of |lse| 2^-23
 * in it: 10^-4 for logits of a thousand, a tenth for a million.
 */
avq_status_t avq_cross_attention_bwd(avq_dtype_t dtype, int32_t S, int32_t Tq, int32_t Tk,
                                     int32_t Hq, int32_t Hkv, int32_t d, float scale,
                                     const void* dY, int64_t dy_stride, const void* Q,
                                     int64_t q_stride, const void* K, int64_t k_stride,
                                     const void* V, int64_t v_stride, const void* Y,
                                     const float* lse, const int32_t* cu_q, const int32_t* cu_k,
                                     const uint8_t* mask, void* dQ, void* dK, void* dV,
                                     void* workspace, int64_t workspace_bytes, void* stream);

/* Bytes of the workspace of avq_cache_prefix_attention_fwd (-1: unsupported
 * sizes). Its contents need not be set and mean nothing afterwards; calls that may
 * run at the same time need one each. */
int64_t avq_cache_prefix_attention_workspace(int32_t S, int32_t n_groups, int32_t n_q, int32_t Hq,
                                             int32_t Hkv, int32_t d);

/*
 * avq_cache_prefix_attention_fwd - avq_cache_attention_fwd for groups of sequences
 * that share their first positions (several answers to one long prompt): those are
 * attended to once for the whole group, and read once.
 *
 * Group g is the sequences cu_groups[g] .. cu_groups[g+1]-1 of the batch, whose
 * first shared[g] positions are the same ones: their block tables may name the same
 * pages for them, or copies (of the page in which the shared positions end, say).
 * Positions below P_g = min(shared[g], lens[cu_groups[g]]) are read through the
 * table of the group's first sequence, for all of its sequences (where sharing does
 * not pay, through each one's own; a group whose sequences do not hold the same there
 * gets unspecified outputs). A group of one sequence, sequences of no group, and those
 * that hold fewer than P_g positions share nothing. If the first sequence of a group
 * is idle (lens 0), so is the sharing: P_g = 0, and every sequence reads its own pages;
 * put one that is not idle first.
 * Y and lse are those of avq_cache_attention_fwd on the same arguments, but for the
 * rounding of the sums.
 *
 *   cu_groups    [n_groups + 1] int32; it must not decrease (if it does, outputs are
 *                unspecified); values outside [0, S] are taken as the nearest
 *   shared       [n_groups] int32, below 0: none
 *   others       as avq_cache_attention_fwd
 *   workspace    avq_cache_prefix_attention_workspace() bytes; NULL allowed if
 *                max_pages * page_size <= AVQ_CACHE_UNDIVIDED (nothing is then shared)
 * n_groups >= 1; (S n_q Hq / Hkv / 128 + n_groups) Hkv < 2^24. Two launches, one without a
 * workspace. It pays in batches of dozens of sequences, four or more a group (in 4 bits
 * eight), that share thousands of positions. In smaller batches and groups, with shorter
 * shared parts, or where most positions are the sequences' own, avq_cache_attention_fwd is
 * as fast or faster (32 pairs in 4 bits: up to four times): the choice is the caller's.
 */
avq_status_t avq_cache_prefix_attention_fwd(avq_dtype_t dtype, avq_cache_t format, int32_t S,
                                            int32_t n_groups, int32_t n_q, int32_t Hq, int32_t Hkv,
                                            int32_t d, int32_t n_pages, int32_t page_size,
                                            int32_t max_pages, float scale, const void* Q,
                                            int64_t q_stride, const void* cache,
                                            const int32_t* lens, const int32_t* block_table,
                                            const int32_t* cu_groups, const int32_t* shared,
                                            void* Y, float* lse, void* workspace,
                                            int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* AVQ_H */
