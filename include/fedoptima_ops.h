/*
 * fedoptima_ops.h -- transformer operators of libfedoptima for networks beyond
 * the built-in configurations: masked attention with its gradients, a learned
 * bias by distance, dropout, and what stands around them in a language model:
 * embedding, RMS norm, products of 8-bit rows, log probabilities of tokens with
 * the cross-entropy, and a preference loss.
 *
 * A server that trains a transformer of its own (another width, longer
 * sequences, causal or prefix language models, grouped key heads, dropout)
 * builds its step from these calls and the products of fedoptima_kernels.h.
 *
 * Conventions, beside those of fedoptima.h:
 *   - Each call enqueues its kernels on `hip_stream` and returns at once.  It
 *     allocates nothing, synchronises nothing and may be captured into a HIP
 *     graph.  Scratch memory is the caller's: `workspace` (device, 16-byte
 *     aligned) of at least the bytes that the *_workspace call returns; its
 *     contents need not be kept between calls.
 *   - Arguments are checked on the host (FO_EINVAL before any launch).
 *   - dtype names the type of all operands and results of a call; sums, softmax
 *     statistics and the workspace are fp32.  In bf16 the operands of the matrix
 *     products are bf16 too: probabilities (after dropout) before their products
 *     with v and dout, score gradients before theirs with q and k are rounded once
 *     (heads of up to eight columns keep them in fp32).  The tanh of a cap is
 *     within 2^-19 in bf16 calls, 2^-22 in fp32 calls, so that a score is within
 *     that times the cap.
 *   - Results do not depend on timing: no sum's order varies between calls.
 */
#ifndef FEDOPTIMA_OPS_H
#define FEDOPTIMA_OPS_H

#include "fedoptima.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FO_DT_BF16 = 0,   /* uint16 bit patterns */
       FO_DT_F32 = 1 };

/* ------------------------------------------------------------------ attention
 * For sequence b, head h (key head h / (heads / kv_heads)), query i and key j of
 * Lq queries and Lk keys, the last query standing at the last key:
 *
 *   n = j - i - (Lk - Lq)                          distance
 *   c = cap tanh(scale q_i.k_j / cap)              (scale q_i.k_j if cap == 0)
 *   u = c + table[bucket[clamp(n, -radius, radius) + radius]][h]
 *   P = softmax of u over the keys that i sees     (FO_ATTN_*)
 *   out_i = sum_j P_ij drop_ij v_j                 drop = 0 or 1 / (1 - p)
 *
 * A bias of -1e30 or less (-infinity, a type's lowest value) hides its distances
 * as the mask does.  A query that sees no key has out = 0 and takes no part in
 * any gradient.
 *
 * drop_ij comes from the generator below: call (c0, c1, c2, c3) = (2 (j / 16) +
 * (j / 4) % 2, i, b heads + h, offset) of the key `seed` gives eight 16-bit
 * numbers (low halves first), of which number j % 4 + 4 ((j / 8) % 2) decides.
 */
enum { FO_ATTN_FULL = 0,     /* every key of the sequence                          */
       FO_ATTN_CAUSAL = 1,   /* keys with n <= 0                                   */
       FO_ATTN_PREFIX = 2 }; /* those and the first prefix[b] keys of the sequence */

typedef struct {
    int32_t dtype;                       /* FO_DT_*                                            */
    int32_t batch, heads, kv_heads;      /* kv_heads divides heads                             */
    int32_t head_dim;                    /* 1..128                                             */
    int32_t max_q, max_k;                /* upper bounds of the sequences' lengths: queries,
                                          * and keys of a backward pass, up to 2^20; keys 2^30 */
    int64_t q_rows, k_rows;              /* rows of q and out, of k and v                      */
    /* Sequence b: query rows [q_begin[b], q_end[b]), key rows [k_begin[b],
     * k_end[b]), device int32[batch] each.  Rows packed by offsets cu[batch + 1]:
     * begin = cu, end = cu + 1; a cache of fixed rooms: begin = b room, end =
     * begin + length.  No two sequences share query rows, nor, in the backward
     * pass, key rows.  Rows of no sequence are neither read nor written.  The
     * values are not checked: the kernels clamp them to the rows there are and
     * the lengths to max_q and max_k. */
    const int32_t *q_begin, *q_end, *k_begin, *k_end;
    /* Element (row r, head h, d) of x is at x[r x_ld + h x_hs + d], strides in
     * elements; no two elements share an address (FO_EINVAL).  Results share no
     * memory with operands or with each other. */
    int64_t q_ld, q_hs, k_ld, k_hs, v_ld, v_hs, out_ld, out_hs;
    float scale;                         /* usually 1 / sqrt(head_dim)                         */
    float cap;                           /* >= 0; 0: scores are not capped.  scale log2(e),
                                          * cap log2(e) and scale / cap have to be finite in
                                          * fp32                                               */
    int32_t mask;                        /* FO_ATTN_*                                          */
    const int32_t* prefix;               /* FO_ATTN_PREFIX: device int32[batch]                */
    const void* table;                   /* bias [n_buckets][heads], or NULL for none          */
    const int32_t* bucket;               /* device int32[2 radius + 1], clamped to the buckets */
    int32_t n_buckets, radius;           /* 1..1024; 0..1024                                   */
    float p;                             /* dropout of the probabilities, [0, 1)               */
    uint64_t seed;
    uint32_t offset;                     /* another for each layer and step                    */
} fo_attn;

/* Bytes of workspace for fo_attn_fwd (backward == 0), or for either call
 * (backward != 0).  Host only.  -1 on bad arguments. */
FO_API int64_t fo_attn_workspace(const fo_attn* a, int32_t backward);

/* Forward.  lse (device fp32 [heads][q_rows], may be NULL) receives the base-2
 * logarithm of sum_j exp(u_ij), -infinity for a query that sees no key: the
 * backward pass needs it.  Rows of no sequence may hold anything, and so may the
 * rows of a cache past a sequence's end.  The rows of a sequence have to be
 * finite, those that the mask or the bias hides too: a probability of zero still
 * multiplies its value row, as in a product of matrices.  Errors: FO_EINVAL,
 * FO_EHIP. */
FO_API fo_status fo_attn_fwd(const fo_attn* a, const void* q, const void* k, const void* v, void* out, float* lse,
                             void* workspace, int64_t workspace_bytes, void* hip_stream);

/* Backward.  q, k, v as in the forward call, out and lse as it left them, dout
 * with out's strides.  dq, dk, dv have the strides of q, k and v; every row of
 * a sequence is written (a shared key head gets the sum over its heads).
 * The rows of a sequence in out, lse and dout have to be finite as those of q, k
 * and v (lse apart where it is -infinity).
 * dtable ([n_buckets][heads], may be NULL without a table; else required)
 * receives the table's gradient, 0 for buckets that no visible pair has.
 * Errors: FO_EINVAL, FO_EHIP. */
FO_API fo_status fo_attn_bwd(const fo_attn* a, const void* q, const void* k, const void* v, const void* out,
                             const float* lse, const void* dout, void* dq, void* dk, void* dv, void* dtable,
                             void* workspace, int64_t workspace_bytes, void* hip_stream);

/* Buckets of the distances -radius..radius (host int32[2 radius + 1]) for a
 * learned bias: with `half` buckets for a direction (all of them if causal,
 * else half), distances below near = half / 2 get one each, and distance a >=
 * near gets min(half - 1, near + floor(log(a / near) / log(radius / near)
 * (half - near))), a power boundary counting as reached.  Later keys (n > 0) use
 * the second half of the buckets, or, if causal, bucket 0.  Host only.  Errors:
 * FO_EINVAL (fewer than 2 buckets for a direction, an odd number of them for
 * two, radius <= near). */
FO_API fo_status fo_relpos_buckets(int32_t n_buckets, int32_t radius, int32_t causal, int32_t* out);

/* ------------------------------------------------------------------ dropout
 * y = drop (x + bias) + residual over [rows][cols], drop = 0 or 1 / (1 - p) per
 * element, p taken to the nearest multiple of 2^-16, at most 65535 of them (drop
 * if the element's 16-bit number is below 65536 p).  The mask is never stored: the backward pass draws
 * it again from (seed, offset).
 *
 * Generator: Philox 4x32 with seven rounds (Salmon, Moraes, Dror and Shaw,
 * "Parallel random numbers: as easy as 1, 2, 3", 2011), four counter words, the
 * key `seed`.  Element (r, c) takes number c % 8 of the eight 16-bit numbers
 * (low halves first) of call (n % 2^32, n / 2^32, 0, offset), n = r ceil(cols /
 * 8) + c / 8: the mask depends on rows, columns, seed and offset alone.
 *
 * bias ([cols]) and residual may be NULL; y may be x or residual, with its row
 * stride.  ld: row strides in elements, >= cols.  Errors: FO_EINVAL, FO_EHIP. */
FO_API fo_status fo_dropout_fwd(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld,
                                const void* bias, const void* residual, int64_t res_ld, float p, uint64_t seed,
                                uint32_t offset, void* y, int64_t y_ld, void* hip_stream);

/* dx = drop dy (the residual's gradient is dy itself); dbias ([cols], may be
 * NULL) = the column sums of drop dy before their rounding, and needs the
 * workspace.  dx may be dy, with its row stride. */
FO_API int64_t fo_dropout_workspace(int64_t rows, int32_t cols);
FO_API fo_status fo_dropout_bwd(int32_t dtype, int64_t rows, int32_t cols, const void* dy, int64_t dy_ld, float p,
                                uint64_t seed, uint32_t offset, void* dx, int64_t dx_ld, void* dbias,
                                void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ embedding
 * out_r = scale table[tokens[r]] over rows of `cols` elements; a token outside
 * [0, vocab) (padding) has a row of zeros and takes part in no gradient.  tokens:
 * device int32[rows].  ld: row strides in elements, >= cols.  cols up to 2^22.  The product is
 * rounded once.  Errors: FO_EINVAL, FO_EHIP. */
FO_API fo_status fo_embed_fwd(int32_t dtype, int64_t rows, int32_t cols, int32_t vocab, const int32_t* tokens,
                              const void* table, int64_t table_ld, float scale, void* out, int64_t out_ld,
                              void* hip_stream);

/* dtable_v = scale * the sum of dout's rows of token v; every row of dtable is
 * written (0 for tokens that do not come).  accumulate !=
 * 0 adds to what dtable holds instead (a table that is the output's weights too)
 * and leaves the rows of other tokens as they are.  Sums are fp32 and rounded
 * once, after that addition.  rows up to 2^28. */
FO_API int64_t fo_embed_workspace(int64_t rows, int32_t cols, int32_t vocab);
FO_API fo_status fo_embed_bwd(int32_t dtype, int64_t rows, int32_t cols, int32_t vocab, const int32_t* tokens,
                              const void* dout, int64_t dout_ld, float scale, int32_t accumulate, void* dtable,
                              int64_t dtable_ld, void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ RMS norm
 * For each row of [rows][cols]:
 *
 *   h = x + residual                       residual may be NULL
 *   rstd = 1 / sqrt(mean h^2 + eps)
 *   y = h rstd w                           w [cols], may be NULL: ones
 *
 * h (may be NULL) and rstd (fp32 [rows], may be NULL) are what the backward pass
 * needs; h is x itself without a residual.  y is computed from h before h is
 * rounded.  y or h may be x or residual, with its row stride; y is not h.
 * eps >= 0.  A row of zeros has y = 0, with eps = 0 too.  Squares are summed in fp32:
 * |h| has to stay below 1e19 over the root of cols, and above 1e-19 where eps = 0.
 * Errors: FO_EINVAL, FO_EHIP. */
FO_API fo_status fo_rmsnorm_fwd(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld,
                                const void* residual, int64_t res_ld, const void* w, float eps, void* h, int64_t h_ld,
                                void* y, int64_t y_ld, float* rstd, void* hip_stream);

/* With g = dy w:  dx = dres + rstd (g - h rstd^2 mean(g h)), the gradient of x
 * and of residual alike, and dw_c = sum over the rows of dy h rstd.  dres (may be
 * NULL) is the gradient that reaches h on its other way.  h as stored (x without
 * a residual).  dx may be dy, dres or h, with its row stride.  dw ([cols], may be
 * NULL) needs the workspace. */
FO_API int64_t fo_rmsnorm_workspace(int64_t rows, int32_t cols);
FO_API fo_status fo_rmsnorm_bwd(int32_t dtype, int64_t rows, int32_t cols, const void* dy, int64_t dy_ld,
                                const void* h, int64_t h_ld, const void* w, const float* rstd, const void* dres,
                                int64_t dres_ld, void* dx, int64_t dx_ld, void* dw, void* workspace,
                                int64_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ 8-bit rows
 * A row in 8 bits is e4m3 (4 exponent and 3 mantissa bits, no infinity, largest
 * 448), one byte an element, with one fp32 scale: element c stands for scale
 * y8[c].  scale = max |y| / 448, and y8 = y 448 / max |y| rounded to nearest even.
 * A row of zeros has scale 0.  Rows whose largest element is below 2^-100 are
 * divided by 2^-100 in its place.  A row that holds NaN or infinities gets a scale
 * or elements that are NaN; other rows do not notice.
 *
 * fo_rmsnorm_f8: the forward norm above with y in 8 bits (for the next product, in
 * passes without a gradient).  fo_quant_f8: the rows of x themselves (weights,
 * other activations). */
FO_API fo_status fo_rmsnorm_f8(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld,
                               const void* residual, int64_t res_ld, const void* w, float eps, void* h, int64_t h_ld,
                               uint8_t* y8, int64_t y8_ld, float* y_scale, void* hip_stream);
FO_API fo_status fo_quant_f8(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld, uint8_t* y8,
                             int64_t y8_ld, float* y_scale, void* hip_stream);

/* c_mn = a_scale[m] b_scale[n] sum_k a_mk b_nk, a [M][K] and b [N][K] in 8 bits,
 * summed in fp32 and rounded once to dtype.  a_scale [M] and b_scale [N] may be
 * NULL (ones); the sum is multiplied by a_scale first, in fp32.  M >= 0; N, K >= 1.  In bf16 calls the products enter those sums by
 * eights, each cut below 2^-13 of the largest of its eight (the 8-bit matrix
 * instruction's way: some 1.4e-5 of the result's norm); fp32 calls keep all bits of
 * the products and take about twice as long.  Rows that start 16-byte aligned with
 * K a multiple of 16 are read as they lie; with another K the workspace has room
 * for copies that are; strides below 2^23 that are no multiple of 16 beside such a K
 * cost most. */
FO_API int64_t fo_gemm_f8_workspace(int64_t M, int32_t N, int32_t K);
FO_API fo_status fo_gemm_f8(int32_t dtype, int64_t M, int32_t N, int32_t K, const uint8_t* a, int64_t lda,
                            const float* a_scale, const uint8_t* b, int64_t ldb, const float* b_scale, void* c,
                            int64_t ldc, void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ log probabilities
 * For row r of logits [rows][vocab] with target t = targets[r] (device int32):
 *
 *   z = scale logits_r                     scale > 0, scale log2(e) finite in fp32
 *   lse[r] = log sum_v exp(z_v)            natural logarithm
 *   logp[r] = z_t - lse[r]
 *
 * A row whose target is outside [0, vocab) is ignored: it is not read, logp = lse =
 * 0, and its gradient is 0.  Logits of -infinity count as probability 0; a row of
 * nothing else has logp = lse = -infinity and no gradient.  logp and lse are fp32
 * (lse may be NULL in the forward call).  The terms other than the target's are
 * summed apart, so that logp near 0 and its gradient keep their leading bits.
 * Errors: FO_EINVAL, FO_EHIP. */
FO_API int64_t fo_logp_workspace(int64_t rows, int32_t vocab);
FO_API fo_status fo_logp_fwd(int32_t dtype, int64_t rows, int32_t vocab, const void* logits, int64_t ld,
                             const int32_t* targets, float scale, float* logp, float* lse, void* workspace,
                             int64_t workspace_bytes, void* hip_stream);

/* dlogits_v = scale dlogp[r] (1{v = t} - exp(z_v - lse)), logp and lse as the
 * forward call left them.  Every row is written (zeros where it is ignored; its
 * dlogp is not read).  dlogits may be logits, with its row stride. */
FO_API fo_status fo_logp_bwd(int32_t dtype, int64_t rows, int32_t vocab, const void* logits, int64_t ld,
                             const int32_t* targets, float scale, const float* logp, const float* lse,
                             const float* dlogp, void* dlogits, int64_t dlogits_ld, void* hip_stream);

/* Cross-entropy with its gradient, in one pass over the logits where a row fits
 * the registers: loss[r] = -logp[r], and dlogits the gradient of sum_r weight[r]
 * loss[r] (weight: device fp32[rows], not read for ignored rows).  dlogits may be
 * logits, with its row stride. */
FO_API fo_status fo_xent(int32_t dtype, int64_t rows, int32_t vocab, const void* logits, int64_t ld,
                         const int32_t* targets, float scale, const float* weight, float* loss, void* dlogits,
                         int64_t dlogits_ld, void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ preference loss
 * Pairs of answers whose tokens' log probabilities lie in rows: answer 2 i, the
 * chosen one of pair i, rows [begin[2 i], end[2 i]); answer 2 i + 1 the rejected
 * one.
 *
 *   reward_q = beta sum over its rows of (logp - ref)      (mean != 0: beta mean)
 *   d = reward_{2i} - reward_{2i+1}
 *   loss_i = (1 - smooth) log(1 + exp(-d)) + smooth log(1 + exp(d))
 *   dlogp = the gradient of dloss sum_i loss_i
 *
 * ref (the frozen model's log probabilities) may be NULL: zeros.  An answer without
 * rows has reward 0.  logp, ref, dlogp: device fp32[rows]; begin, end: device
 * int32[2 pairs], clamped to the rows; loss fp32[pairs], reward fp32[2 pairs].  No
 * two answers share rows.  Rows of no answer are neither read nor written.  dlogp
 * (may be NULL) may be logp.  Computed in fp64 and rounded once.  beta finite,
 * smooth in [0, 1].  An infinite reward (a token of probability 0) gives the loss's
 * limit, infinity or, where the growing term has no weight, 0, and a finite
 * gradient; two of the same infinity, and an infinity times beta = 0, give NaN in
 * their pair.
 * Errors: FO_EINVAL, FO_EHIP. */
FO_API fo_status fo_pref_loss(int32_t pairs, int64_t rows, const int32_t* begin, const int32_t* end, const float* logp,
                              const float* ref, float beta, float smooth, int32_t mean, float dloss, float* loss,
                              float* reward, float* dlogp, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FEDOPTIMA_OPS_H */
