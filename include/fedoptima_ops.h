/*
 * fedoptima_ops.h -- transformer operators of libfedoptima for networks beyond
 * the built-in configurations: masked attention with its gradients, a learned
 * bias by distance, and dropout.
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

#ifdef __cplusplus
}
#endif
#endif /* FEDOPTIMA_OPS_H */
