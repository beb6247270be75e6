// Operators of a language model around its attention (fedoptima_ops.h): argument
// records and launchers.
#pragma once

#include "ops.h"

namespace fo {

// ------------------------------------------------------------------ embedding
struct EmbedArgs {
    int64_t rows;
    int32_t cols, vocab;
    const int32_t* tokens;
    const void* table;  // forward
    int64_t table_ld;
    void* out;
    int64_t out_ld;
    const void* dout;   // backward
    int64_t dout_ld;
    void* dtable;
    int64_t dtable_ld;
    float scale;
    bool accumulate;
};
fo_status launch_embed_fwd(int32_t dtype, const EmbedArgs& a, hipStream_t s);
int64_t embed_workspace(int64_t rows, int32_t cols, int32_t vocab);
fo_status launch_embed_bwd(int32_t dtype, const EmbedArgs& a, void* ws, hipStream_t s);

// ------------------------------------------------------------------ RMS norm, 8-bit rows
enum NormOut { kNorm, kNormF8, kQuantF8 };
struct NormArgs {
    int64_t rows;
    int32_t cols;
    const void *x, *res, *w;
    int64_t x_ld, res_ld;
    float eps;
    void* h;
    int64_t h_ld;
    void* y;  // T, or e4m3
    int64_t y_ld;
    float* rstd;     // kNorm
    float* y_scale;  // the 8-bit forms
};
fo_status launch_norm_fwd(int32_t dtype, NormOut out, const NormArgs& a, hipStream_t s);

struct NormBwdArgs {
    int64_t rows;
    int32_t cols;
    const void *dy, *h, *w, *dres;
    int64_t dy_ld, h_ld, dres_ld;
    const float* rstd;
    void* dx;
    int64_t dx_ld;
    float* part;  // [parts][cols] sums of dw, or NULL
    void* dw;     // where the rows are few: see norm_bwd_kernel
};
int64_t norm_workspace(int64_t rows, int32_t cols);
fo_status launch_norm_bwd(int32_t dtype, const NormBwdArgs& a, void* dw, hipStream_t s);

// ------------------------------------------------------------------ 8-bit product
struct GemmF8Args {
    int64_t M;
    int32_t N, K;
    const uint8_t *a, *b;
    int64_t lda, ldb, ldc;
    const float *a_scale, *b_scale;
    void* c;
};
int64_t gemm_f8_workspace(int64_t M, int32_t N, int32_t K);
fo_status launch_gemm_f8(int32_t dtype, const GemmF8Args& g, void* ws, hipStream_t s);

// ------------------------------------------------------------------ log probabilities
struct LogpArgs {
    int64_t rows;
    int32_t vocab;
    const void* logits;
    int64_t ld;
    const int32_t* targets;
    float scale;
    float *logp, *lse;   // forward: results; backward: operands (lse may be NULL in the forward pass)
    const float* weight; // the gradient by logp (backward), minus that (cross-entropy)
    void* dlogits;
    int64_t dlogits_ld;
};
int64_t logp_workspace(int64_t rows, int32_t vocab);
fo_status launch_logp_fwd(int32_t dtype, const LogpArgs& a, void* ws, hipStream_t s);
fo_status launch_logp_bwd(int32_t dtype, const LogpArgs& a, hipStream_t s);
fo_status launch_xent(int32_t dtype, const LogpArgs& a, void* ws, hipStream_t s);

// ------------------------------------------------------------------ preference loss
struct PrefArgs {
    int32_t pairs;
    int64_t rows;
    const int32_t *begin, *end;
    const float *logp, *ref;
    float beta, smooth, dloss;
    bool mean;
    float *loss, *reward, *dlogp;
};
fo_status launch_pref_loss(const PrefArgs& p, hipStream_t s);

}  // namespace fo
