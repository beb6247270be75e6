// C entry points of the language model's operators around its attention
// (fedoptima_ops.h): argument checks, then the launchers.
#include <cmath>

#include "lm.h"

using namespace fo;

namespace {

int64_t elem_size(int32_t dtype) { return dtype == FO_DT_BF16 ? 2 : 4; }
bool aligned(const void* p, int64_t n) { return ((uintptr_t)p & (uintptr_t)(n - 1)) == 0; }

fo_status check_sizes(const char* what, int32_t dtype, int64_t rows, int32_t cols) {
    FO_CHECK(dtype == FO_DT_BF16 || dtype == FO_DT_F32, "%s: dtype=%d", what, dtype);
    FO_CHECK(rows >= 0 && rows <= INT32_MAX && cols >= 1 && cols <= (1 << 30), "%s: %lld rows of %d", what,
             (long long)rows, cols);
    return FO_OK;
}

// A [rows][cols] matrix of elements of e bytes; NULL where `optional`, or where it has no rows.
fo_status check_rows(const char* what, const char* name, const void* p, int64_t ld, int64_t rows, int32_t cols,
                     int64_t e, bool optional) {
    FO_CHECK(p || optional || rows == 0, "%s: NULL %s", what, name);
    if (!p) return FO_OK;
    constexpr int64_t kMaxStride = int64_t(1) << 31;
    FO_CHECK(ld >= cols && ld <= kMaxStride, "%s: %s with row stride %lld for %d columns", what, name, (long long)ld,
             cols);
    FO_CHECK((__int128)rows * ld * e <= INT64_MAX, "%s: %s with %lld rows of stride %lld passes 2^63 bytes", what,
             name, (long long)rows, (long long)ld);
    FO_CHECK(aligned(p, e), "%s: unaligned %s", what, name);
    return FO_OK;
}

fo_status check_vector(const char* what, const char* name, const void* p, int64_t n, int64_t e, bool optional) {
    FO_CHECK(p || optional || n == 0, "%s: NULL %s", what, name);
    FO_CHECK(aligned(p, e), "%s: unaligned %s", what, name);
    return FO_OK;
}

// Rows written over rows that are read: element over element, or a row's end would be another's.
fo_status check_in_place(const char* what, const void* x, int64_t x_ld, const void* y, int64_t y_ld, int64_t rows) {
    FO_CHECK(!x || x != y || rows <= 1 || x_ld == y_ld, "%s: in place with row strides %lld and %lld", what,
             (long long)x_ld, (long long)y_ld);
    return FO_OK;
}

fo_status check_workspace(const char* what, const void* ws, int64_t bytes, int64_t need) {
    FO_CHECK(bytes >= need && (need == 0 || ws), "%s: workspace of %lld bytes, %lld are needed", what,
             (long long)bytes, (long long)need);
    FO_CHECK(aligned(ws, 16), "%s: the workspace is not 16-byte aligned", what);
    return FO_OK;
}

}  // namespace

#define FO_TRY(call)                          \
    do {                                      \
        const fo_status st_ = (call);         \
        if (st_ != FO_OK) return st_;         \
    } while (0)

// ------------------------------------------------------------------ embedding
// 128 columns a workgroup in a launch's third dimension; tiles of the sort of 1024 rows, of 4096 above 2^20 rows.
constexpr int32_t kMaxEmbedCols = 1 << 22;
constexpr int64_t kMaxEmbedRows = int64_t(1) << 28;

static fo_status check_embed(const char* what, int32_t dtype, int64_t rows, int32_t cols, int32_t vocab,
                             const int32_t* tokens, float scale) {
    FO_TRY(check_sizes(what, dtype, rows, cols));
    FO_CHECK(cols <= kMaxEmbedCols, "%s: %d columns", what, cols);
    FO_CHECK(vocab >= 1 && vocab <= (1 << 30), "%s: vocab=%d", what, vocab);
    FO_CHECK(std::isfinite(scale), "%s: scale=%g", what, scale);
    return check_vector(what, "tokens", tokens, rows, 4, false);
}

extern "C" fo_status fo_embed_fwd(int32_t dtype, int64_t rows, int32_t cols, int32_t vocab, const int32_t* tokens,
                                  const void* table, int64_t table_ld, float scale, void* out, int64_t out_ld,
                                  void* hip_stream) {
    const char* what = "fo_embed_fwd";
    FO_TRY(check_embed(what, dtype, rows, cols, vocab, tokens, scale));
    const int64_t e = elem_size(dtype);
    FO_TRY(check_rows(what, "table", table, table_ld, vocab, cols, e, rows == 0));
    FO_TRY(check_rows(what, "out", out, out_ld, rows, cols, e, false));
    FO_CHECK(!out || out != table, "%s: out is the table", what);
    if (rows == 0) return FO_OK;
    EmbedArgs a{};
    a.rows = rows; a.cols = cols; a.vocab = vocab;
    a.tokens = tokens; a.scale = scale;
    a.table = table; a.table_ld = table_ld;
    a.out = out; a.out_ld = out_ld;
    return launch_embed_fwd(dtype, a, (hipStream_t)hip_stream);
}

extern "C" int64_t fo_embed_workspace(int64_t rows, int32_t cols, int32_t vocab) {
    if (rows < 0 || rows > kMaxEmbedRows || cols < 1 || cols > kMaxEmbedCols || vocab < 1 || vocab > (1 << 30)) {
        set_error("fo_embed_workspace: %lld rows of %d, vocab=%d", (long long)rows, cols, vocab);
        return -1;
    }
    return embed_workspace(rows, cols, vocab);
}

extern "C" fo_status fo_embed_bwd(int32_t dtype, int64_t rows, int32_t cols, int32_t vocab, const int32_t* tokens,
                                  const void* dout, int64_t dout_ld, float scale, int32_t accumulate, void* dtable,
                                  int64_t dtable_ld, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    const char* what = "fo_embed_bwd";
    FO_TRY(check_embed(what, dtype, rows, cols, vocab, tokens, scale));
    FO_CHECK(rows <= kMaxEmbedRows, "%s: %lld rows", what, (long long)rows);
    const int64_t e = elem_size(dtype);
    FO_TRY(check_rows(what, "dout", dout, dout_ld, rows, cols, e, false));
    FO_TRY(check_rows(what, "dtable", dtable, dtable_ld, vocab, cols, e, false));
    FO_CHECK(!dout || dout != dtable, "%s: dout is dtable", what);
    FO_TRY(check_workspace(what, workspace, workspace_bytes, embed_workspace(rows, cols, vocab)));
    if (rows == 0 && accumulate) return FO_OK;
    EmbedArgs a{};
    a.rows = rows; a.cols = cols; a.vocab = vocab;
    a.tokens = tokens; a.scale = scale; a.accumulate = accumulate != 0;
    a.dout = dout; a.dout_ld = dout_ld;
    a.dtable = dtable; a.dtable_ld = dtable_ld;
    return launch_embed_bwd(dtype, a, workspace, (hipStream_t)hip_stream);
}

// ------------------------------------------------------------------ RMS norm, 8-bit rows
static fo_status norm_fwd(const char* what, NormOut out, int32_t dtype, int64_t rows, int32_t cols, const void* x,
                          int64_t x_ld, const void* residual, int64_t res_ld, const void* w, float eps, void* h,
                          int64_t h_ld, void* y, int64_t y_ld, float* rstd, float* y_scale, void* hip_stream) {
    FO_TRY(check_sizes(what, dtype, rows, cols));
    const int64_t e = elem_size(dtype);
    FO_TRY(check_rows(what, "x", x, x_ld, rows, cols, e, false));
    FO_TRY(check_rows(what, "residual", residual, res_ld, rows, cols, e, true));
    FO_TRY(check_rows(what, "h", h, h_ld, rows, cols, e, true));
    FO_TRY(check_rows(what, "y", y, y_ld, rows, cols, out == kNorm ? e : 1, false));
    FO_TRY(check_vector(what, "w", w, cols, e, true));
    FO_TRY(check_vector(what, "rstd", rstd, rows, 4, true));
    FO_TRY(check_vector(what, "y_scale", y_scale, rows, 4, out == kNorm));
    FO_CHECK(eps >= 0.f && std::isfinite(eps), "%s: eps=%g", what, eps);
    FO_CHECK(!y || y != h, "%s: y is h", what);
    FO_CHECK(out == kNorm || !y || (y != x && y != residual), "%s: 8-bit rows in place", what);
    FO_TRY(check_in_place(what, x, x_ld, h, h_ld, rows));
    FO_TRY(check_in_place(what, residual, res_ld, h, h_ld, rows));
    FO_TRY(check_in_place(what, x, x_ld, y, y_ld, rows));
    FO_TRY(check_in_place(what, residual, res_ld, y, y_ld, rows));
    if (rows == 0) return FO_OK;
    NormArgs a{};
    a.rows = rows; a.cols = cols;
    a.x = x; a.res = residual; a.w = w; a.h = h; a.y = y;
    a.x_ld = x_ld; a.res_ld = res_ld; a.h_ld = h_ld; a.y_ld = y_ld;
    a.eps = eps; a.rstd = rstd; a.y_scale = y_scale;
    return launch_norm_fwd(dtype, out, a, (hipStream_t)hip_stream);
}

extern "C" fo_status fo_rmsnorm_fwd(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld,
                                    const void* residual, int64_t res_ld, const void* w, float eps, void* h,
                                    int64_t h_ld, void* y, int64_t y_ld, float* rstd, void* hip_stream) {
    return norm_fwd("fo_rmsnorm_fwd", kNorm, dtype, rows, cols, x, x_ld, residual, res_ld, w, eps, h, h_ld, y, y_ld,
                    rstd, nullptr, hip_stream);
}

extern "C" fo_status fo_rmsnorm_f8(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld,
                                   const void* residual, int64_t res_ld, const void* w, float eps, void* h,
                                   int64_t h_ld, uint8_t* y8, int64_t y8_ld, float* y_scale, void* hip_stream) {
    return norm_fwd("fo_rmsnorm_f8", kNormF8, dtype, rows, cols, x, x_ld, residual, res_ld, w, eps, h, h_ld, y8, y8_ld,
                    nullptr, y_scale, hip_stream);
}

extern "C" fo_status fo_quant_f8(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld, uint8_t* y8,
                                 int64_t y8_ld, float* y_scale, void* hip_stream) {
    return norm_fwd("fo_quant_f8", kQuantF8, dtype, rows, cols, x, x_ld, nullptr, 0, nullptr, 0.f, nullptr, 0, y8,
                    y8_ld, nullptr, y_scale, hip_stream);
}

extern "C" int64_t fo_rmsnorm_workspace(int64_t rows, int32_t cols) {
    if (rows < 0 || rows > INT32_MAX || cols < 1 || cols > (1 << 30)) {
        set_error("fo_rmsnorm_workspace: %lld rows of %d", (long long)rows, cols);
        return -1;
    }
    return norm_workspace(rows, cols);
}

extern "C" fo_status fo_rmsnorm_bwd(int32_t dtype, int64_t rows, int32_t cols, const void* dy, int64_t dy_ld,
                                    const void* h, int64_t h_ld, const void* w, const float* rstd, const void* dres,
                                    int64_t dres_ld, void* dx, int64_t dx_ld, void* dw, void* workspace,
                                    int64_t workspace_bytes, void* hip_stream) {
    const char* what = "fo_rmsnorm_bwd";
    FO_TRY(check_sizes(what, dtype, rows, cols));
    const int64_t e = elem_size(dtype);
    FO_TRY(check_rows(what, "dy", dy, dy_ld, rows, cols, e, false));
    FO_TRY(check_rows(what, "h", h, h_ld, rows, cols, e, false));
    FO_TRY(check_rows(what, "dres", dres, dres_ld, rows, cols, e, true));
    FO_TRY(check_rows(what, "dx", dx, dx_ld, rows, cols, e, false));
    FO_TRY(check_vector(what, "w", w, cols, e, true));
    FO_TRY(check_vector(what, "rstd", rstd, rows, 4, false));
    FO_TRY(check_vector(what, "dw", dw, cols, e, true));
    FO_TRY(check_in_place(what, dy, dy_ld, dx, dx_ld, rows));
    FO_TRY(check_in_place(what, dres, dres_ld, dx, dx_ld, rows));
    FO_TRY(check_in_place(what, h, h_ld, dx, dx_ld, rows));
    if (dw) FO_TRY(check_workspace(what, workspace, workspace_bytes, norm_workspace(rows, cols)));
    if (rows == 0 && !dw) return FO_OK;
    NormBwdArgs a{};
    a.rows = rows; a.cols = cols;
    a.dy = dy; a.h = h; a.w = w; a.dres = dres; a.rstd = rstd; a.dx = dx;
    a.dy_ld = dy_ld; a.h_ld = h_ld; a.dres_ld = dres_ld; a.dx_ld = dx_ld;
    a.part = dw ? (float*)workspace : nullptr;
    return launch_norm_bwd(dtype, a, dw, (hipStream_t)hip_stream);
}

// ------------------------------------------------------------------ 8-bit product
extern "C" int64_t fo_gemm_f8_workspace(int64_t M, int32_t N, int32_t K) {
    if (M < 0 || M > INT32_MAX || N < 1 || N > (1 << 30) || K < 1 || K > (1 << 30)) {
        set_error("fo_gemm_f8_workspace: %lld x %d x %d", (long long)M, N, K);
        return -1;
    }
    return gemm_f8_workspace(M, N, K);
}

extern "C" fo_status fo_gemm_f8(int32_t dtype, int64_t M, int32_t N, int32_t K, const uint8_t* a, int64_t lda,
                                const float* a_scale, const uint8_t* b, int64_t ldb, const float* b_scale, void* c,
                                int64_t ldc, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    const char* what = "fo_gemm_f8";
    FO_TRY(check_sizes(what, dtype, M, N));
    FO_CHECK(K >= 1 && K <= (1 << 30), "%s: K=%d", what, K);
    FO_TRY(check_rows(what, "a", a, lda, M, K, 1, false));
    FO_TRY(check_rows(what, "b", b, ldb, N, K, 1, M == 0));
    FO_TRY(check_rows(what, "c", c, ldc, M, N, elem_size(dtype), false));
    FO_TRY(check_vector(what, "a_scale", a_scale, M, 4, true));
    FO_TRY(check_vector(what, "b_scale", b_scale, N, 4, true));
    FO_CHECK(cdiv(M, 256) * cdiv(N, 256) <= 1 << 22, "%s: more workgroups than a launch holds (%lld x %d)", what,
             (long long)M, N);
    FO_CHECK(!c || (c != (const void*)a && c != (const void*)b), "%s: c is an operand", what);
    FO_TRY(check_workspace(what, workspace, workspace_bytes, gemm_f8_workspace(M, N, K)));
    if (M == 0) return FO_OK;
    GemmF8Args g{};
    g.M = M; g.N = N; g.K = K;
    g.a = a; g.b = b; g.c = c;
    g.lda = lda; g.ldb = ldb; g.ldc = ldc;
    g.a_scale = a_scale; g.b_scale = b_scale;
    return launch_gemm_f8(dtype, g, workspace, (hipStream_t)hip_stream);
}

// ------------------------------------------------------------------ log probabilities
extern "C" int64_t fo_logp_workspace(int64_t rows, int32_t vocab) {
    if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > (1 << 30)) {
        set_error("fo_logp_workspace: %lld rows, vocab=%d", (long long)rows, vocab);
        return -1;
    }
    return logp_workspace(rows, vocab);
}

static fo_status check_logp(const char* what, int32_t dtype, int64_t rows, int32_t vocab, const void* logits,
                            int64_t ld, const int32_t* targets, float scale) {
    FO_TRY(check_sizes(what, dtype, rows, vocab));
    FO_TRY(check_rows(what, "logits", logits, ld, rows, vocab, elem_size(dtype), false));
    FO_TRY(check_vector(what, "targets", targets, rows, 4, false));
    FO_CHECK(scale > 0.f && std::isfinite(scale * 1.4426950408889634f), "%s: scale=%g", what, scale);
    return FO_OK;
}

static LogpArgs logp_args(int64_t rows, int32_t vocab, const void* logits, int64_t ld, const int32_t* targets,
                          float scale) {
    LogpArgs a{};
    a.rows = rows; a.vocab = vocab; a.logits = logits; a.ld = ld; a.targets = targets; a.scale = scale;
    return a;
}

extern "C" fo_status fo_logp_fwd(int32_t dtype, int64_t rows, int32_t vocab, const void* logits, int64_t ld,
                                 const int32_t* targets, float scale, float* logp, float* lse, void* workspace,
                                 int64_t workspace_bytes, void* hip_stream) {
    const char* what = "fo_logp_fwd";
    FO_TRY(check_logp(what, dtype, rows, vocab, logits, ld, targets, scale));
    FO_TRY(check_vector(what, "logp", logp, rows, 4, false));
    FO_TRY(check_vector(what, "lse", lse, rows, 4, true));
    FO_TRY(check_workspace(what, workspace, workspace_bytes, logp_workspace(rows, vocab)));
    if (rows == 0) return FO_OK;
    LogpArgs a = logp_args(rows, vocab, logits, ld, targets, scale);
    a.logp = logp; a.lse = lse;
    return launch_logp_fwd(dtype, a, workspace, (hipStream_t)hip_stream);
}

extern "C" fo_status fo_logp_bwd(int32_t dtype, int64_t rows, int32_t vocab, const void* logits, int64_t ld,
                                 const int32_t* targets, float scale, const float* logp, const float* lse,
                                 const float* dlogp, void* dlogits, int64_t dlogits_ld, void* hip_stream) {
    const char* what = "fo_logp_bwd";
    FO_TRY(check_logp(what, dtype, rows, vocab, logits, ld, targets, scale));
    FO_TRY(check_vector(what, "logp", logp, rows, 4, false));
    FO_TRY(check_vector(what, "lse", lse, rows, 4, false));
    FO_TRY(check_vector(what, "dlogp", dlogp, rows, 4, false));
    FO_TRY(check_rows(what, "dlogits", dlogits, dlogits_ld, rows, vocab, elem_size(dtype), false));
    FO_TRY(check_in_place(what, logits, ld, dlogits, dlogits_ld, rows));
    if (rows == 0) return FO_OK;
    LogpArgs a = logp_args(rows, vocab, logits, ld, targets, scale);
    a.logp = const_cast<float*>(logp); a.lse = const_cast<float*>(lse); a.weight = dlogp;
    a.dlogits = dlogits; a.dlogits_ld = dlogits_ld;
    return launch_logp_bwd(dtype, a, (hipStream_t)hip_stream);
}

extern "C" fo_status fo_xent(int32_t dtype, int64_t rows, int32_t vocab, const void* logits, int64_t ld,
                             const int32_t* targets, float scale, const float* weight, float* loss, void* dlogits,
                             int64_t dlogits_ld, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    const char* what = "fo_xent";
    FO_TRY(check_logp(what, dtype, rows, vocab, logits, ld, targets, scale));
    FO_TRY(check_vector(what, "weight", weight, rows, 4, false));
    FO_TRY(check_vector(what, "loss", loss, rows, 4, false));
    FO_TRY(check_rows(what, "dlogits", dlogits, dlogits_ld, rows, vocab, elem_size(dtype), false));
    FO_TRY(check_in_place(what, logits, ld, dlogits, dlogits_ld, rows));
    FO_TRY(check_workspace(what, workspace, workspace_bytes, logp_workspace(rows, vocab)));
    if (rows == 0) return FO_OK;
    LogpArgs a = logp_args(rows, vocab, logits, ld, targets, scale);
    a.logp = loss; a.weight = weight;
    a.dlogits = dlogits; a.dlogits_ld = dlogits_ld;
    return launch_xent(dtype, a, workspace, (hipStream_t)hip_stream);
}

// ------------------------------------------------------------------ preference loss
extern "C" fo_status fo_pref_loss(int32_t pairs, int64_t rows, const int32_t* begin, const int32_t* end,
                                  const float* logp, const float* ref, float beta, float smooth, int32_t mean,
                                  float dloss, float* loss, float* reward, float* dlogp, void* hip_stream) {
    const char* what = "fo_pref_loss";
    FO_CHECK(pairs >= 0 && pairs <= (1 << 29) && rows >= 0 && rows <= INT32_MAX, "%s: %d pairs, %lld rows", what,
             pairs, (long long)rows);
    FO_TRY(check_vector(what, "begin", begin, pairs, 4, false));
    FO_TRY(check_vector(what, "end", end, pairs, 4, false));
    FO_TRY(check_vector(what, "logp", logp, pairs ? rows : 0, 4, false));
    FO_TRY(check_vector(what, "ref", ref, rows, 4, true));
    FO_TRY(check_vector(what, "loss", loss, pairs, 4, false));
    FO_TRY(check_vector(what, "reward", reward, pairs, 4, false));
    FO_TRY(check_vector(what, "dlogp", dlogp, rows, 4, true));
    FO_CHECK(std::isfinite(beta) && std::isfinite(dloss), "%s: beta=%g dloss=%g", what, beta, dloss);
    FO_CHECK(smooth >= 0.f && smooth <= 1.f, "%s: smooth=%g outside [0, 1]", what, smooth);
    if (pairs == 0) return FO_OK;
    PrefArgs p{};
    p.pairs = pairs; p.rows = rows;
    p.begin = begin; p.end = end; p.logp = logp; p.ref = ref;
    p.beta = beta; p.smooth = smooth; p.dloss = dloss; p.mean = mean != 0;
    p.loss = loss; p.reward = reward; p.dlogp = dlogp;
    return launch_pref_loss(p, (hipStream_t)hip_stream);
}
