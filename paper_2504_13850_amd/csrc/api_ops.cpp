// C entry points of the transformer operators (fedoptima_ops.h): argument
// checks, then the launchers.
#include <cmath>

#include "ops.h"

using namespace fo;

namespace {

int64_t elem_size(int32_t dtype) { return dtype == FO_DT_BF16 ? 2 : 4; }
bool aligned(const void* p, int64_t n) { return ((uintptr_t)p & (uintptr_t)(n - 1)) == 0; }

// A [rows][heads][dim] operand of elements of `size` bytes: distinct elements have distinct addresses, and the last
// one's offset in bytes fits int64.
fo_status check_strides(const char* what, int64_t rows, int32_t heads, int32_t dim, int64_t ld, int64_t hs,
                        int64_t size) {
    constexpr int64_t kMaxStride = int64_t(1) << 40;
    FO_CHECK(ld >= 0 && hs >= 0 && ld <= kMaxStride && hs <= kMaxStride, "fo_attn: %s strides %lld, %lld", what,
             (long long)ld, (long long)hs);
    const bool rows_outer = (heads == 1 || hs >= dim) && (rows <= 1 || ld >= (heads - 1) * hs + dim);
    const bool heads_outer = (rows <= 1 || ld >= dim) &&
                             (heads == 1 || (__int128)hs >= (__int128)(rows > 0 ? rows - 1 : 0) * ld + dim);
    FO_CHECK(rows_outer || heads_outer, "fo_attn: %s strides %lld, %lld overlap (%lld rows, %d heads of %d)", what,
             (long long)ld, (long long)hs, (long long)rows, heads, dim);
    const __int128 last = (__int128)(rows > 0 ? rows - 1 : 0) * ld + (__int128)(heads - 1) * hs + dim;
    FO_CHECK(last * size <= INT64_MAX, "fo_attn: %s strides %lld, %lld pass 2^63 bytes (%lld rows, %d heads)", what,
             (long long)ld, (long long)hs, (long long)rows, heads);
    return FO_OK;
}

fo_status check_attn(const fo_attn* a) {
    FO_CHECK(a, "fo_attn: NULL record");
    FO_CHECK(a->dtype == FO_DT_BF16 || a->dtype == FO_DT_F32, "fo_attn: dtype=%d", a->dtype);
    FO_CHECK(a->batch >= 1 && a->heads >= 1 && a->kv_heads >= 1 && a->heads % a->kv_heads == 0,
             "fo_attn: batch=%d heads=%d kv_heads=%d", a->batch, a->heads, a->kv_heads);
    FO_CHECK(a->batch <= 65535 && a->heads <= 65535, "fo_attn: batch=%d heads=%d beyond 65535", a->batch, a->heads);
    FO_CHECK(a->head_dim >= 1 && a->head_dim <= 128, "fo_attn: head_dim=%d outside [1, 128]", a->head_dim);
    constexpr int32_t kMaxQ = 1 << 20, kMaxK = 1 << 30;  // 32-row tiles in a launch's third dimension
    FO_CHECK(a->max_q >= 0 && a->max_k >= 0 && a->max_q <= kMaxQ && a->max_k <= kMaxK,
             "fo_attn: max_q=%d max_k=%d", a->max_q, a->max_k);
    FO_CHECK(a->q_rows >= 0 && a->k_rows >= 0 && a->q_rows <= INT32_MAX && a->k_rows <= INT32_MAX,
             "fo_attn: q_rows=%lld k_rows=%lld", (long long)a->q_rows, (long long)a->k_rows);
    FO_CHECK((int64_t)a->batch * a->heads * ((a->max_q > a->max_k ? a->max_q : a->max_k) / 32 + 1) < INT32_MAX,
             "fo_attn: more workgroups than a launch holds");
    FO_CHECK(a->q_begin && a->q_end && a->k_begin && a->k_end, "fo_attn: NULL sequence bounds");
    fo_status st;
    const int64_t e = elem_size(a->dtype);
    if ((st = check_strides("q", a->q_rows, a->heads, a->head_dim, a->q_ld, a->q_hs, e)) != FO_OK) return st;
    if ((st = check_strides("k", a->k_rows, a->kv_heads, a->head_dim, a->k_ld, a->k_hs, e)) != FO_OK) return st;
    if ((st = check_strides("v", a->k_rows, a->kv_heads, a->head_dim, a->v_ld, a->v_hs, e)) != FO_OK) return st;
    if ((st = check_strides("out", a->q_rows, a->heads, a->head_dim, a->out_ld, a->out_hs, e)) != FO_OK) return st;
    // the kernels multiply by scale log2(e), or by scale / cap and cap log2(e), rounded to fp32
    constexpr float kLog2e = 1.4426950408889634f;
    FO_CHECK(std::isfinite(a->scale * kLog2e), "fo_attn: scale=%g", a->scale);
    FO_CHECK(a->cap >= 0.f && std::isfinite(a->cap * kLog2e) && (a->cap == 0.f || std::isfinite(a->scale / a->cap)),
             "fo_attn: cap=%g, scale=%g", a->cap, a->scale);
    FO_CHECK(a->mask == FO_ATTN_FULL || a->mask == FO_ATTN_CAUSAL || a->mask == FO_ATTN_PREFIX, "fo_attn: mask=%d",
             a->mask);
    FO_CHECK((a->mask == FO_ATTN_PREFIX) == (a->prefix != nullptr), "fo_attn: prefix lengths go with FO_ATTN_PREFIX");
    FO_CHECK((a->table != nullptr) == (a->bucket != nullptr), "fo_attn: a bias needs both table and bucket");
    if (a->table) {
        FO_CHECK(a->n_buckets >= 1 && a->n_buckets <= 1024 && a->radius >= 0 && a->radius <= 1024,
                 "fo_attn: n_buckets=%d radius=%d outside [1, 1024] and [0, 1024]", a->n_buckets, a->radius);
        FO_CHECK(aligned(a->table, elem_size(a->dtype)), "fo_attn: unaligned table");
    }
    FO_CHECK(a->p >= 0.f && a->p < 1.f, "fo_attn: p=%g outside [0, 1)", a->p);
    return FO_OK;
}

fo_status check_operands(const fo_attn* a, const void* q, const void* k, const void* v, const void* out,
                         const void* ws, int64_t ws_bytes, bool backward) {
    const int64_t e = elem_size(a->dtype);
    FO_CHECK((a->q_rows == 0 || (q && out)) && (a->k_rows == 0 || (k && v)), "fo_attn: NULL operand");
    FO_CHECK(aligned(q, e) && aligned(k, e) && aligned(v, e) && aligned(out, e), "fo_attn: unaligned operand");
    const int64_t need = attn_workspace(*a, backward);
    FO_CHECK(ws_bytes >= need && (need == 0 || ws), "fo_attn: workspace of %lld bytes, %lld are needed",
             (long long)ws_bytes, (long long)need);
    FO_CHECK(aligned(ws, 16), "fo_attn: the workspace is not 16-byte aligned");
    return FO_OK;
}

AttnArgs make_args(const fo_attn* a, const void* q, const void* k, const void* v, const void* out, const float* lse) {
    AttnArgs x{};
    x.a = *a;
    x.q = q; x.k = k; x.v = v;
    x.out = const_cast<void*>(out);
    x.lse = const_cast<float*>(lse);
    x.thr = drop_threshold(a->p);
    x.keep_scale = 65536.f / (float)(65536u - x.thr);
    return x;
}

}  // namespace

extern "C" int64_t fo_attn_workspace(const fo_attn* a, int32_t backward) {
    if (check_attn(a) != FO_OK) return -1;
    const int64_t f = attn_workspace(*a, false);
    if (!backward) return f;
    const int64_t b = attn_workspace(*a, true);
    return f > b ? f : b;
}

extern "C" fo_status fo_attn_fwd(const fo_attn* a, const void* q, const void* k, const void* v, void* out, float* lse,
                                 void* workspace, int64_t workspace_bytes, void* hip_stream) {
    fo_status st = check_attn(a);
    if (st != FO_OK) return st;
    if ((st = check_operands(a, q, k, v, out, workspace, workspace_bytes, false)) != FO_OK) return st;
    FO_CHECK(aligned(lse, 4), "fo_attn_fwd: unaligned lse");
    if (a->max_q == 0 || a->q_rows == 0) return FO_OK;  // no query row to write
    return launch_attn_op_fwd(make_args(a, q, k, v, out, lse), workspace, (hipStream_t)hip_stream);
}

extern "C" fo_status fo_attn_bwd(const fo_attn* a, const void* q, const void* k, const void* v, const void* out,
                                 const float* lse, const void* dout, void* dq, void* dk, void* dv, void* dtable,
                                 void* workspace, int64_t workspace_bytes, void* hip_stream) {
    fo_status st = check_attn(a);
    if (st != FO_OK) return st;
    if ((st = check_operands(a, q, k, v, out, workspace, workspace_bytes, true)) != FO_OK) return st;
    const int64_t e = elem_size(a->dtype);
    FO_CHECK((a->q_rows == 0 || (lse && dout && dq)) && (a->k_rows == 0 || (dk && dv)), "fo_attn_bwd: NULL operand");
    FO_CHECK(a->max_k <= 1 << 20, "fo_attn_bwd: max_k=%d", a->max_k);
    FO_CHECK(!a->table == !dtable, "fo_attn_bwd: dtable goes with the table");
    FO_CHECK(aligned(lse, 4) && aligned(dout, e) && aligned(dq, e) && aligned(dk, e) && aligned(dv, e) &&
             aligned(dtable, e), "fo_attn_bwd: unaligned operand");
    AttnArgs x = make_args(a, q, k, v, out, lse);
    x.dout = dout;
    x.dq = dq; x.dk = dk; x.dv = dv; x.dtable = dtable;
    return launch_attn_op_bwd(x, workspace, (hipStream_t)hip_stream);
}

extern "C" fo_status fo_relpos_buckets(int32_t n_buckets, int32_t radius, int32_t causal, int32_t* out) {
    FO_CHECK(out, "fo_relpos_buckets: NULL output");
    FO_CHECK(n_buckets >= 2 && n_buckets <= 1024 && (causal || (n_buckets % 2 == 0 && n_buckets >= 4)),
             "fo_relpos_buckets: n_buckets=%d", n_buckets);
    const int32_t half = causal ? n_buckets : n_buckets / 2, near = half / 2;
    FO_CHECK(radius > near && radius <= 1024, "fo_relpos_buckets: radius=%d outside [%d, 1024]", radius, near + 1);
    for (int32_t n = -radius; n <= radius; ++n) {
        const int32_t dist = causal ? (n < 0 ? -n : 0) : (n < 0 ? -n : n);
        int32_t b = dist;
        if (dist >= near) {
            // 1e-9 above the rounding of the logarithms: a boundary that is a whole number counts as reached
            const double x = std::log((double)dist / near) / std::log((double)radius / near) * (half - near);
            b = near + (int32_t)(x + 1e-9);
            if (b > half - 1) b = half - 1;
        }
        out[n + radius] = b + (n > 0 && !causal ? half : 0);
    }
    return FO_OK;
}

// Rows written over rows that are read: element over element, or a thread's rows would be another's.
static bool in_place(const void* x, int64_t x_ld, const void* y, int64_t y_ld, int64_t rows) {
    return x != y || rows <= 1 || x_ld == y_ld;
}

static fo_status check_drop(const char* what, int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld,
                            const void* y, int64_t y_ld, float p) {
    FO_CHECK(dtype == FO_DT_BF16 || dtype == FO_DT_F32, "%s: dtype=%d", what, dtype);
    FO_CHECK(rows >= 0 && rows <= INT32_MAX && cols >= 1 && cols <= (1 << 30), "%s: %lld rows of %d", what,
             (long long)rows, cols);
    FO_CHECK(rows == 0 || (x && y), "%s: NULL operand", what);
    constexpr int64_t kMaxStride = int64_t(1) << 31;
    FO_CHECK(x_ld >= cols && y_ld >= cols && x_ld <= kMaxStride && y_ld <= kMaxStride,
             "%s: row strides %lld, %lld for %d columns", what, (long long)x_ld, (long long)y_ld, cols);
    const int64_t e = elem_size(dtype);
    FO_CHECK(in_place(x, x_ld, y, y_ld, rows), "%s: in place with row strides %lld and %lld", what, (long long)x_ld,
             (long long)y_ld);
    FO_CHECK((__int128)rows * x_ld * e <= INT64_MAX && (__int128)rows * y_ld * e <= INT64_MAX,
             "%s: %lld rows of strides %lld, %lld pass 2^63 bytes", what, (long long)rows, (long long)x_ld, (long long)y_ld);
    FO_CHECK(p >= 0.f && p < 1.f, "%s: p=%g outside [0, 1)", what, p);
    FO_CHECK(aligned(x, e) && aligned(y, e), "%s: unaligned operand", what);
    return FO_OK;
}

extern "C" fo_status fo_dropout_fwd(int32_t dtype, int64_t rows, int32_t cols, const void* x, int64_t x_ld,
                                    const void* bias, const void* residual, int64_t res_ld, float p, uint64_t seed,
                                    uint32_t offset, void* y, int64_t y_ld, void* hip_stream) {
    const fo_status st = check_drop("fo_dropout_fwd", dtype, rows, cols, x, x_ld, y, y_ld, p);
    if (st != FO_OK) return st;
    const int64_t e = elem_size(dtype);
    FO_CHECK(!residual || (res_ld >= cols && res_ld <= (int64_t(1) << 31) && (__int128)rows * res_ld * e <= INT64_MAX),
             "fo_dropout_fwd: residual row stride %lld", (long long)res_ld);
    FO_CHECK(!residual || in_place(residual, res_ld, y, y_ld, rows),
             "fo_dropout_fwd: in place with row strides %lld and %lld", (long long)res_ld, (long long)y_ld);
    FO_CHECK(aligned(bias, e) && aligned(residual, e), "fo_dropout_fwd: unaligned operand");
    if (rows == 0) return FO_OK;
    DropArgs d{};
    d.rows = rows; d.cols = cols;
    d.x = x; d.bias = bias; d.res = residual; d.y = y;
    d.x_ld = x_ld; d.res_ld = res_ld; d.y_ld = y_ld;
    d.thr = drop_threshold(p);
    d.keep_scale = 65536.f / (float)(65536u - d.thr);
    d.k0 = (uint32_t)seed; d.k1 = (uint32_t)(seed >> 32); d.offset = offset;
    return launch_dropout_fwd(dtype, d, (hipStream_t)hip_stream);
}

extern "C" int64_t fo_dropout_workspace(int64_t rows, int32_t cols) {
    if (rows < 0 || cols < 1) {
        set_error("fo_dropout_workspace: %lld rows of %d", (long long)rows, cols);
        return -1;
    }
    return dropout_workspace(rows, cols);
}

extern "C" fo_status fo_dropout_bwd(int32_t dtype, int64_t rows, int32_t cols, const void* dy, int64_t dy_ld, float p,
                                    uint64_t seed, uint32_t offset, void* dx, int64_t dx_ld, void* dbias,
                                    void* workspace, int64_t workspace_bytes, void* hip_stream) {
    const fo_status st = check_drop("fo_dropout_bwd", dtype, rows, cols, dy, dy_ld, dx, dx_ld, p);
    if (st != FO_OK) return st;
    if (dbias) {
        const int64_t need = dropout_workspace(rows, cols);
        FO_CHECK(workspace_bytes >= need && (need == 0 || workspace),
                 "fo_dropout_bwd: workspace of %lld bytes, %lld are needed", (long long)workspace_bytes,
                 (long long)need);
        FO_CHECK(aligned(workspace, 16) && aligned(dbias, elem_size(dtype)), "fo_dropout_bwd: unaligned operand");
    }
    if (rows == 0 && !dbias) return FO_OK;
    DropArgs d{};
    d.rows = rows; d.cols = cols;
    d.x = dy; d.y = dx;
    d.x_ld = dy_ld; d.y_ld = dx_ld;
    d.thr = drop_threshold(p);
    d.keep_scale = 65536.f / (float)(65536u - d.thr);
    d.k0 = (uint32_t)seed; d.k1 = (uint32_t)(seed >> 32); d.offset = offset;
    return launch_dropout_bwd(dtype, d, dbias, (float*)workspace, (hipStream_t)hip_stream);
}
