// Masked attention with capped scores, a learned bias by distance and dropout
// (fedoptima_ops.h): launch shapes, the joining of key slices and of the bias
// gradient's sums.
#include <algorithm>

#include "attn_narrow.h"
#include "attn_small.h"

namespace fo {
#define FO_EXTERN(T, D)                                                                              \
    extern template fo_status attn_fwd_launch<T, D>(const AttnArgs&, const FwdShape&, hipStream_t);  \
    extern template fo_status attn_bwd_launch<T, D>(const AttnArgs&, const BwdShape&, hipStream_t)
FO_EXTERN(bf16_t, 32); FO_EXTERN(bf16_t, 64); FO_EXTERN(bf16_t, 128);
FO_EXTERN(float, 32); FO_EXTERN(float, 64); FO_EXTERN(float, 128);
#undef FO_EXTERN
#define FO_EXTERN(T, D)                                                                                \
    extern template fo_status narrow_fwd_launch<T, D>(const AttnArgs&, const FwdShape&, hipStream_t);  \
    extern template fo_status narrow_bwd_launch<T, D>(const AttnArgs&, const BwdShape&, hipStream_t)
FO_EXTERN(bf16_t, 2); FO_EXTERN(bf16_t, 4); FO_EXTERN(bf16_t, 8);
FO_EXTERN(float, 2); FO_EXTERN(float, 4); FO_EXTERN(float, 8);
#undef FO_EXTERN
#define FO_EXTERN(T, D) extern template fo_status small_bwd_launch<T, D>(const AttnArgs&, hipStream_t)
FO_EXTERN(bf16_t, 32); FO_EXTERN(bf16_t, 64); FO_EXTERN(bf16_t, 128); FO_EXTERN(float, 32); FO_EXTERN(float, 64);
#undef FO_EXTERN

namespace {

// The table's gradient from the key kernel's sums by distance: a workgroup per
// head, 256 distances at a time and four groups of threads on the tiles of all
// sequences, which meet in order; then 32 threads per bucket.  Latency: 4 us for 12 heads
// and 32 sequences.  It grows with the tiles that max_k allows each sequence, there or
// not: (2 radius + 1) floats each for a head, read by the head's one workgroup.
template <class T>
__global__ void __launch_bounds__(1024) bucket_sums(AttnArgs x, int parts) {
    const fo_attn& a = x.a;
    __shared__ float sum[4][2 * 1024 + 1];
    __shared__ int of[2 * 1024 + 1];
    const int h = blockIdx.x, W = 2 * a.radius + 1, tid = threadIdx.x, g4 = tid >> 8;
    const float* hist = x.hist + (int64_t)h * W;
    const int64_t step = (int64_t)a.heads * W;
    each(tid & 255, 256, W, [&](int n) {
        float s = 0.f;
#pragma unroll 8
        for (int p = g4; p < parts; p += 4) s += hist[p * step + n];
        sum[g4][n] = s;
        if (g4 == 0) of[n] = min(max(a.bucket[n], 0), a.n_buckets - 1);
    });
    __syncthreads();
    each(tid, 1024, W, [&](int n) { sum[0][n] = sum[0][n] + sum[1][n] + sum[2][n] + sum[3][n]; });
    __syncthreads();
    each(tid >> 5, 32, a.n_buckets, [&](int g) {
        float s = 0.f;
        each(tid & 31, 32, W, [&](int n) { s += of[n] == g ? sum[0][n] : 0.f; });
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor(s, o);
        if ((tid & 31) == 0) ((T*)x.dtable)[(int64_t)g * a.heads + h] = from_f<T>(s);
    });
}

// Joins the key slices of a row: one wave per row and head.  A lane holds a slice's
// maximum and sum (64 slices at most), then eight slices' sums fly at a time: bound by
// the latency of those rounds.  One token of 32 heads against 16k keys in 64 slices:
// the call takes 31 us, 83 when the slices were read one after the other.
constexpr int kMaxSplits = 64;
template <class T>
__global__ void __launch_bounds__(256) join_slices(AttnArgs x, FwdShape f) {
    const fo_attn& a = x.a;
    const int lane = threadIdx.x & 63, D = a.head_dim;
    int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int h = (int)(id % a.heads);
    id /= a.heads;
    const int i = (int)(id % a.max_q), b = (int)(id / a.max_q);
    if (b >= a.batch) return;
    const Span s = span_of(a, b);
    if (i >= s.nq) return;
    const int64_t row = (int64_t)h * a.q_rows + s.q0 + i, step = (int64_t)a.heads * a.q_rows;
    float mk = -INFINITY, lk = 0.f;
    if (lane < f.splits) {
        mk = f.ml[2 * (row + lane * step)];
        lk = f.ml[2 * (row + lane * step) + 1];
    }
    float m = mk;
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float g = __builtin_amdgcn_exp2f(mk - (m == -INFINITY ? 0.f : m));
    float l = lk * g, o[2] = {0.f, 0.f};
#pragma unroll
    for (int w = 32; w; w >>= 1) l += __shfl_xor(l, w);
    const uint64_t some = __ballot(lk > 0.f);  // the others, of no keys, wrote no sums
    const int c0 = min(lane, D - 1), c1 = min(lane + 64, D - 1);
    for (int k0 = 0; k0 < f.splits; k0 += 8) {
        float v0[8], v1[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float* at = f.part + (row + min(k0 + u, f.splits - 1) * step) * D;
            v0[u] = at[c0];
            v1[u] = at[c1];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int k = (k0 + u) & (kMaxSplits - 1);
            const float gk = __shfl(g, k);
            if ((some >> k) & 1) {
                o[0] = fmaf(v0[u], gk, o[0]);
                o[1] = fmaf(v1[u], gk, o[1]);
            }
        }
    }
    const float inv = l > 0.f ? x.keep_scale / l : l;  // 0 for a row that sees nothing, NaN stays NaN
    T* out = (T*)x.out + (int64_t)(s.q0 + i) * a.out_ld + h * a.out_hs;
    if (lane < D) out[lane] = from_f<T>(o[0] * inv);
    if (lane + 64 < D) out[lane + 64] = from_f<T>(o[1] * inv);
    if (x.lse && lane == 0) x.lse[row] = l > 0.f ? m + __builtin_amdgcn_logf(l) : -INFINITY;
}

// Adds the key kernel's cuts of a key row in order: one wave per row and key head.
// 11 us for 5000 rows of 4 heads of 64 in three cuts (31 MB).
template <class T>
__global__ void __launch_bounds__(256) join_keys(AttnArgs x, BwdShape f) {
    const fo_attn& a = x.a;
    const int lane = threadIdx.x & 63, D = a.head_dim, parts = f.h_parts * f.q_parts;
    int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int hk = (int)(id % a.kv_heads);
    id /= a.kv_heads;
    const int j = (int)(id % a.max_k), b = (int)(id / a.max_k);
    if (b >= a.batch) return;
    const Span s = span_of(a, b);
    if (j >= s.nk) return;
    const int64_t step = a.k_rows * a.kv_heads * D;
    const float* dk = f.part + ((int64_t)(s.k0 + j) * a.kv_heads + hk) * D;
    const float* dv = dk + parts * step;
    T* outk = (T*)x.dk + (int64_t)(s.k0 + j) * a.k_ld + hk * a.k_hs;
    T* outv = (T*)x.dv + (int64_t)(s.k0 + j) * a.v_ld + hk * a.v_hs;
    each(lane, 64, D, [&](int c) {
        float sk = 0.f, sv = 0.f;
#pragma unroll 4
        for (int p = 0; p < parts; ++p) {
            sk += dk[p * step + c];
            sv += dv[p * step + c];
        }
        outk[c] = from_f<T>(sk * a.scale);
        outv[c] = from_f<T>(sv * x.keep_scale);
    });
}

// 16-byte aligned rows of a [rows][heads][dim] operand, their stride below 2^24 bytes.
bool aligned_rows(const void* p, int64_t ld, int64_t hs, int64_t size) {
    return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0 && hs * size % 16 == 0 && ld * size < (1 << 24);
}
bool vec_fwd(const AttnArgs& x) {
    const fo_attn& a = x.a;
    const int64_t e = a.dtype == FO_DT_BF16 ? 2 : 4;
    return a.head_dim * e % 16 == 0 && aligned_rows(x.q, a.q_ld, a.q_hs, e) && aligned_rows(x.k, a.k_ld, a.k_hs, e) &&
           aligned_rows(x.v, a.v_ld, a.v_hs, e) && aligned_rows(x.out, a.out_ld, a.out_hs, e);
}

// Rows per workgroup by the longest query side; single tokens take the heads of
// a group as rows, so that a key head's cache is read once for all of them.
// Where the row tiles do not fill the chip's 256 compute units twice, the keys
// are cut into slices of at least 256 as well.
constexpr int kNarrowDim = 8;  // the widest head of attn_narrow.h

FwdShape fwd_shape(const fo_attn& a) {
    FwdShape f{};
    f.group = a.heads / a.kv_heads;
    f.pack = a.max_q == 1;
    f.narrow = a.head_dim <= kNarrowDim && a.max_q > 32;
    f.wq = f.pack || a.max_q <= 32 ? 1 : a.max_q <= 64 ? 2 : 4;
    const int64_t rows = f.pack ? a.heads / a.kv_heads : a.max_q;
    f.row_tiles = (int)cdiv(rows, f.narrow ? kNarrowRows : 32 * f.wq);
    const int64_t wgs = (int64_t)f.row_tiles * (f.pack ? a.kv_heads : a.heads) * a.batch / (f.narrow ? 4 : 1);
    int64_t sp = cdiv(512, std::max<int64_t>(1, wgs));
    sp = std::min<int64_t>(sp, std::max<int64_t>(1, a.max_k / 256));
    f.splits = (int)std::min<int64_t>(sp, kMaxSplits);
    return f;
}

BwdShape bwd_shape(const fo_attn& a) {
    BwdShape f{};
    f.group = a.heads / a.kv_heads;
    f.narrow = a.head_dim <= kNarrowDim && a.max_q > 32 && a.max_k > 32;
    if (f.narrow) f.wq = f.wk = kNarrowRows / 32;
    else f.wq = a.max_q <= 32 ? 1 : a.max_q <= 64 ? 2 : 4;
    f.q_tiles = a.q_rows ? (int)cdiv(a.max_q, 32 * f.wq) : 0;
    if (!f.narrow)
        f.wk = a.max_k > 64 ? 4 : a.max_k > 32 || (a.dtype == FO_DT_F32 && a.head_dim > 64) ? 2 : 1;  // see min_wk
    f.k_tiles = a.k_rows ? (int)cdiv(a.max_k, 32 * f.wk) : 0;
    // The key kernel's work is cut until about 512 workgroups share it, each with
    // 512 query rows of one head or more, so that the cuts' sums stay a small part.
    const int64_t wgs = std::max<int64_t>(1, (int64_t)f.k_tiles * a.kv_heads * a.batch / (f.narrow ? 4 : 1)), G = a.heads / a.kv_heads;
    const int64_t cuts = std::max<int64_t>(1, std::min<int64_t>({cdiv(512, wgs), G * a.max_q / 512, 64}));
    f.h_parts = f.q_parts = 1;
    if (!f.k_tiles) return f;  // no key rows: nothing to cut or to join
    f.h_parts = (int)std::min(G, cuts);
    while (G % f.h_parts) --f.h_parts;
    f.q_parts = (int)(cuts / f.h_parts);
    return f;
}
int64_t part_floats(const fo_attn& a, const BwdShape& f) {
    const int64_t parts = (int64_t)f.h_parts * f.q_parts;
    return parts > 1 ? (2 * parts * a.k_rows * a.kv_heads * a.head_dim + 3) & ~int64_t(3) : 0;
}
int64_t hist_floats(const fo_attn& a, const BwdShape& f) {
    return a.table ? (int64_t)f.q_parts * f.k_tiles * a.batch * a.heads * (2 * a.radius + 1) : 0;
}
// delta of every row and head, in whole 16-byte units
int64_t stat_floats(const fo_attn& a) { return (a.q_rows * a.heads + 3) & ~int64_t(3); }

}  // namespace

int64_t attn_workspace(const fo_attn& a, bool backward) {
    if (!backward) {
        const FwdShape f = fwd_shape(a);
        return f.splits > 1 ? (int64_t)f.splits * a.heads * a.q_rows * (a.head_dim + 2) * 4 : 0;
    }
    const BwdShape f = bwd_shape(a);
    return 4 * (stat_floats(a) + part_floats(a, f) + hist_floats(a, f));
}

template <class T>
static fo_status fwd_narrow(const AttnArgs& x, const FwdShape& f, hipStream_t s) {
    return x.a.head_dim <= 2   ? narrow_fwd_launch<T, 2>(x, f, s)
           : x.a.head_dim <= 4 ? narrow_fwd_launch<T, 4>(x, f, s)
                               : narrow_fwd_launch<T, 8>(x, f, s);
}
template <class T>
static fo_status bwd_narrow(const AttnArgs& x, const BwdShape& f, hipStream_t s) {
    return x.a.head_dim <= 2   ? narrow_bwd_launch<T, 2>(x, f, s)
           : x.a.head_dim <= 4 ? narrow_bwd_launch<T, 4>(x, f, s)
                               : narrow_bwd_launch<T, 8>(x, f, s);
}

template <class T>
static fo_status fwd(const AttnArgs& x, void* ws, hipStream_t s) {
    const fo_attn& a = x.a;
    FwdShape f = fwd_shape(a);
    f.vec = vec_fwd(x);
    f.part = (float*)ws;
    f.ml = f.part + (int64_t)f.splits * a.heads * a.q_rows * a.head_dim;
    const fo_status st = f.narrow           ? fwd_narrow<T>(x, f, s)
                         : a.head_dim <= 32 ? attn_fwd_launch<T, 32>(x, f, s)
                         : a.head_dim <= 64 ? attn_fwd_launch<T, 64>(x, f, s)
                                            : attn_fwd_launch<T, 128>(x, f, s);
    if (st != FO_OK || f.splits == 1) return st;
    join_slices<T><<<(unsigned)cdiv((int64_t)a.batch * a.max_q * a.heads, 4), 256, 0, s>>>(x, f);
    FO_LAUNCHED();
    return FO_OK;
}

fo_status launch_attn_op_fwd(const AttnArgs& x, void* ws, hipStream_t s) {
    return x.a.dtype == FO_DT_BF16 ? fwd<bf16_t>(x, ws, s) : fwd<float>(x, ws, s);
}

template <class T>
static fo_status bias_gradient(const AttnArgs& x, const BwdShape& f, hipStream_t s) {
    if (!x.a.table) return FO_OK;
    bucket_sums<T><<<(unsigned)x.a.heads, 1024, 0, s>>>(x, f.q_parts * f.k_tiles * x.a.batch);
    FO_LAUNCHED();
    return FO_OK;
}

// One launch for sequences that a workgroup holds whole (attn_small.h).
static bool short_sequences(const fo_attn& a) {
    return a.max_q >= 1 && a.max_q <= 128 && a.max_k >= 1 && a.max_k <= 128 && a.heads == a.kv_heads;
}
template <class T>
static bool small_holds(const fo_attn& a) {
    if (a.head_dim <= 32) return small_fits<T, 32>(a);
    if (a.head_dim <= 64) return small_fits<T, 64>(a);
    if constexpr (sizeof(T) == 2) return small_fits<T, 128>(a);
    return false;  // fp32 rows of 128 do not fit
}
template <class T>
static fo_status run_small(const AttnArgs& x, hipStream_t s) {
    if (x.a.head_dim <= 32) return small_bwd_launch<T, 32>(x, s);
    if constexpr (sizeof(T) == 2)
        if (x.a.head_dim > 64) return small_bwd_launch<T, 128>(x, s);
    return small_bwd_launch<T, 64>(x, s);
}

template <class T>
static fo_status bwd(AttnArgs& x, float* ws, hipStream_t s) {
    const fo_attn& a = x.a;
    const int64_t e = sizeof(T);
    BwdShape f = bwd_shape(a);
    x.delta = ws;
    f.part = ws + stat_floats(a);
    x.hist = f.part + part_floats(a, f);
    f.vec = vec_fwd(x) && aligned_rows(x.dout, a.out_ld, a.out_hs, e) && aligned_rows(x.dq, a.q_ld, a.q_hs, e) &&
            aligned_rows(x.dk, a.k_ld, a.k_hs, e) && aligned_rows(x.dv, a.v_ld, a.v_hs, e);
    if (f.vec && a.q_rows && a.k_rows && short_sequences(a) && small_holds<T>(a)) {
        f.k_tiles = f.h_parts = f.q_parts = 1;
        const fo_status st = run_small<T>(x, s);
        if (st != FO_OK) return st;
        return bias_gradient<T>(x, f, s);
    }
    const fo_status st = f.narrow           ? bwd_narrow<T>(x, f, s)
                         : a.head_dim <= 32 ? attn_bwd_launch<T, 32>(x, f, s)
                         : a.head_dim <= 64 ? attn_bwd_launch<T, 64>(x, f, s)
                                            : attn_bwd_launch<T, 128>(x, f, s);
    if (st != FO_OK) return st;
    if (part_floats(a, f)) {
        join_keys<T><<<(unsigned)cdiv((int64_t)a.batch * a.max_k * a.kv_heads, 4), 256, 0, s>>>(x, f);
        FO_LAUNCHED();
    }
    return bias_gradient<T>(x, f, s);
}

fo_status launch_attn_op_bwd(AttnArgs& x, void* ws, hipStream_t s) {
    return x.a.dtype == FO_DT_BF16 ? bwd<bf16_t>(x, (float*)ws, s) : bwd<float>(x, (float*)ws, s);
}

}  // namespace fo
