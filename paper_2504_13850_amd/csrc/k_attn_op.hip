// Masked attention with capped scores, a learned bias by distance and dropout
// (fedoptima_ops.h): the plainest form, one wave per row.
#include "ops.h"

namespace fo {
namespace {

constexpr int DMAX = 128;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

template <class T>
__device__ __forceinline__ float dot(const float* x, const T* y, int d) {
    float s = 0.f;
    for (int c = 0; c < d; ++c) s = fmaf(x[c], to_f(y[c]), s);
    return s;
}

// One past the last key that query i sees (of one contiguous range starting at 0).
__device__ __forceinline__ int limit_of(const fo_attn& a, const Span& s, int b, int i) {
    if (a.mask == FO_ATTN_FULL) return s.nk;
    int m = i + (s.nk - s.nq) + 1;
    if (a.mask == FO_ATTN_PREFIX) m = max(m, a.prefix[b]);
    return max(0, min(m, s.nk));
}

// u of a pair and the derivative du / ds of its cap.
template <class T>
__device__ __forceinline__ float score(const fo_attn& a, float s, int n, int h, float* slope) {
    *slope = 1.f;
    if (a.cap > 0.f) {
        const float t = tanhf(s / a.cap);
        s = a.cap * t;
        *slope = 1.f - t * t;
    }
    if (a.table) {
        int g = a.bucket[min(max(n, -a.radius), a.radius) + a.radius];
        g = min(max(g, 0), a.n_buckets - 1);
        const float t = to_f(((const T*)a.table)[(int64_t)g * a.heads + h]);
        s = t <= -1e30f ? -INFINITY : s + t;
    }
    return s;
}

__device__ __forceinline__ float drop_of(const AttnArgs& x, int b, int h, int i, int j) {
    if (!x.thr) return 1.f;
    const uint4 w = philox7(2 * (j >> 4) + ((j >> 2) & 1), i, b * x.a.heads + h, x.a.offset, (uint32_t)x.a.seed,
                            (uint32_t)(x.a.seed >> 32));
    return half_of(w, (j & 3) + 4 * ((j >> 3) & 1)) >= x.thr ? x.keep_scale : 0.f;
}

template <class T>
__global__ void __launch_bounds__(64) fwd_rows(AttnArgs x) {
    const fo_attn& a = x.a;
    const int lane = threadIdx.x, i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, D = a.head_dim;
    const Span s = span_of(a, b);
    if (i >= s.nq) return;
    __shared__ float qs[DMAX], ps[64];
    const int hk = h / (a.heads / a.kv_heads);
    const T* q = (const T*)x.q + (int64_t)(s.q0 + i) * a.q_ld + h * a.q_hs;
    for (int c = lane; c < D; c += 64) qs[c] = to_f(q[c]);
    __syncthreads();
    const int lim = limit_of(a, s, b, i), off = s.nk - s.nq;
    float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f}, slope;
    for (int j0 = 0; j0 < lim; j0 += 64) {
        const int j = j0 + lane;
        float u = -INFINITY;
        if (j < lim)
            u = score<T>(a, a.scale * dot(qs, (const T*)x.k + (int64_t)(s.k0 + j) * a.k_ld + hk * a.k_hs, D),
                         j - i - off, h, &slope);
        const float mn = fmaxf(m, wave_max(u)), m0 = mn == -INFINITY ? 0.f : mn, f = expf(m - m0);
        const float p = expf(u - m0);
        l = l * f + wave_sum(p);
        ps[lane] = j < lim ? p * drop_of(x, b, h, i, j) : 0.f;
        __syncthreads();
        o[0] *= f;
        o[1] *= f;
        for (int t = 0; t < min(64, lim - j0); ++t) {
            const T* v = (const T*)x.v + (int64_t)(s.k0 + j0 + t) * a.v_ld + hk * a.v_hs;
            if (lane < D) o[0] = fmaf(ps[t], to_f(v[lane]), o[0]);
            if (lane + 64 < D) o[1] = fmaf(ps[t], to_f(v[lane + 64]), o[1]);
        }
        __syncthreads();
        m = mn;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    T* out = (T*)x.out + (int64_t)(s.q0 + i) * a.out_ld + h * a.out_hs;
    if (lane < D) out[lane] = from_f<T>(o[0] * inv);
    if (lane + 64 < D) out[lane + 64] = from_f<T>(o[1] * inv);
    if (x.lse && lane == 0) x.lse[(int64_t)h * a.q_rows + s.q0 + i] = l > 0.f ? m + logf(l) : -INFINITY;
}

// P and dP of one pair; both rows in LDS as floats.
template <class T>
__device__ __forceinline__ float pair_grad(const AttnArgs& x, int b, int h, int i, int j, int off, float s, float dp,
                                           float lse, float* p, float* drop, float* slope) {
    const float u = score<T>(x.a, x.a.scale * s, j - i - off, h, slope);
    *p = u == -INFINITY ? 0.f : expf(u - lse);
    *drop = drop_of(x, b, h, i, j);
    return dp * *drop;
}

template <class T>
__global__ void __launch_bounds__(64) dq_rows(AttnArgs x) {
    const fo_attn& a = x.a;
    const int lane = threadIdx.x, i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, D = a.head_dim;
    const Span sp = span_of(a, b);
    if (i >= sp.nq) return;
    __shared__ float qs[DMAX], gs[DMAX], ds[64];
    const int hk = h / (a.heads / a.kv_heads);
    const T* q = (const T*)x.q + (int64_t)(sp.q0 + i) * a.q_ld + h * a.q_hs;
    const T* g = (const T*)x.dout + (int64_t)(sp.q0 + i) * a.out_ld + h * a.out_hs;
    for (int c = lane; c < D; c += 64) qs[c] = to_f(q[c]), gs[c] = to_f(g[c]);
    __syncthreads();
    const int lim = limit_of(a, sp, b, i), off = sp.nk - sp.nq;
    const float lse = x.lse[(int64_t)h * a.q_rows + sp.q0 + i];
    float delta = 0.f, o[2] = {0.f, 0.f}, p, drop, slope;
    for (int pass = 0; pass < 2; ++pass) {
        float part = 0.f;
        for (int j0 = 0; j0 < lim; j0 += 64) {
            const int j = j0 + lane;
            float d = 0.f;
            if (j < lim) {
                const T* k = (const T*)x.k + (int64_t)(sp.k0 + j) * a.k_ld + hk * a.k_hs;
                const T* v = (const T*)x.v + (int64_t)(sp.k0 + j) * a.v_ld + hk * a.v_hs;
                const float dp = pair_grad<T>(x, b, h, i, j, off, dot(qs, k, D), dot(gs, v, D), lse, &p, &drop, &slope);
                part += p * dp;
                d = p * (dp - delta) * slope;
            }
            if (!pass) continue;
            ds[lane] = d;
            __syncthreads();
            for (int t = 0; t < min(64, lim - j0); ++t) {
                const T* k = (const T*)x.k + (int64_t)(sp.k0 + j0 + t) * a.k_ld + hk * a.k_hs;
                if (lane < D) o[0] = fmaf(ds[t], to_f(k[lane]), o[0]);
                if (lane + 64 < D) o[1] = fmaf(ds[t], to_f(k[lane + 64]), o[1]);
            }
            __syncthreads();
        }
        if (!pass) delta = wave_sum(part);
    }
    T* dq = (T*)x.dq + (int64_t)(sp.q0 + i) * a.q_ld + h * a.q_hs;
    if (lane < D) dq[lane] = from_f<T>(o[0] * a.scale);
    if (lane + 64 < D) dq[lane + 64] = from_f<T>(o[1] * a.scale);
    if (lane == 0) x.delta[(int64_t)h * a.q_rows + sp.q0 + i] = delta;
}

template <class T>
__global__ void __launch_bounds__(64) dkv_rows(AttnArgs x) {
    const fo_attn& a = x.a;
    const int lane = threadIdx.x, j = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, D = a.head_dim;
    const Span sp = span_of(a, b);
    if (j >= sp.nk) return;
    __shared__ float ks[DMAX], vs[DMAX], ps[64], ds[64];
    const T* k = (const T*)x.k + (int64_t)(sp.k0 + j) * a.k_ld + hk * a.k_hs;
    const T* v = (const T*)x.v + (int64_t)(sp.k0 + j) * a.v_ld + hk * a.v_hs;
    for (int c = lane; c < D; c += 64) ks[c] = to_f(k[c]), vs[c] = to_f(v[c]);
    __syncthreads();
    const int off = sp.nk - sp.nq, G = a.heads / a.kv_heads;
    float ok[2] = {0.f, 0.f}, ov[2] = {0.f, 0.f}, p, drop, slope;
    for (int h = hk * G; h < hk * G + G; ++h)
        for (int i0 = 0; i0 < sp.nq; i0 += 64) {
            const int i = i0 + lane;
            float pd = 0.f, d = 0.f;
            if (i < sp.nq && j < limit_of(a, sp, b, i)) {
                const T* q = (const T*)x.q + (int64_t)(sp.q0 + i) * a.q_ld + h * a.q_hs;
                const T* g = (const T*)x.dout + (int64_t)(sp.q0 + i) * a.out_ld + h * a.out_hs;
                const int64_t r = (int64_t)h * a.q_rows + sp.q0 + i;
                const float dp = pair_grad<T>(x, b, h, i, j, off, dot(ks, q, D), dot(vs, g, D), x.lse[r], &p, &drop,
                                              &slope);
                pd = p * drop;
                d = p * (dp - x.delta[r]) * slope;
            }
            ps[lane] = pd;
            ds[lane] = d;
            __syncthreads();
            for (int t = 0; t < min(64, sp.nq - i0); ++t) {
                const T* q = (const T*)x.q + (int64_t)(sp.q0 + i0 + t) * a.q_ld + h * a.q_hs;
                const T* g = (const T*)x.dout + (int64_t)(sp.q0 + i0 + t) * a.out_ld + h * a.out_hs;
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (lane + 64 * c < D) {
                        ok[c] = fmaf(ds[t], to_f(q[lane + 64 * c]), ok[c]);
                        ov[c] = fmaf(ps[t], to_f(g[lane + 64 * c]), ov[c]);
                    }
            }
            __syncthreads();
        }
    T* dk = (T*)x.dk + (int64_t)(sp.k0 + j) * a.k_ld + hk * a.k_hs;
    T* dv = (T*)x.dv + (int64_t)(sp.k0 + j) * a.v_ld + hk * a.v_hs;
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (lane + 64 * c < D) {
            dk[lane + 64 * c] = from_f<T>(ok[c] * a.scale);
            dv[lane + 64 * c] = from_f<T>(ov[c]);
        }
}

// The bias gradient by (clamped) distance: one wave per sequence, head and distance.
template <class T>
__global__ void __launch_bounds__(64) dist_sums(AttnArgs x) {
    const fo_attn& a = x.a;
    const int lane = threadIdx.x, h = blockIdx.y, b = blockIdx.z, D = a.head_dim, R = a.radius;
    const int n0 = (int)blockIdx.x - R;
    const Span sp = span_of(a, b);
    const int off = sp.nk - sp.nq, hk = h / (a.heads / a.kv_heads);
    float sum = 0.f, p, drop, slope;
    for (int i = lane; i < sp.nq; i += 64) {
        const int lim = limit_of(a, sp, b, i);
        const T* q = (const T*)x.q + (int64_t)(sp.q0 + i) * a.q_ld + h * a.q_hs;
        const T* g = (const T*)x.dout + (int64_t)(sp.q0 + i) * a.out_ld + h * a.out_hs;
        const int64_t r = (int64_t)h * a.q_rows + sp.q0 + i;
        const int lo = n0 == -R ? 0 : n0 + i + off, hi = n0 == R ? lim - 1 : n0 + i + off;
        for (int j = max(lo, 0); j <= min(hi, lim - 1); ++j) {
            const T* k = (const T*)x.k + (int64_t)(sp.k0 + j) * a.k_ld + hk * a.k_hs;
            const T* v = (const T*)x.v + (int64_t)(sp.k0 + j) * a.v_ld + hk * a.v_hs;
            float s = 0.f, dp = 0.f;
            for (int c = 0; c < D; ++c) s = fmaf(to_f(q[c]), to_f(k[c]), s), dp = fmaf(to_f(g[c]), to_f(v[c]), dp);
            dp = pair_grad<T>(x, b, h, i, j, off, s, dp, x.lse[r], &p, &drop, &slope);
            sum += p * (dp - x.delta[r]);
        }
    }
    sum = wave_sum(sum);
    if (lane == 0) x.hist[((int64_t)b * a.heads + h) * (2 * R + 1) + blockIdx.x] = sum;
}

template <class T>
__global__ void __launch_bounds__(64) bucket_sums(AttnArgs x) {
    const fo_attn& a = x.a;
    const int g = blockIdx.x, h = blockIdx.y, W = 2 * a.radius + 1;
    float s = 0.f;
    for (int n = threadIdx.x; n < W; n += 64)
        if (min(max(a.bucket[n], 0), a.n_buckets - 1) == g)
            for (int b = 0; b < a.batch; ++b) s += x.hist[((int64_t)b * a.heads + h) * W + n];
    s = wave_sum(s);
    if (threadIdx.x == 0) ((T*)x.dtable)[(int64_t)g * a.heads + h] = from_f<T>(s);
}

template <class T>
fo_status fwd(const AttnArgs& x, hipStream_t s) {
    fwd_rows<T><<<dim3(x.a.max_q, x.a.heads, x.a.batch), 64, 0, s>>>(x);
    FO_LAUNCHED();
    return FO_OK;
}
template <class T>
fo_status bwd(const AttnArgs& x, hipStream_t s) {
    const fo_attn& a = x.a;
    if (a.max_q) dq_rows<T><<<dim3(a.max_q, a.heads, a.batch), 64, 0, s>>>(x);
    FO_LAUNCHED();
    if (a.max_k) dkv_rows<T><<<dim3(a.max_k, a.kv_heads, a.batch), 64, 0, s>>>(x);
    FO_LAUNCHED();
    if (a.table) {
        dist_sums<T><<<dim3(2 * a.radius + 1, a.heads, a.batch), 64, 0, s>>>(x);
        FO_LAUNCHED();
        bucket_sums<T><<<dim3(a.n_buckets, a.heads), 64, 0, s>>>(x);
        FO_LAUNCHED();
    }
    return FO_OK;
}

}  // namespace

int64_t attn_workspace(const fo_attn& a, bool backward) {
    if (!backward) return 0;
    const int64_t rows = ((a.q_rows * a.heads + 3) & ~int64_t(3)) * 4;
    return rows + (a.table ? (int64_t)a.batch * a.heads * (2 * a.radius + 1) * 4 : 0);
}

fo_status launch_attn_op_fwd(const AttnArgs& x, void*, hipStream_t s) {
    return x.a.dtype == FO_DT_BF16 ? fwd<bf16_t>(x, s) : fwd<float>(x, s);
}

fo_status launch_attn_op_bwd(AttnArgs& x, void* ws, hipStream_t s) {
    x.delta = (float*)ws;
    x.hist = x.delta + ((x.a.q_rows * x.a.heads + 3) & ~int64_t(3));
    return x.a.dtype == FO_DT_BF16 ? bwd<bf16_t>(x, s) : bwd<float>(x, s);
}

}  // namespace fo
