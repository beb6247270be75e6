// The attention operator for heads of up to eight columns: products this narrow
// would leave a 32x32 matrix tile mostly empty (fp32 heads of width 2: 1/16 of a
// score product's columns, 1/16 of an output's rows), so each lane takes a row of
// its own and the other side's rows are broadcast from LDS.  A wave is on its own:
// no barrier, and the four waves of a workgroup have different heads or rows.
//
// Bound by the vector unit: about 30 instructions a pair forward, most of them
// the cap's and the softmax's exponentials; the two gradient kernels compute score, cap
// and exponential again, each.  16 sequences of 16 to 256 tokens, fp32, 50 heads of width
// 2, capped at 30: 28 us forward, 34 and 37 us for the gradient kernels, 92 us in all
// where the scores stay below a third of the cap (cap_scores), 123 where they are as
// large as it, 66 without a cap.
#pragma once

#include "attn_bwd.h"
#include "attn_fwd.h"

namespace fo {

template <class T, int DN>
__device__ __forceinline__ void ld_narrow(float* v, const T* row, int D, bool ok) {
#pragma unroll
    for (int d = 0; d < DN; ++d) v[d] = ok && d < D ? to_f(row[d]) : 0.f;
}
template <int DN>
__device__ __forceinline__ float dot_narrow(const float* x, const float* y) {
    float s = x[0] * y[0];
#pragma unroll
    for (int d = 1; d < DN; ++d) s = fmaf(x[d], y[d], s);
    return s;
}
// Scores -> u log2(e) + add, and du/ds.
template <class T, bool CAP, int N>
__device__ __forceinline__ void narrow_exponent(float (&S)[N], float* slope, const ScoreK& k, float mul, float add) {
    if (CAP) cap_scores<T, N>(S, k, slope);
#pragma unroll
    for (int r = 0; r < N; ++r) S[r] = fmaf(S[r], CAP ? k.cl : mul, add);
}

// Rows of one wave: 64 queries of head h (fwd, dq) or 64 keys of head hk.
constexpr int kNarrowRows = 64;

template <class T, int DN, bool CAP, bool EXTRA>
__global__ void __launch_bounds__(256) narrow_fwd(AttnArgs x, FwdShape f) {
    __shared__ __attribute__((aligned(16))) float kv_all[4][64 * 2 * DN];
    extern __shared__ float lut_all[];
    const fo_attn& a = x.a;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, D = a.head_dim;
    int id = __builtin_amdgcn_readfirstlane(block_of() * 4 + w);
    const int split = id % f.splits;
    id /= f.splits;
    const int h = id % a.heads, hk = h / (a.heads / a.kv_heads);
    id /= a.heads;
    const int b = id % a.batch, i0 = (f.row_tiles - 1 - id / a.batch) * kNarrowRows;
    if (i0 < 0) return;
    const Span s = span_of(a, b);
    if (i0 >= s.nq) return;
    const int pre = a.mask == FO_ATTN_PREFIX ? a.prefix[b] : 0, off = s.nk - s.nq;
    const int qi = i0 + lane;
    const bool ok = qi < s.nq;
    const int lim = ok ? limit_of(a, s, pre, qi) : 0x7fffffff;
    const int end = limit_of(a, s, pre, min(i0 + kNarrowRows, s.nq) - 1), all = limit_of(a, s, pre, i0);
    const int tiles = (end + 63) / 64, per = (tiles + f.splits - 1) / f.splits;
    const int t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);
    float* kv = kv_all[w];
    const T* kb = (const T*)x.k + (int64_t)s.k0 * a.k_ld + hk * a.k_hs;
    const T* vb = (const T*)x.v + (int64_t)s.k0 * a.v_ld + hk * a.v_hs;
    float q[DN], nk[DN], nv[DN];
    ld_narrow<T, DN>(q, (const T*)x.q + (int64_t)(s.q0 + (ok ? qi : 0)) * a.q_ld + h * a.q_hs, D, ok);
    const ScoreK sc = score_k(a);
    const float mul = a.scale * kLog2e;
    const bool bias = EXTRA && a.table != nullptr;
    float far_lo = 0.f, far_hi = 0.f, *lut = lut_all + w * lut_floats(a);
    if (bias) {
        far_lo = bias_at<T>(a, h, -a.radius);
        far_hi = bias_at<T>(a, h, a.radius);
        fill_lut<T>(lut, a, h, lane, 64);
        wave_sync();
    }
    auto load = [&](int t) {
        const int j = t * 64 + lane;
        const bool in = j < s.nk;
        ld_narrow<T, DN>(nk, kb + (int64_t)(in ? j : 0) * a.k_ld, D, in);
        ld_narrow<T, DN>(nv, vb + (int64_t)(in ? j : 0) * a.v_ld, D, in);
    };
    if (t0 < t1) load(t0);
    float m = -INFINITY, l = 0.f, O[DN] = {};
    for (int t = t0; t < t1; ++t) {
        wave_sync();
#pragma unroll
        for (int d = 0; d < DN; ++d) kv[lane * 2 * DN + d] = nk[d], kv[lane * 2 * DN + DN + d] = nv[d];
        wave_sync();
        if (t + 1 < t1) load(t + 1);
        for (int g = 0; g < 4; ++g) {
            const int j0 = t * 64 + 16 * g;
            if (j0 >= end) break;
            const int n_lo = j0 - (i0 + 63) - off, n_hi = j0 + 15 - i0 - off;
            const bool near = EXTRA && bias && n_lo < a.radius && n_hi > -a.radius;
            const float add0 = !EXTRA || !bias || near ? 0.f : n_lo >= a.radius ? far_hi : far_lo;
            float S[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) S[r] = dot_narrow<DN>(q, &kv[(16 * g + r) * 2 * DN]);
            narrow_exponent<T, CAP, 16>(S, nullptr, sc, mul, add0);
            if (near) {
                const float* at = &lut[j0 - qi - off + a.radius + kReach];
#pragma unroll
                for (int r = 0; r < 16; ++r) S[r] += at[r];
            }
            if (j0 + 16 > all) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (j0 + r >= lim) S[r] = -INFINITY;
            }
            float mt = S[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mt = fmaxf(mt, S[r]);
            const float mn = fmaxf(m, mt);
            if (__any(mn > m + 8.f)) {  // see attn_fwd_kernel
                const float c = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.f : mn));
                l *= c;
#pragma unroll
                for (int d = 0; d < DN; ++d) O[d] *= c;
                m = mn;
            }
            const float sub = m == -INFINITY ? 0.f : m;
            uint32_t bits[2] = {0xFFFFu, 0xFFFFu};
            if (EXTRA && x.thr) {
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const uint4 c = philox7(2 * (j0 >> 4) + hh, qi, b * a.heads + h, a.offset, (uint32_t)a.seed,
                                            (uint32_t)(a.seed >> 32));
                    bits[hh] = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) bits[hh] |= (half_of(c, e) >= x.thr ? 1u : 0u) << e;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float p = __builtin_amdgcn_exp2f(S[r] - sub);
                l += p;
                if (EXTRA && x.thr) p = (bits[(r >> 2) & 1] >> ((r & 3) | ((r >> 1) & 4))) & 1 ? p : 0.f;
#pragma unroll
                for (int d = 0; d < DN; ++d) O[d] = fmaf(p, kv[(16 * g + r) * 2 * DN + DN + d], O[d]);
            }
        }
    }
    if (!ok) return;
    if (f.splits > 1) {
        const int64_t at = ((int64_t)split * a.heads + h) * a.q_rows + s.q0 + qi;
#pragma unroll
        for (int d = 0; d < DN; ++d)
            if (d < D) f.part[at * D + d] = O[d];
        f.ml[2 * at] = m;
        f.ml[2 * at + 1] = l;
        return;
    }
    const float inv = l > 0.f ? x.keep_scale / l : 0.f;
    T* out = (T*)x.out + (int64_t)(s.q0 + qi) * a.out_ld + h * a.out_hs;
#pragma unroll
    for (int d = 0; d < DN; ++d)
        if (d < D) out[d] = from_f<T>(O[d] * inv);
    if (x.lse) x.lse[(int64_t)h * a.q_rows + s.q0 + qi] = l > 0.f ? m + __builtin_amdgcn_logf(l) : -INFINITY;
}

// dq and delta: see attn_dq_kernel.
template <class T, int DN, bool CAP, bool EXTRA>
__global__ void __launch_bounds__(256) narrow_dq(AttnArgs x, BwdShape f) {
    constexpr bool FIX = sizeof(T) == 2;
    __shared__ __attribute__((aligned(16))) float kv_all[4][64 * 2 * DN];
    extern __shared__ float lut_all[];
    const fo_attn& a = x.a;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, D = a.head_dim;
    int id = __builtin_amdgcn_readfirstlane(block_of() * 4 + w);
    const int h = id % a.heads, hk = h / (a.heads / a.kv_heads);
    id /= a.heads;
    const int b = id % a.batch, i0 = (f.q_tiles - 1 - id / a.batch) * kNarrowRows;
    if (i0 < 0) return;
    const Span s = span_of(a, b);
    if (i0 >= s.nq) return;
    const int pre = a.mask == FO_ATTN_PREFIX ? a.prefix[b] : 0, off = s.nk - s.nq;
    const int qi = i0 + lane;
    const bool ok = qi < s.nq;
    const int lim = ok ? limit_of(a, s, pre, qi) : 0;
    const int end = limit_of(a, s, pre, min(i0 + kNarrowRows, s.nq) - 1);
    const int all = i0 + kNarrowRows <= s.nq ? limit_of(a, s, pre, i0) : 0;
    const int tiles = (end + 63) / 64;
    float* kv = kv_all[w];
    const T* kb = (const T*)x.k + (int64_t)s.k0 * a.k_ld + hk * a.k_hs;
    const T* vb = (const T*)x.v + (int64_t)s.k0 * a.v_ld + hk * a.v_hs;
    const int64_t row = s.q0 + (ok ? qi : 0), stat = (int64_t)h * a.q_rows + s.q0 + qi;
    float q[DN], g[DN], o[DN], nk[DN], nv[DN];
    ld_narrow<T, DN>(q, (const T*)x.q + row * a.q_ld + h * a.q_hs, D, ok);
    ld_narrow<T, DN>(g, (const T*)x.dout + row * a.out_ld + h * a.out_hs, D, ok);
    ld_narrow<T, DN>(o, (const T*)x.out + row * a.out_ld + h * a.out_hs, D, ok);
    const float dl = dot_narrow<DN>(g, o);
    float lse = ok ? x.lse[stat] : INFINITY;
    if (lse == -INFINITY) lse = INFINITY;
    const ScoreK sc = score_k(a);
    const float mul = a.scale * kLog2e;
    const bool bias = EXTRA && a.table != nullptr;
    float far_lo = 0.f, far_hi = 0.f, *lut = lut_all + w * lut_floats(a);
    if (bias) {
        far_lo = bias_at<T>(a, h, -a.radius);
        far_hi = bias_at<T>(a, h, a.radius);
        fill_lut<T>(lut, a, h, lane, 64);
        wave_sync();
    }
    auto load = [&](int t) {
        const int j = t * 64 + lane;
        const bool in = j < s.nk;
        ld_narrow<T, DN>(nk, kb + (int64_t)(in ? j : 0) * a.k_ld, D, in);
        ld_narrow<T, DN>(nv, vb + (int64_t)(in ? j : 0) * a.v_ld, D, in);
    };
    if (tiles) load(0);
    float dQ[DN] = {}, X[DN] = {}, err = 0.f;
    for (int t = 0; t < tiles; ++t) {
        wave_sync();
#pragma unroll
        for (int d = 0; d < DN; ++d) kv[lane * 2 * DN + d] = nk[d], kv[lane * 2 * DN + DN + d] = nv[d];
        wave_sync();
        if (t + 1 < tiles) load(t + 1);
        for (int gr = 0; gr < 4; ++gr) {
            const int j0 = t * 64 + 16 * gr;
            if (j0 >= end) break;
            const int n_lo = j0 - (i0 + 63) - off, n_hi = j0 + 15 - i0 - off;
            const bool near = EXTRA && bias && n_lo < a.radius && n_hi > -a.radius;
            const float add0 = !EXTRA || !bias || near ? 0.f : n_lo >= a.radius ? far_hi : far_lo;
            const float* at = near ? &lut[j0 - qi - off + a.radius + kReach] : nullptr;
            const bool masked = j0 + 16 > all;
            uint32_t bits[2] = {0xFFFFu, 0xFFFFu};
            if (EXTRA && x.thr) {
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const uint4 c = philox7(2 * (j0 >> 4) + hh, qi, b * a.heads + h, a.offset, (uint32_t)a.seed,
                                            (uint32_t)(a.seed >> 32));
                    bits[hh] = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) bits[hh] |= (half_of(c, e) >= x.thr ? 1u : 0u) << e;
                }
            }
            float S[16], slope[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) S[r] = dot_narrow<DN>(q, &kv[(16 * gr + r) * 2 * DN]);
            narrow_exponent<T, CAP, 16>(S, slope, sc, mul, add0 - lse);
            if (near) {
#pragma unroll
                for (int r = 0; r < 16; ++r) S[r] += at[r];
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float* kr = &kv[(16 * gr + r) * 2 * DN];
                float p = __builtin_amdgcn_exp2f(S[r]);
                if (masked) p = j0 + r < lim ? p : 0.f;
                float dp = dot_narrow<DN>(g, kr + DN);
                if (EXTRA && x.thr) dp = (bits[(r >> 2) & 1] >> ((r & 3) | ((r >> 1) & 4))) & 1 ? dp * x.keep_scale : 0.f;
                const float du = p * (dp - dl);
                err += du;
                const float ds = CAP ? du * slope[r] : du, ps = CAP ? p * slope[r] : p;
#pragma unroll
                for (int d = 0; d < DN; ++d) {
                    dQ[d] = fmaf(ds, kr[d], dQ[d]);
                    if (FIX) X[d] = fmaf(ps, kr[d], X[d]);
                }
            }
        }
    }
    if (!ok) return;
    T* dq = (T*)x.dq + (int64_t)(s.q0 + qi) * a.q_ld + h * a.q_hs;
#pragma unroll
    for (int d = 0; d < DN; ++d)
        if (d < D) dq[d] = from_f<T>((FIX ? fmaf(-err, X[d], dQ[d]) : dQ[d]) * a.scale);
    x.delta[stat] = FIX ? dl + err : dl;
}

// dk, dv and the bias sums: see attn_dkv_kernel.
template <class T, int DN, bool CAP, bool EXTRA>
__global__ void __launch_bounds__(256) narrow_dkv(AttnArgs x, BwdShape f) {
    constexpr int QW = 2 * DN + 2;  // a query's row in LDS: q, dO, lse, delta
    __shared__ __attribute__((aligned(16))) float qg_all[4][64 * QW];
    __shared__ uint64_t keep_all[4][64];
    extern __shared__ float dyn[];  // with a bias, per wave: its values by distance, and the sums
    const fo_attn& a = x.a;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int D = a.head_dim, G = a.heads / a.kv_heads, R = a.radius, W = lut_floats(a);
    int id = __builtin_amdgcn_readfirstlane(block_of() * 4 + w);
    const int hk = id % a.kv_heads;
    id /= a.kv_heads;
    const int b = id % a.batch;
    id /= a.batch;
    const int parts = f.h_parts * f.q_parts, part = id % parts, qp = part / f.h_parts, kt = id / parts;
    if (kt >= f.k_tiles) return;
    const int j0 = kt * kNarrowRows, hb = (G + f.h_parts - 1) / f.h_parts;
    const int h0 = min(part % f.h_parts * hb, G), h1 = min(h0 + hb, G);
    float* hist = EXTRA && a.table
                      ? x.hist + ((((int64_t)qp * f.k_tiles + kt) * a.batch + b) * a.heads + hk * G) * (2 * R + 1)
                      : nullptr;
    const Span s = span_of(a, b);
    if (j0 >= s.nk) {
        if (hist) each(lane, 64, (h1 - h0) * (2 * R + 1), [&](int e) { hist[h0 * (2 * R + 1) + e] = 0.f; });
        return;
    }
    const int pre = a.mask == FO_ATTN_PREFIX ? a.prefix[b] : 0, off = s.nk - s.nq;
    const int j = j0 + lane;
    const bool ok = j < s.nk;
    auto first_of = [&](int key) { return a.mask == FO_ATTN_FULL || key < pre ? 0 : max(0, key - off); };
    const int first = ok ? first_of(j) : 0x7fffffff;
    const int from = first_of(j0), all = j0 + kNarrowRows <= s.nk ? first_of(j0 + kNarrowRows - 1) : 0x7fffffff;
    int t0 = min(from, s.nq) / 64, t1 = (s.nq + 63) / 64;
    {
        const int per = (t1 - t0 + f.q_parts - 1) / f.q_parts;
        t0 = min(t0 + qp * per, t1);
        t1 = min(t0 + per, t1);
    }
    float k[DN], v[DN], dK[DN] = {}, dV[DN] = {};
    {
        const int64_t row = s.k0 + (ok ? j : 0);
        ld_narrow<T, DN>(k, (const T*)x.k + row * a.k_ld + hk * a.k_hs, D, ok);
        ld_narrow<T, DN>(v, (const T*)x.v + row * a.v_ld + hk * a.v_hs, D, ok);
    }
    const ScoreK sc = score_k(a);
    const float mul = a.scale * kLog2e;
    const bool bias = EXTRA && a.table != nullptr;
    float *qg = qg_all[w], *lut = dyn + 2 * w * W, *line = lut + W;
    for (int hg = h0; hg < h1; ++hg) {
        const int h = hk * G + hg;
        const T* qb = (const T*)x.q + (int64_t)s.q0 * a.q_ld + h * a.q_hs;
        const T* gb = (const T*)x.dout + (int64_t)s.q0 * a.out_ld + h * a.out_hs;
        const int64_t stat = (int64_t)h * a.q_rows + s.q0;
        float far_lo = 0.f, far_hi = 0.f, sum_lo = 0.f, sum_hi = 0.f;
        if (bias) {
            wave_sync();
            far_lo = bias_at<T>(a, h, -R);
            far_hi = bias_at<T>(a, h, R);
            fill_lut<T>(lut, a, h, lane, 64);
            each(lane, 64, W, [&](int n) { line[n] = 0.f; });
        }
        float nq[DN], ng[DN], nl = 0.f, nd = 0.f;
        auto load = [&](int t) {
            const int i = t * 64 + lane;
            const bool in = i < s.nq;
            ld_narrow<T, DN>(nq, qb + (int64_t)(in ? i : 0) * a.q_ld, D, in);
            ld_narrow<T, DN>(ng, gb + (int64_t)(in ? i : 0) * a.out_ld, D, in);
            nl = in ? x.lse[stat + i] : INFINITY;
            nd = in ? x.delta[stat + i] : 0.f;
            if (nl == -INFINITY) nl = INFINITY;
        };
        if (t0 < t1) load(t0);
        for (int t = t0; t < t1; ++t) {
            const int it = t * 64;
            wave_sync();
#pragma unroll
            for (int d = 0; d < DN; ++d) qg[lane * QW + d] = nq[d], qg[lane * QW + DN + d] = ng[d];
            qg[lane * QW + 2 * DN] = nl;
            qg[lane * QW + 2 * DN + 1] = nd;
            if (EXTRA && x.thr) {  // the 64 keys' bits for query it + lane
                uint64_t bits = 0;
                for (int mh = 0; mh < 8; ++mh) {
                    const uint4 c = philox7(2 * (j0 >> 4) + mh, it + lane, b * a.heads + h, a.offset,
                                            (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        bits |= (uint64_t)(half_of(c, e) >= x.thr ? 1 : 0)
                                << (16 * (mh >> 1) + 8 * (e >> 2) + 4 * (mh & 1) + (e & 3));
                }
                keep_all[w][lane] = bits;
            }
            wave_sync();
            if (t + 1 < t1) load(t + 1);
            const int n_lo = j0 - (min(it + 63, s.nq - 1)) - off, n_hi = j0 + 63 - it - off;
            // all of the tile's distances past the radius on one side: one bias for it
            const bool far = !EXTRA || !bias || n_lo >= R || n_hi <= -R, high = n_lo >= R;
            const float add0 = !EXTRA || !bias ? 0.f : high ? far_hi : far_lo;
            const bool masked = it < all;
            // eight rows at a time; rows past the last have P = 0
            for (int r8 = 0; r8 < 64 && it + r8 < s.nq; r8 += 8) {
              float S[8], slope[8];
#pragma unroll
              for (int r = 0; r < 8; ++r) S[r] = dot_narrow<DN>(k, &qg[(r8 + r) * QW]);
              narrow_exponent<T, CAP, 8>(S, slope, sc, mul, far ? add0 : 0.f);
#pragma unroll
              for (int r0 = 0; r0 < 8; ++r0) {
                const int r = r8 + r0;
                const float* qr = &qg[r * QW];
                const int at = min(max(j - it - r - off, -R), R) + R + kReach;
                if (EXTRA && bias && !far) S[r0] += lut[at];
                float p = __builtin_amdgcn_exp2f(S[r0] - qr[2 * DN]);
                if (masked) p = it + r >= first ? p : 0.f;
                float dp = dot_narrow<DN>(v, qr + DN), pd = p;
                if (EXTRA && x.thr) {
                    const bool kept = (keep_all[w][r] >> lane) & 1;
                    dp = kept ? dp * x.keep_scale : 0.f;
                    pd = kept ? p : 0.f;
                }
                const float du = p * (dp - qr[2 * DN + 1]);
                if (EXTRA && bias) {
                    if (far) {
                        if (high) sum_hi += du;
                        else sum_lo += du;
                    } else if (j - it - r - off >= R) {
                        sum_hi += du;
                    } else if (j - it - r - off <= -R) {
                        sum_lo += du;
                    } else {
                        line[at] += du;  // the lanes' distances are 64 different ones
                    }
                    wave_sync();
                }
                const float ds = CAP ? du * slope[r0] : du;
#pragma unroll
                for (int d = 0; d < DN; ++d) {
                    dK[d] = fmaf(ds, qr[d], dK[d]);
                    dV[d] = fmaf(pd, qr[DN + d], dV[d]);
                }
              }
            }
        }
        if (bias) {
            wave_sync();
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                sum_lo += __shfl_xor(sum_lo, o);
                sum_hi += __shfl_xor(sum_hi, o);
            }
            float* out = hist + hg * (2 * R + 1);
            each(lane, 64, 2 * R - 1, [&](int n) { out[1 + n] = line[1 + n + kReach]; });
            if (lane == 0) {  // nothing is ever added to the lines of the radius itself
                if (R == 0) {
                    out[0] = sum_lo + sum_hi;
                } else {
                    out[0] = sum_lo;
                    out[2 * R] = sum_hi;
                }
            }
        }
    }
    if (!ok) return;
    if (parts > 1) {
        const int64_t at = (((int64_t)part * a.k_rows + s.k0 + j) * a.kv_heads + hk) * D;
        const int64_t step = (int64_t)parts * a.k_rows * a.kv_heads * D;
#pragma unroll
        for (int d = 0; d < DN; ++d)
            if (d < D) f.part[at + d] = dK[d], f.part[step + at + d] = dV[d];
        return;
    }
    T* dk = (T*)x.dk + (int64_t)(s.k0 + j) * a.k_ld + hk * a.k_hs;
    T* dv = (T*)x.dv + (int64_t)(s.k0 + j) * a.v_ld + hk * a.v_hs;
#pragma unroll
    for (int d = 0; d < DN; ++d)
        if (d < D) {
            dk[d] = from_f<T>(dK[d] * a.scale);
            dv[d] = from_f<T>(dV[d] * x.keep_scale);
        }
}

// (defined for every type and width in a file of its own)
template <class T, int DN>
fo_status narrow_fwd_launch(const AttnArgs& x, const FwdShape& f, hipStream_t s) {
    const fo_attn& a = x.a;
    const dim3 n = grid_of(cdiv((int64_t)f.row_tiles * a.heads * a.batch * f.splits, 4));
    const unsigned lds = a.table ? 16 * lut_floats(a) : 0;
    const bool cap = a.cap > 0.f, extra = a.table || x.thr;
    if (cap && extra) narrow_fwd<T, DN, true, true><<<n, 256, lds, s>>>(x, f);
    else if (cap) narrow_fwd<T, DN, true, false><<<n, 256, lds, s>>>(x, f);
    else if (extra) narrow_fwd<T, DN, false, true><<<n, 256, lds, s>>>(x, f);
    else narrow_fwd<T, DN, false, false><<<n, 256, lds, s>>>(x, f);
    FO_LAUNCHED();
    return FO_OK;
}
template <class T, int DN>
fo_status narrow_bwd_launch(const AttnArgs& x, const BwdShape& f, hipStream_t s) {
    const fo_attn& a = x.a;
    const unsigned lds = a.table ? 16 * lut_floats(a) : 0;
    const bool cap = a.cap > 0.f, extra = a.table || x.thr;
    if (f.q_tiles) {
        const dim3 n = grid_of(cdiv((int64_t)f.q_tiles * a.heads * a.batch, 4));
        if (cap && extra) narrow_dq<T, DN, true, true><<<n, 256, lds, s>>>(x, f);
        else if (cap) narrow_dq<T, DN, true, false><<<n, 256, lds, s>>>(x, f);
        else if (extra) narrow_dq<T, DN, false, true><<<n, 256, lds, s>>>(x, f);
        else narrow_dq<T, DN, false, false><<<n, 256, lds, s>>>(x, f);
        FO_LAUNCHED();
    }
    if (f.k_tiles) {
        const dim3 n = grid_of(cdiv((int64_t)f.k_tiles * f.h_parts * f.q_parts * a.kv_heads * a.batch, 4));
        if (cap && extra) narrow_dkv<T, DN, true, true><<<n, 256, 2 * lds, s>>>(x, f);
        else if (cap) narrow_dkv<T, DN, true, false><<<n, 256, 2 * lds, s>>>(x, f);
        else if (extra) narrow_dkv<T, DN, false, true><<<n, 256, 2 * lds, s>>>(x, f);
        else narrow_dkv<T, DN, false, false><<<n, 256, 2 * lds, s>>>(x, f);
        FO_LAUNCHED();
    }
    return FO_OK;
}

}  // namespace fo
