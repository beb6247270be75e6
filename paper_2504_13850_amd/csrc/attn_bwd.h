// Backward kernels of the attention operator, instantiated per type and width.
//
//   P = softmax(u), dP_ij = drop_ij dO_i.v_j, delta_i = sum_j P_ij dP_ij,
//   dU = P (dP - delta), dS = dU du/ds
//   dq_i = scale sum_j dS_ij k_j, dk_j = scale sum_i dS_ij q_i,
//   dv_j = sum_i P_ij drop_ij dO_i, dtable[bucket] = sum of dU over its pairs
//
// Two passes over the scores, so that every sum has one owner and a fixed order:
// the query kernel (dq and delta), then the key kernel (dk, dv and the bias
// sums).  Each recomputes P from the forward pass's lse.
//
// Bound by the matrix pipe, which one wave a SIMD (some 400 registers at width 128)
// does not keep fed: four causal documents of 500 to 4096 tokens, bf16, 16 heads of
// 128 over 4 key heads, capped, 700 us (640 TFLOP/s over its four products) and 847 us
// (530).  EXTRA is one form for a bias, for dropout and for both: the key kernel with it
// spills 16 to 87 registers in bf16 at width 64 (37 with a bias, four waves over keys and
// aligned rows: 61 us on six prefix sequences of 700 to 1023 tokens, 12 over 4 heads),
// and the fp32 one at width 128 up to 90, with a cap 14 and 28 of them without EXTRA too.
#pragma once

#include "attn_tile.h"

namespace fo {

struct BwdShape {
    int group;        // heads per key head
    int wq, q_tiles;  // query kernel: waves side by side over rows, row tiles
    int wk, k_tiles;  // key kernel: the same over keys
    int h_parts, q_parts;  // and its cuts over a key head's heads and over the queries
    bool vec, narrow;  // narrow: attn_narrow.h, tiles of 64
    float* part;  // partial dk, then dv, of the cuts: [h_parts q_parts][k_rows][kv_heads][D] each
};

// The key kernel's waves side by side, at least: with fp32 rows of 128, four
// query waves' tiles and the bias sums together would pass the LDS.
template <class T, int DP>
constexpr int min_wk() { return sizeof(T) == 4 && DP == 128 ? 2 : 1; }

// Workgroups per compute unit that the registers are held to.
template <class T, int DP>
constexpr int bwd_occ() { return sizeof(T) == 4 || DP == 128 ? 1 : 2; }

constexpr int bwd_kb(int wn) { return wn == 4 ? 64 : 32 * (4 / wn); }

// Scores S -> u log2(e) + add(r), and du/ds.
template <class T, bool CAP, class F>
__device__ __forceinline__ void to_exponent(f32x16& S, float* slope, const ScoreK& k, F add) {
    if (CAP) cap_scores<T, 16>(S, k, slope);
    const float mul = CAP ? k.cl : k.mul;
#pragma unroll
    for (int r = 0; r < 16; ++r) S[r] = fmaf(S[r], mul, add(r));
}
template <class F>
__device__ __forceinline__ void near_bias(f32x16& S, F f) {
#pragma unroll
    for (int r = 0; r < 16; ++r) S[r] += f(r);
}

// dq and delta.  bf16: delta is first taken as dO.out, whose rounding (2^-9 of
// out) would be the largest error of the gradients.  dU then misses delta's error
// e_i by -P e_i; e_i itself is the row sum of dU, which has to be zero.  So the
// kernel also sums X_i = sum_j P_ij du/ds k_j and subtracts e_i X_i: one more
// product instead of a pass for delta, which would take two and the
// exponentials again.
template <class T, int DP, int WQ, bool CAP, bool EXTRA, bool VEC>
__global__ void __launch_bounds__(256, (bwd_occ<T, DP>())) attn_dq_kernel(AttnArgs x, BwdShape f) {
    constexpr int WK = 4 / WQ, KB = bwd_kb(WQ), KT = KB / 32 / WK, NK = DP / 16, ND = DP / 32;
    constexpr bool FIX = sizeof(T) == 2;
    using TL = Tile<T, DP>;
    constexpr int TILE = KB * TL::LD, JW = (FIX ? 2 : 1) * DP * 32 + 64;
    constexpr int JOIN = WK > 1 ? (WK - 1) * WQ * JW * 4 : 0;
    constexpr int BYTES = 2 * TILE * (int)sizeof(T) > JOIN ? 2 * TILE * (int)sizeof(T) : JOIN;
    __shared__ __attribute__((aligned(16))) char smem[BYTES];
    extern __shared__ float lut[];  // with a bias: its values by distance
    T *Ks = (T*)smem, *Vs = Ks + TILE;
    const fo_attn& a = x.a;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane & 31, lh = lane >> 5;
    const int wq = w % WQ, wk = w / WQ;
    const int D = a.head_dim;
    const int h = blockIdx.x, hk = f.group > 1 ? h / f.group : h, b = blockIdx.y;
    const int i0 = (f.q_tiles - 1 - blockIdx.z) * 32 * WQ;  // longest first
    const Span s = span_of(a, b);
    if (i0 >= s.nq) return;
    const int pre = a.mask == FO_ATTN_PREFIX ? a.prefix[b] : 0, off = s.nk - s.nq;
    const int iw = i0 + 32 * wq, qi = iw + lr;
    const bool ok = qi < s.nq;
    const int lim = ok ? limit_of(a, s, pre, qi) : 0x7fffffff;
    const int wg_end = limit_of(a, s, pre, min(i0 + 32 * WQ, s.nq) - 1);
    const int wave_end = iw < s.nq ? limit_of(a, s, pre, min(iw + 32, s.nq) - 1) : 0;
    const int wave_all = iw < s.nq ? limit_of(a, s, pre, iw) : 0;
    const int tiles = (wg_end + KB - 1) / KB;

    const T* kb = (const T*)x.k + (int64_t)s.k0 * a.k_ld + hk * a.k_hs;
    const T* vb = (const T*)x.v + (int64_t)s.k0 * a.v_ld + hk * a.v_hs;
    Stage<T, DP, KB, VEC> sk, sv;
    if (tiles) {
        sk.load(kb, a.k_ld, 0, s.nk, D, tid);
        sv.load(vb, a.v_ld, 0, s.nk, D, tid);
    }
    const int64_t stat = (int64_t)h * a.q_rows + s.q0 + qi;
    Frag<T> q[NK], g[NK];
    float dl = 0.f;  // delta
    {
        const int64_t row = s.q0 + (ok ? qi : 0);
        const T* qr = (const T*)x.q + row * a.q_ld + h * a.q_hs;
        const T* gr = (const T*)x.dout + row * a.out_ld + h * a.out_hs;
        const T* orow = (const T*)x.out + row * a.out_ld + h * a.out_hs;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            q[kk] = ld_frag<VEC>(qr, 16 * kk + 8 * lh, D, ok);
            g[kk] = ld_frag<VEC>(gr, 16 * kk + 8 * lh, D, ok);
            const Frag<T> o = ld_frag<VEC>(orow, 16 * kk + 8 * lh, D, ok);
#pragma unroll
            for (int e = 0; e < 8; ++e) dl = fmaf((float)g[kk].v[e], (float)o.v[e], dl);
            if (!CAP && a.scale < 0.f) negate(q[kk]);
        }
        dl += __shfl_xor(dl, 32);
    }
    float lse = ok ? x.lse[stat] : INFINITY;
    if (lse == -INFINITY) lse = INFINITY;  // a row that sees nothing: every P is exp2(-inf) = 0
    const ScoreK sc = score_k(a);
    const bool bias = EXTRA && a.table != nullptr;
    float far_lo = 0.f, far_hi = 0.f;
    if (bias) {
        far_lo = bias_at<T>(a, h, -a.radius);
        far_hi = bias_at<T>(a, h, a.radius);
        fill_lut<T>(lut, a, h, tid);
    }
    f32x16 dQ[ND], X[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dQ[d][r] = X[d][r] = 0.f;
    float err = 0.f;  // this lane's part of the row sum of dU
    f32x16 g0;        // dP - delta starts from -delta, unless dropout comes between the two
#pragma unroll
    for (int r = 0; r < 16; ++r) g0[r] = EXTRA && x.thr ? 0.f : -dl;

    for (int t = 0; t < tiles; ++t) {
        __syncthreads();
        sk.store(Ks, tid, D);
        sv.store(Vs, tid, D);
        __syncthreads();
        if (t + 1 < tiles) {
            sk.load(kb, a.k_ld, (t + 1) * KB, s.nk, D, tid);
            sv.load(vb, a.v_ld, (t + 1) * KB, s.nk, D, tid);
        }
#pragma unroll
        for (int c = 0; c < KT; ++c) {
            const int kw = 32 * (KT * wk + c), j0 = t * KB + kw;
            if (j0 >= wave_end) continue;
            f32x16 S, G = g0;
#pragma unroll
            for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                S = mma(TL::frag_row(Ks, kw, 16 * kk, lane), q[kk], S);
                G = mma(TL::frag_row(Vs, kw, 16 * kk, lane), g[kk], G);
            }
            float slope[16];
            const int n_lo = j0 - (iw + 31) - off, n_hi = j0 + 31 - iw - off;
            const bool near = EXTRA && bias && n_lo < a.radius && n_hi > -a.radius;
            const float add0 = !bias || near ? 0.f : n_lo >= a.radius ? far_hi : far_lo;
            const float add = add0 - lse;
            to_exponent<T, CAP>(S, slope, sc, [&](int) { return add; });
            if (near) {
                const float* at = &lut[j0 + 4 * lh - qi - off + a.radius + kReach];
                near_bias(S, [&](int r) { return at[8 * (r >> 2) + (r & 3)]; });
            }
            if (j0 + 32 > wave_all) {
                const int left = lim - j0 - 4 * lh;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (8 * (r >> 2) + (r & 3) >= left) S[r] = -INFINITY;
            }
            if (EXTRA && x.thr) {
                const uint32_t bits = keep_bits(x.thr, j0, lh, qi, b * a.heads + h, a);
#pragma unroll
                for (int r = 0; r < 16; ++r) G[r] = ((bits >> r) & 1 ? G[r] * x.keep_scale : 0.f) - dl;
            }
            float ds[16], ps[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(S[r]), du = p * G[r];
                err += du;
                ds[r] = CAP ? du * slope[r] : du;
                ps[r] = CAP ? p * slope[r] : p;
            }
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2) {
                const Frag<T> df = pack8<T>(ds + 8 * k2), pf = pack8<T>(ps + 8 * k2);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const Frag<T> kf = TL::frag_col(Ks, kw + 16 * k2, 32 * d, lane);
                    dQ[d] = mma(kf, df, dQ[d]);
                    if (FIX) X[d] = mma(kf, pf, X[d]);
                }
            }
        }
    }
    err += __shfl_xor(err, 32);
    if (WK > 1) {
        float* J = (float*)smem;
        __syncthreads();
        if (wk > 0) {
            float* mine = J + ((wk - 1) * WQ + wq) * JW;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    mine[(d * 16 + r) * 64 + lane] = dQ[d][r];
                    if (FIX) mine[32 * DP + (d * 16 + r) * 64 + lane] = X[d][r];
                }
            mine[JW - 64 + lane] = err;
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int k = 0; k < WK - 1; ++k) {
            const float* its = J + (k * WQ + wq) * JW;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    dQ[d][r] += its[(d * 16 + r) * 64 + lane];
                    if (FIX) X[d][r] += its[32 * DP + (d * 16 + r) * 64 + lane];
                }
            err += its[JW - 64 + lane];
        }
    }
    if (!ok) return;
    if (FIX) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) dQ[d][r] = fmaf(-err, X[d][r], dQ[d][r]);
        dl += err;
    }
    store_row<T, DP>((T*)x.dq + (int64_t)(s.q0 + qi) * a.q_ld + h * a.q_hs, dQ, a.scale, lh, D, VEC);
    if (lh == 0) x.delta[stat] = dl;
}

// Adds a 32x32 tile of dU (lane: key l % 32, register r: query 8 (r / 4) + 4 (l /
// 32) + r % 4) to sums by distance: lane L takes the entries whose key - query is L
// or L - 32 from the lanes that hold them.  line[0] is the distance of key 0
// and query 0 of the tile.
__device__ __forceinline__ void add_diagonals(const f32x16& du, float* line, int lr, int lh) {
    float pos = 0.f, neg = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int q = 8 * (r >> 2) + (r & 3) + 4 * lh, src = ((lr + q) & 31) + 32 * lh;
        const float mine = du[r];  // (a bit cast of the element itself reads element 0)
        const float v = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(4 * src, __builtin_bit_cast(int, mine)));
        const bool wrap = lr + q >= 32;
        pos += wrap ? 0.f : v;
        neg += wrap ? v : 0.f;
    }
    pos += __shfl_xor(pos, 32);
    neg += __shfl_xor(neg, 32);
    wave_sync();  // the next tile's 64 distances overlap these by 32, in other lanes
    line[lr - 32 * lh] += lh ? neg : pos;  // 64 lanes, 64 distances
    wave_sync();
}

// dk, dv and the bias gradient by distance.  WN waves take 32 keys each, 4 / WN
// different queries of a tile.  Scores come as S = Q K^T here, keys on the lanes.
// Where there are few key tiles the work of one is cut over the heads that share
// it and over the queries, and join_keys adds the cuts.
template <class T, int DP, int WN, bool CAP, bool EXTRA, bool VEC>
__global__ void __launch_bounds__(256, (bwd_occ<T, DP>())) attn_dkv_kernel(AttnArgs x, BwdShape f) {
    constexpr int WK = 4 / WN, QB = bwd_kb(WN), QT = QB / 32 / WK, NK = DP / 16, ND = DP / 32;
    using TL = Tile<T, DP>;
    constexpr int TILE = QB * TL::LD, JW = 2 * DP * 32;
    constexpr int JOIN = WK > 1 ? (WK - 1) * WN * JW * 4 : 0;
    constexpr int BYTES = 2 * TILE * (int)sizeof(T) > JOIN ? 2 * TILE * (int)sizeof(T) : JOIN;
    __shared__ __attribute__((aligned(16))) char smem[BYTES];
    extern __shared__ float dyn[];  // with a bias: its values by distance, and each wave's sums
    __shared__ __attribute__((aligned(16))) float sl[QB], sd[QB];
    __shared__ __attribute__((aligned(16))) uint16_t drops[4][64];
    T *Qs = (T*)smem, *Gs = Qs + TILE;
    const fo_attn& a = x.a;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane & 31, lh = lane >> 5;
    const int wn = w % WN, wk = w / WN;
    const int D = a.head_dim, G = f.group, R = a.radius;
    const int hk = blockIdx.x, b = blockIdx.y, parts = f.h_parts * f.q_parts;
    int kt = blockIdx.z, part = 0, qp = 0, h0 = 0, h1 = G;  // h0, h1: the workgroup's heads of the group
    if (parts > 1) {
        part = kt % parts;
        kt /= parts;
        qp = part / f.h_parts;
        const int hb = (G + f.h_parts - 1) / f.h_parts;
        h0 = min(part % f.h_parts * hb, G);
        h1 = min(h0 + hb, G);
    }
    const int j0 = kt * 32 * WN;
    float* hist = EXTRA && a.table
                      ? x.hist + ((((int64_t)qp * f.k_tiles + kt) * a.batch + b) * a.heads + hk * G) * (2 * R + 1)
                      : nullptr;
    const Span s = span_of(a, b);
    if (j0 >= s.nk) {  // no such keys: their sums are zero
        if (hist)
            each(tid, 256, (h1 - h0) * (2 * R + 1), [&](int e) { hist[h0 * (2 * R + 1) + e] = 0.f; });
        return;
    }
    const int pre = a.mask == FO_ATTN_PREFIX ? a.prefix[b] : 0, off = s.nk - s.nq;
    const int jw = j0 + 32 * wn, j = jw + lr;
    const bool ok = j < s.nk;
    // the first query that sees key j (limits grow with the query)
    auto first_of = [&](int key) { return a.mask == FO_ATTN_FULL || key < pre ? 0 : max(0, key - off); };
    const int first = ok ? first_of(j) : 0x7fffffff;
    const int wave_from = jw < s.nk ? first_of(jw) : 0x7fffffff;
    const int wave_all = jw + 32 <= s.nk ? first_of(jw + 31) : 0x7fffffff;  // all 32 keys are seen from here on
    int t0 = min(first_of(j0), s.nq) / QB, t1 = (s.nq + QB - 1) / QB;
    if (f.q_parts > 1) {
        const int per = (t1 - t0 + f.q_parts - 1) / f.q_parts;
        t0 = min(t0 + qp * per, t1);
        t1 = min(t0 + per, t1);
    }

    Frag<T> k[NK], v[NK];
    {
        const int64_t row = s.k0 + (ok ? j : 0);
        const T* kr = (const T*)x.k + row * a.k_ld + hk * a.k_hs;
        const T* vr = (const T*)x.v + row * a.v_ld + hk * a.v_hs;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            k[kk] = ld_frag<VEC>(kr, 16 * kk + 8 * lh, D, ok);
            v[kk] = ld_frag<VEC>(vr, 16 * kk + 8 * lh, D, ok);
            if (!CAP && a.scale < 0.f) negate(k[kk]);
        }
    }
    const ScoreK sc = score_k(a);
    const bool bias = EXTRA && a.table != nullptr;
    const int W = lut_floats(a);
    float *lut = dyn, *line = dyn + (1 + w) * W;
    f32x16 dK[ND], dV[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dK[d][r] = dV[d][r] = 0.f;

    for (int hg = h0; hg < h1; ++hg) {
        const int h = hk * G + hg;
        const T* qb = (const T*)x.q + (int64_t)s.q0 * a.q_ld + h * a.q_hs;
        const T* gb = (const T*)x.dout + (int64_t)s.q0 * a.out_ld + h * a.out_hs;
        const int64_t stat = (int64_t)h * a.q_rows + s.q0;
        float far_lo = 0.f, far_hi = 0.f, sum_lo = 0.f, sum_hi = 0.f;
        __syncthreads();  // the previous head's bias and sums have been read
        if (bias) {
            far_lo = bias_at<T>(a, h, -R);
            far_hi = bias_at<T>(a, h, R);
            fill_lut<T>(lut, a, h, tid);
            each(lane, 64, W, [&](int n) { line[n] = 0.f; });
        }
        Stage<T, DP, QB, VEC> sq, sg;
        float pl = 0.f, pd = 0.f;
        auto load = [&](int t) {
            sq.load(qb, a.q_ld, t * QB, s.nq, D, tid);
            sg.load(gb, a.out_ld, t * QB, s.nq, D, tid);
            if (tid < QB) {
                const int i = t * QB + tid;
                pl = i < s.nq ? -x.lse[stat + i] : -INFINITY;  // no such row: P = exp2(-inf) = 0
                pd = i < s.nq ? -x.delta[stat + i] : 0.f;
                if (pl == INFINITY) pl = -INFINITY;
            }
        };
        if (t0 < t1) load(t0);
        for (int t = t0; t < t1; ++t) {
            __syncthreads();
            sq.store(Qs, tid, D);
            sg.store(Gs, tid, D);
            if (tid < QB) sl[tid] = pl, sd[tid] = pd;
            __syncthreads();
            if (t + 1 < t1) load(t + 1);
#pragma unroll
            for (int c = 0; c < QT; ++c) {
                const int qw = 32 * (QT * wk + c), it = t * QB + qw;
                if (it + 32 <= wave_from || it >= s.nq) continue;
                f32x16 S, Gd;  // sd: -delta, from where dP - delta starts, unless dropout comes between the two
#pragma unroll
                for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const f32x4 dl = *reinterpret_cast<const f32x4*>(&sd[qw + 8 * q4 + 4 * lh]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) Gd[4 * q4 + e] = EXTRA && x.thr ? 0.f : dl[e];
                }
#pragma unroll
                for (int kk = 0; kk < NK; ++kk) {
                    S = mma(TL::frag_row(Qs, qw, 16 * kk, lane), k[kk], S);
                    Gd = mma(TL::frag_row(Gs, qw, 16 * kk, lane), v[kk], Gd);
                }
                const int n0 = jw - it - off;  // distance of key 0 and query 0 of the tile
                const bool near = EXTRA && bias && n0 - 31 < R && n0 + 31 > -R, high = n0 - 31 >= R;
                const float add0 = !bias || near ? 0.f : high ? far_hi : far_lo;
                float slope[16];
                f32x4 ls[4];  // sl: -lse
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) ls[q4] = *reinterpret_cast<const f32x4*>(&sl[qw + 8 * q4 + 4 * lh]);
                to_exponent<T, CAP>(S, slope, sc, [&](int r) { return EXTRA ? ls[r >> 2][r & 3] + add0 : ls[r >> 2][r & 3]; });
                if (near) {
                    const float* at = &lut[n0 + lr - 4 * lh + R + kReach];
                    near_bias(S, [&](int r) { return at[-8 * (r >> 2) - (r & 3)]; });
                }
                if (it < wave_all) {
                    const int from = first - it - 4 * lh;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r >> 2) + (r & 3) < from) S[r] = -INFINITY;
                }
                float ps[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) ps[r] = S[r] = __builtin_amdgcn_exp2f(S[r]);
                if (EXTRA && x.thr) {
                    // drawn with the queries on the lanes, as in the other passes, and turned through LDS
                    drops[w][32 * lh + lr] = (uint16_t)keep_bits(x.thr, jw, lh, it + lr, b * a.heads + h, a);
                    wave_sync();
                    const int kr = ((lr >> 3) << 2) | (lr & 3);  // the key's bit in a query's word
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        uint2 words;
                        __builtin_memcpy(&words, __builtin_assume_aligned(&drops[w][32 * ((lr >> 2) & 1) + 8 * q4 + 4 * lh], 8), 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool kept = ((e < 2 ? words.x : words.y) >> (kr + 16 * (e & 1))) & 1;
                            Gd[4 * q4 + e] = (kept ? Gd[4 * q4 + e] * x.keep_scale : 0.f) + sd[qw + 8 * q4 + 4 * lh + e];
                            ps[4 * q4 + e] = kept ? ps[4 * q4 + e] : 0.f;
                        }
                    }
                    wave_sync();  // read before the next tile's words are written
                }
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) {
                    const Frag<T> pf = pack8<T>(ps + 8 * k2);
#pragma unroll
                    for (int d = 0; d < ND; ++d) dV[d] = mma(TL::frag_col(Gs, qw + 16 * k2, 32 * d, lane), pf, dV[d]);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) S[r] *= Gd[r];  // dU
                if (EXTRA && bias) {
                    if (near) {
                        add_diagonals(S, &line[n0 + R + kReach], lr, lh);
                    } else {
                        float sum = 0.f;
#pragma unroll
                        for (int r = 0; r < 16; ++r) sum += S[r];
                        if (high) sum_hi += sum;
                        else sum_lo += sum;
                    }
                }
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) {
                    float ds[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) ds[e] = CAP ? S[8 * k2 + e] * slope[8 * k2 + e] : S[8 * k2 + e];
                    const Frag<T> df = pack8<T>(ds);
#pragma unroll
                    for (int d = 0; d < ND; ++d) dK[d] = mma(TL::frag_col(Qs, qw + 16 * k2, 32 * d, lane), df, dK[d]);
                }
            }
        }
        if (bias) {  // this head's sums: the waves' in order, distances past the radius at its ends
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                sum_lo += __shfl_xor(sum_lo, o);
                sum_hi += __shfl_xor(sum_hi, o);
            }
            if (lane == 0) {
                line[0] += sum_lo;
                line[W - 1] += sum_hi;
            }
            __syncthreads();
            float* out = hist + hg * (2 * R + 1);
            auto all = [&](int e) { return dyn[W + e] + dyn[2 * W + e] + dyn[3 * W + e] + dyn[4 * W + e]; };
            if (w < (R ? 2 : 1)) {  // a wave for each end; without a radius all distances are one
                float sum = 0.f;
                each(lane, 64, R ? kReach + 1 : W, [&](int e) { sum += all(w ? W - 1 - e : e); });
#pragma unroll
                for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
                if (lane == 0) out[w * 2 * R] = sum;
            }
            each(tid, 256, 2 * R - 1, [&](int n) { out[1 + n] = all(1 + n + kReach); });
        }
    }
    if (WK > 1) {
        float* J = (float*)smem;
        __syncthreads();
        if (wk > 0) {
            float* mine = J + ((wk - 1) * WN + wn) * JW;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    mine[(d * 16 + r) * 64 + lane] = dK[d][r];
                    mine[32 * DP + (d * 16 + r) * 64 + lane] = dV[d][r];
                }
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int y = 0; y < WK - 1; ++y) {
            const float* its = J + (y * WN + wn) * JW;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    dK[d][r] += its[(d * 16 + r) * 64 + lane];
                    dV[d][r] += its[32 * DP + (d * 16 + r) * 64 + lane];
                }
        }
    }
    if (!ok) return;
    if (parts > 1) {
        const int64_t at = (((int64_t)part * a.k_rows + s.k0 + j) * a.kv_heads + hk) * D;
        const int64_t all = (int64_t)parts * a.k_rows * a.kv_heads * D;
        store_row<float, DP>(f.part + at, dK, 1.f, lh, D, (D & 3) == 0);
        store_row<float, DP>(f.part + all + at, dV, 1.f, lh, D, (D & 3) == 0);
        return;
    }
    store_row<T, DP>((T*)x.dk + (int64_t)(s.k0 + j) * a.k_ld + hk * a.k_hs, dK, a.scale, lh, D, VEC);
    store_row<T, DP>((T*)x.dv + (int64_t)(s.k0 + j) * a.v_ld + hk * a.v_hs, dV, x.keep_scale, lh, D, VEC);
}

template <class T, int DP>
fo_status attn_bwd_launch(const AttnArgs& x, const BwdShape& f, hipStream_t s) {
    const fo_attn& a = x.a;
    const bool cap = a.cap > 0.f, extra = a.table || x.thr;  // EXTRA: a bias or dropout
    const unsigned lds = a.table ? 4 * lut_floats(a) : 0;
    if (f.q_tiles) {
        const dim3 n(a.heads, a.batch, f.q_tiles);
#define FO_DQ(W, CAP, EXTRA, VEC) attn_dq_kernel<T, DP, W, CAP, EXTRA, VEC><<<n, 256, lds, s>>>(x, f)
#define FO_DQ_W(CAP, EXTRA)                                    \
    {                                                          \
        if (!f.vec) FO_DQ(4, CAP, EXTRA, false);               \
        else if (f.wq == 1) FO_DQ(1, CAP, EXTRA, true);        \
        else if (f.wq == 2) FO_DQ(2, CAP, EXTRA, true);        \
        else FO_DQ(4, CAP, EXTRA, true);                       \
    }
        if (extra) {
            if (cap) FO_DQ_W(true, true) else FO_DQ_W(false, true)
        } else {
            if (cap) FO_DQ_W(true, false) else FO_DQ_W(false, false)
        }
#undef FO_DQ_W
#undef FO_DQ
        FO_LAUNCHED();
    }
    if (f.k_tiles) {
        const dim3 n(a.kv_heads, a.batch, f.k_tiles * f.h_parts * f.q_parts);
#define FO_DKV(W, CAP, EXTRA, VEC) attn_dkv_kernel<T, DP, W, CAP, EXTRA, VEC><<<n, 256, 5 * lds, s>>>(x, f)
#define FO_DKV_W(CAP, EXTRA)                                                  \
    {                                                                         \
        if (!f.vec) FO_DKV(4, CAP, EXTRA, false);                             \
        else if (f.wk == 4) FO_DKV(4, CAP, EXTRA, true);                      \
        else if (f.wk == 2) FO_DKV(2, CAP, EXTRA, true);                      \
        else if constexpr (min_wk<T, DP>() == 1) FO_DKV(1, CAP, EXTRA, true); \
    }
        if (extra) {
            if (cap) FO_DKV_W(true, true) else FO_DKV_W(false, true)
        } else {
            if (cap) FO_DKV_W(true, false) else FO_DKV_W(false, false)
        }
#undef FO_DKV_W
#undef FO_DKV
        FO_LAUNCHED();
    }
    return FO_OK;
}

}  // namespace fo
