// Backward of the attention operator for sequences of up to LM = 64 or 128 queries
// and keys whose heads share no keys: one workgroup per sequence and head holds
// everything, so the scores are computed once, delta is the row sum of P dP itself, and one launch
// gives dq, dk, dv and the bias sums.
//
// Query phase: a wave has 32 queries on its lanes and all their keys in registers
// (P, dP), then dS and dq.  Key phase: P and dS go to LDS where K and V were, and a
// wave sums them over the queries for 32 keys.
//
// The BERT-shaped block, 32 x 12 heads, bias and dropout: 25 us for one round of
// workgroups; the query and the key kernel took 15 and 22, and a launch more.  A wave's
// 80 matrix instructions are about 2 us of that; the rest (loads, the bias' two dependent
// loads, generator, diagonal sums, two passes through LDS, five barriers) has not been
// timed apart.
#pragma once

#include "attn_bwd.h"

namespace fo {

template <class T, int DP, int LM>
struct SmallLds {
    static constexpr int TILE = LM * Tile<T, DP>::LD, PTILE = LM * Tile<T, LM>::LD;
    static constexpr int A = 2 * TILE > PTILE ? 2 * TILE : PTILE;  // K and V, then P, then dS
    static constexpr int ALL = A + 2 * TILE;                       // and Q and dO
};

// add_diagonals for a tile with queries on the lanes and keys in the registers.
__device__ __forceinline__ void add_diagonals_t(const f32x16& du, float* line, int lr, int lh) {
    float pos = 0.f, neg = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int k = 8 * (r >> 2) + (r & 3) + 4 * lh, src = ((k - lr) & 31) + 32 * lh;
        const float mine = du[r];
        const float v = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(4 * src, __builtin_bit_cast(int, mine)));
        const bool wrap = lr > k;
        pos += wrap ? 0.f : v;
        neg += wrap ? v : 0.f;
    }
    pos += __shfl_xor(pos, 32);
    neg += __shfl_xor(neg, 32);
    wave_sync();  // as in add_diagonals
    line[lr - 32 * lh] += lh ? neg : pos;
    wave_sync();
}

// A 16-entry half (registers 8 k2 ..) of a lane's row of a [rows][LM] tile: two runs of four columns.
template <class T, int LM>
__device__ __forceinline__ void put_half(T* t, int row, int col, const Frag<T>& f) {
    char* at = (char*)&f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        T* to = &t[Tile<T, LM>::idx(row, col + 8 * u)];
        if constexpr (sizeof(T) == 2) __builtin_memcpy(to, at + 8 * u, 8);
        else __builtin_memcpy(to, at + 16 * u, 16);
    }
}

template <class T, int DP, int LM, bool CAP, bool EXTRA>
__global__ void __launch_bounds__(2 * LM, sizeof(T) == 4 || DP == 128 || CAP ? 1 : 2)
small_bwd_kernel(AttnArgs x) {
    constexpr int NT = 2 * LM, NJ = LM / 32, NW = LM / 32, NK = DP / 16, ND = DP / 32;
    using L = SmallLds<T, DP, LM>;
    using TL = Tile<T, DP>;
    using TP = Tile<T, LM>;
    __shared__ __attribute__((aligned(16))) T smem[L::ALL];
    extern __shared__ float dyn[];  // with a bias: its values by distance, and each wave's sums
    T *Ks = smem, *Vs = smem + L::TILE, *Ps = smem, *Qs = smem + L::A, *Gs = Qs + L::TILE;
    const fo_attn& a = x.a;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane & 31, lh = lane >> 5;
    const int D = a.head_dim, R = a.radius, h = blockIdx.x, b = blockIdx.y;
    const Span s = span_of(a, b);
    float* hist = EXTRA && a.table ? x.hist + ((int64_t)b * a.heads + h) * (2 * R + 1) : nullptr;
    if (s.nq == 0 || s.nk == 0) {  // nothing meets: zero gradients for the rows there are
        if (hist) each(tid, NT, 2 * R + 1, [&](int e) { hist[e] = 0.f; });
        each(tid, NT, s.nq * D, [&](int e) {
            ((T*)x.dq)[(int64_t)(s.q0 + e / D) * a.q_ld + h * a.q_hs + e % D] = T(0);
        });
        each(tid, NT, s.nk * D, [&](int e) {
            const int64_t r = s.k0 + e / D;
            ((T*)x.dk)[r * a.k_ld + h * a.k_hs + e % D] = T(0);
            ((T*)x.dv)[r * a.v_ld + h * a.v_hs + e % D] = T(0);
        });
        return;
    }
    const int pre = a.mask == FO_ATTN_PREFIX ? a.prefix[b] : 0, off = s.nk - s.nq;
    const int iw = 32 * w, qi = iw + lr;
    const bool ok = qi < s.nq;
    const int lim = ok ? limit_of(a, s, pre, qi) : 0x7fffffff;
    const int wave_end = iw < s.nq ? limit_of(a, s, pre, min(iw + 32, s.nq) - 1) : 0;
    const int wave_all = iw < s.nq ? limit_of(a, s, pre, iw) : 0;
    const ScoreK sc = score_k(a);
    const bool bias = EXTRA && a.table != nullptr;
    const int W = lut_floats(a);
    float *lut = dyn, *line = dyn + (1 + w) * W;
    const int64_t stat = (int64_t)h * a.q_rows + s.q0 + qi;
    {
        Stage<T, DP, LM, true, NT> sk, sv, sq, sg;
        sk.load((const T*)x.k + (int64_t)s.k0 * a.k_ld + h * a.k_hs, a.k_ld, 0, s.nk, D, tid);
        sv.load((const T*)x.v + (int64_t)s.k0 * a.v_ld + h * a.v_hs, a.v_ld, 0, s.nk, D, tid);
        sq.load((const T*)x.q + (int64_t)s.q0 * a.q_ld + h * a.q_hs, a.q_ld, 0, s.nq, D, tid);
        sg.load((const T*)x.dout + (int64_t)s.q0 * a.out_ld + h * a.out_hs, a.out_ld, 0, s.nq, D, tid);
        sq.clear_past(D, tid);
        sg.clear_past(D, tid);
        sk.store(Ks, tid, D);
        sv.store(Vs, tid, D);
        sq.store(Qs, tid, D);
        sg.store(Gs, tid, D);
    }
    float lse = ok ? x.lse[stat] : INFINITY, far_lo = 0.f, far_hi = 0.f, sum_lo = 0.f, sum_hi = 0.f;
    if (lse == -INFINITY) lse = INFINITY;
    if (bias) {
        far_lo = bias_at<T>(a, h, -R);
        far_hi = bias_at<T>(a, h, R);
        fill_lut<T>(lut, a, h, tid, NT);
        each(lane, 64, W, [&](int n) { line[n] = 0.f; });
    }
    __syncthreads();

    f32x16 S[NJ], Gd[NJ];
    Frag<T> pf[NJ][2], df[NJ][2];
    float slope[NJ][16], dl = 0.f;
#pragma unroll
    for (int c = 0; c < NJ; ++c) {
        const int j0 = 32 * c;
#pragma unroll
        for (int r = 0; r < 16; ++r) S[c][r] = Gd[c][r] = 0.f;
        if (j0 < wave_end) {
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                Frag<T> q = TL::frag_row(Qs, iw, 16 * kk, lane);
                if (!CAP && a.scale < 0.f) negate(q);
                S[c] = mma(TL::frag_row(Ks, j0, 16 * kk, lane), q, S[c]);
                Gd[c] = mma(TL::frag_row(Vs, j0, 16 * kk, lane), TL::frag_row(Gs, iw, 16 * kk, lane), Gd[c]);
            }
            const int n_lo = j0 - (iw + 31) - off, n_hi = j0 + 31 - iw - off;
            const bool near = EXTRA && bias && n_lo < R && n_hi > -R;
            const float add0 = !bias || near ? 0.f : n_lo >= R ? far_hi : far_lo;
            const float add = add0 - lse;
            to_exponent<T, CAP>(S[c], slope[c], sc, [&](int) { return add; });
            if (near) {
                const float* at = &lut[j0 + 4 * lh - qi - off + R + kReach];
                near_bias(S[c], [&](int r) { return at[8 * (r >> 2) + (r & 3)]; });
            }
            if (j0 + 32 > wave_all) {
                const int left = lim - j0 - 4 * lh;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (8 * (r >> 2) + (r & 3) >= left) S[c][r] = -INFINITY;
            }
            float ps[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) ps[r] = S[c][r] = __builtin_amdgcn_exp2f(S[c][r]);
            if (EXTRA && x.thr) {
                const uint32_t bits = keep_bits(x.thr, j0, lh, qi, b * a.heads + h, a);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool kept = (bits >> r) & 1;
                    Gd[c][r] = kept ? Gd[c][r] * x.keep_scale : 0.f;
                    ps[r] = kept ? ps[r] : 0.f;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) dl = fmaf(S[c][r], Gd[c][r], dl);
            pf[c][0] = pack8<T>(ps);
            pf[c][1] = pack8<T>(ps + 8);
        } else {
            const float none[8] = {};
            pf[c][0] = pf[c][1] = df[c][0] = df[c][1] = pack8<T>(none);
        }
    }
    dl += __shfl_xor(dl, 32);  // delta
    f32x16 dQ[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) dQ[d][r] = 0.f;
#pragma unroll
    for (int c = 0; c < NJ; ++c) {
        const int j0 = 32 * c;
        if (j0 >= wave_end) continue;
#pragma unroll
        for (int r = 0; r < 16; ++r) S[c][r] *= Gd[c][r] - dl;  // dU
        if (EXTRA && bias) {
            const int n0 = j0 - iw - off;  // distance of key 0 and query 0 of the tile
            if (n0 - 31 < R && n0 + 31 > -R) {
                add_diagonals_t(S[c], &line[n0 + R + kReach], lr, lh);
            } else {
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += S[c][r];
                if (n0 - 31 >= R) sum_hi += sum;
                else sum_lo += sum;
            }
        }
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
            float ds[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) ds[e] = CAP ? S[c][8 * k2 + e] * slope[c][8 * k2 + e] : S[c][8 * k2 + e];
            df[c][k2] = pack8<T>(ds);
#pragma unroll
            for (int d = 0; d < ND; ++d)
                dQ[d] = mma(TL::frag_col(Ks, j0 + 16 * k2, 32 * d, lane), df[c][k2], dQ[d]);
        }
    }
    if (ok) store_row<T, DP>((T*)x.dq + (int64_t)(s.q0 + qi) * a.q_ld + h * a.q_hs, dQ, a.scale, lh, D, true);
    if (bias) {
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            sum_lo += __shfl_xor(sum_lo, o);
            sum_hi += __shfl_xor(sum_hi, o);
        }
        if (lane == 0) {
            line[0] += sum_lo;
            line[W - 1] += sum_hi;
        }
    }
    const int nb = (s.nq + 31) / 32 * 2;  // 16-query blocks of the waves that have queries
    const int j = 32 * w + lr;
    auto turn = [&](Frag<T> (&f)[NJ][2], const T* rows, T* out, float scale) {  // out = scale f^T rows, by keys
        __syncthreads();
        if (iw < s.nq) {
#pragma unroll
            for (int c = 0; c < NJ; ++c)
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) put_half<T, LM>(Ps, qi, 32 * c + 16 * k2 + 4 * lh, f[c][k2]);
        }
        __syncthreads();
        if (32 * w >= s.nk) return;
        f32x16 acc[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
#pragma unroll 1
        for (int kk = 0; kk < nb; ++kk) {
            const Frag<T> p = TP::template frag_col<true>(Ps, 16 * kk, 32 * w, lane);
#pragma unroll
            for (int d = 0; d < ND; ++d)
                acc[d] = mma(TL::template frag_col<true>(rows, 16 * kk, 32 * d, lane), p, acc[d]);
        }
        if (j < s.nk) store_row<T, DP>(out, acc, scale, lh, D, true);
    };
    turn(pf, Gs, (T*)x.dv + (int64_t)(s.k0 + j) * a.v_ld + h * a.v_hs, x.keep_scale);
    turn(df, Qs, (T*)x.dk + (int64_t)(s.k0 + j) * a.k_ld + h * a.k_hs, a.scale);
    if (bias) {  // (the waves' sums are complete since the first barrier of turn)
        float* out = hist;
        auto all = [&](int e) {
            float sum = 0.f;
#pragma unroll
            for (int y = 1; y <= NW; ++y) sum += dyn[y * W + e];
            return sum;
        };
        if (w < (R ? 2 : 1)) {
            float sum = 0.f;
            each(lane, 64, R ? kReach + 1 : W, [&](int e) { sum += all(w ? W - 1 - e : e); });
#pragma unroll
            for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
            if (lane == 0) out[w * 2 * R] = sum;
        }
        each(tid, NT, 2 * R - 1, [&](int n) { out[1 + n] = all(1 + n + kReach); });
    }
}

// (defined for every type and width in a file of its own)
template <class T, int DP>
fo_status small_bwd_launch(const AttnArgs& x, hipStream_t s) {
    const fo_attn& a = x.a;
    const dim3 n(a.heads, a.batch);
    const bool cap = a.cap > 0.f, extra = a.table || x.thr, half = a.max_q <= 64 && a.max_k <= 64;
    const unsigned lds = a.table ? 4 * lut_floats(a) * (half ? 3 : 5) : 0;
#define FO_SMALL(CAP, EXTRA)                                                            \
    {                                                                                   \
        if (half) small_bwd_kernel<T, DP, 64, CAP, EXTRA><<<n, 128, lds, s>>>(x);       \
        else small_bwd_kernel<T, DP, 128, CAP, EXTRA><<<n, 256, lds, s>>>(x);           \
    }
    if (extra) {
        if (cap) FO_SMALL(true, true) else FO_SMALL(false, true)
    } else {
        if (cap) FO_SMALL(true, false) else FO_SMALL(false, false)
    }
#undef FO_SMALL
    FO_LAUNCHED();
    return FO_OK;
}

// Whether the kernel holds the call: its tiles and the bias sums have to fit the LDS.
template <class T, int DP>
bool small_fits(const fo_attn& a) {
    const bool half = a.max_q <= 64 && a.max_k <= 64;
    const int64_t tiles = sizeof(T) * (half ? SmallLds<T, DP, 64>::ALL : SmallLds<T, DP, 128>::ALL);
    return tiles + (a.table ? 4 * lut_floats(a) * (half ? 3 : 5) : 0) <= 160 * 1024;
}

}  // namespace fo
