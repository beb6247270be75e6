// Forward kernel of the attention operator, instantiated per type and width.
#pragma once

#include "attn_tile.h"

namespace fo {

// A launch's shape.  rows: query rows of one workgroup (32 WQ); pack: the rows
// of a workgroup are the heads of one key head's group, for one token.
struct FwdShape {
    int wq, pack, row_tiles, splits, group;  // group: heads per key head
    bool vec, narrow;  // narrow: attn_narrow.h, row tiles of 64
    float *part, *ml;  // partial results of the key slices: [split][heads][q_rows][D], [..][2]
};

constexpr int fwd_kt(int wq) { return wq == 4 ? 2 : 1; }
constexpr int fwd_kb(int wq) { return 32 * fwd_kt(wq) * (4 / wq); }

// out = softmax(u) V with running maximum m and sum l.  Four waves: WQ of them
// take 32 rows each, 4 / WQ take different keys of a tile and join at the end.
// K and V tiles pass through registers into LDS, the next tile's loads in flight
// during the products.  EXTRA: a bias or dropout.  VEC: see ld_chunk.
//
// Long sequences are bound by the matrix pipe beside the exponentials: 15.5k tokens in
// two causal documents, bf16, 32 heads of 128 over 8 key heads, 1.11 to 1.18 ms from card
// to card, 840 to 890 TFLOP/s (a large library product: 1140 to 1160).  With a cap, four
// such documents of 14.7k tokens and 16 heads run at 630 to 660: the cap's vector work is not
// hidden behind the products.  At width 128 the 128-row forms spill 2 to 27 registers (4
// in the plain and the capped one with aligned rows).  One token against a long cache is bound
// by HBM: sixteen of 6k to 16k keys, 775 MB in 163 us, 4.8 TB/s.
template <class T, int DP, int WQ, bool CAP, bool EXTRA, bool VEC>
__global__ void __launch_bounds__(256, sizeof(T) == 4 && DP > 32 ? 1 : 2)
attn_fwd_kernel(AttnArgs x, FwdShape f) {
    constexpr int WK = 4 / WQ, KT = fwd_kt(WQ), KB = fwd_kb(WQ), NK = DP / 16, ND = DP / 32;
    using TL = Tile<T, DP>;
    constexpr int TILE = KB * TL::LD;
    constexpr int JOIN = WK > 1 ? (WK - 1) * WQ * 32 * (DP + 2) : 0;  // floats
    // a second buffer saves one of two barriers a tile, where two workgroups still fit
    constexpr int BUF = WQ > 1 && 4 * TILE * (int)sizeof(T) <= 65536 ? 2 : 1;
    constexpr int BYTES = 2 * BUF * TILE * (int)sizeof(T) > JOIN * 4 ? 2 * BUF * TILE * (int)sizeof(T) : JOIN * 4;
    __shared__ __attribute__((aligned(16))) char smem[BYTES];
    extern __shared__ float lut[];  // with a bias: its values by distance
    const fo_attn& a = x.a;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane & 31, lh = lane >> 5;
    const int wq = w % WQ, wk = w / WQ;
    const int D = a.head_dim, G = f.group;

    // workgroup: x: head (or key head and part of its group) and key slice, y: sequence,
    // z: row tile, longest first.  (A grid of three dimensions and branches round the
    // rest: an integer division is some 40 instructions ahead of the first load.)
    int u = blockIdx.x, split = 0;
    if (f.splits > 1) {
        split = u % f.splits;
        u /= f.splits;
    }
    const int b = blockIdx.y;
    int h0 = u, hk = u, rt = f.row_tiles - 1 - blockIdx.z;
    if (f.pack) {
        rt = 0;
        if (f.row_tiles > 1) {
            rt = u % f.row_tiles;
            hk = u / f.row_tiles;
        }
        h0 = hk * G + 32 * rt;
    } else if (G > 1) {
        hk = u / G;
    }
    const Span s = span_of(a, b);
    const int i0 = f.pack ? 0 : rt * 32 * WQ;
    if (i0 >= s.nq) return;
    const int pre = a.mask == FO_ATTN_PREFIX ? a.prefix[b] : 0, off = s.nk - s.nq;

    const int iw = i0 + 32 * wq;                       // the wave's first query
    const int qi = f.pack ? 0 : iw + lr, head = f.pack ? h0 + lr : h0;
    const bool ok = f.pack ? 32 * rt + lr < G : qi < s.nq;
    const int lim = ok ? limit_of(a, s, pre, qi) : 0x7fffffff;
    // keys that any row of the workgroup sees, of the wave (limits grow with the query)
    const int wg_end = limit_of(a, s, pre, f.pack ? 0 : min(i0 + 32 * WQ, s.nq) - 1);
    const int wave_end = f.pack ? wg_end : iw < s.nq ? limit_of(a, s, pre, min(iw + 32, s.nq) - 1) : 0;
    const int wave_all = f.pack ? wg_end : iw < s.nq ? limit_of(a, s, pre, iw) : 0;  // keys that all its rows see
    const int tiles = (wg_end + KB - 1) / KB, per = (tiles + f.splits - 1) / f.splits;
    const int t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);

    const T* kb = (const T*)x.k + (int64_t)s.k0 * a.k_ld + hk * a.k_hs;
    const T* vb = (const T*)x.v + (int64_t)s.k0 * a.v_ld + hk * a.v_hs;
    Stage<T, DP, KB, VEC> sk, sv;
    if (t0 < t1) {
        sk.load(kb, a.k_ld, t0 * KB, s.nk, D, tid);
        sv.load(vb, a.v_ld, t0 * KB, s.nk, D, tid);
    }
    Frag<T> q[NK];
    {
        const T* row = (const T*)x.q + (int64_t)(s.q0 + (ok ? qi : 0)) * a.q_ld + (ok ? head : h0) * a.q_hs;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            q[kk] = ld_frag<VEC>(row, 16 * kk + 8 * lh, D, ok);
            if (!CAP && a.scale < 0.f) negate(q[kk]);
        }
    }
    const ScoreK sc = score_k(a);
    const bool bias = EXTRA && a.table != nullptr;
    float far_lo = 0.f, far_hi = 0.f;  // bias beyond the radius on either side
    if (bias) {
        far_lo = bias_at<T>(a, ok ? head : h0, -a.radius);
        far_hi = bias_at<T>(a, ok ? head : h0, a.radius);
        if (!f.pack) fill_lut<T>(lut, a, h0, tid);
    }

    f32x16 O[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[d][r] = 0.f;
    float m = -INFINITY, l = 0.f;  // l: this lane's keys only

    for (int t = t0; t < t1; ++t) {
        T *Ks = (T*)smem + (BUF == 2 ? (t & 1) * 2 * TILE : 0), *Vs = Ks + TILE;
        if (BUF == 1) __syncthreads();  // the previous tile has been read
        sk.store(Ks, tid, D);
        sv.store(Vs, tid, D);
        __syncthreads();
        if (t + 1 < t1) {
            sk.load(kb, a.k_ld, (t + 1) * KB, s.nk, D, tid);
            sv.load(vb, a.v_ld, (t + 1) * KB, s.nk, D, tid);
        }
        const int kw = 32 * KT * wk, j0 = t * KB + kw;  // the wave's first key in the tile, in the sequence
        if (j0 >= wave_end) continue;
        f32x16 S[KT];
#pragma unroll
        for (int c = 0; c < KT; ++c) {
#pragma unroll
            for (int r = 0; r < 16; ++r) S[c][r] = 0.f;
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) S[c] = mma(TL::frag_row(Ks, kw + 32 * c, 16 * kk, lane), q[kk], S[c]);
        }
        // distances of the wave's rows to this tile: [n_lo, n_hi]
        const int n_lo = j0 - (f.pack ? 0 : iw + 31) - off, n_hi = j0 + 32 * KT - 1 - (f.pack ? 0 : iw) - off;
        const bool near = EXTRA && bias && n_lo < a.radius && n_hi > -a.radius;
        const float add0 = !EXTRA || !bias || near ? 0.f : n_lo >= a.radius ? far_hi : far_lo;
        float mul = sc.mul, add = add0;
        if (CAP) {
#pragma unroll
            for (int c = 0; c < KT; ++c) cap_scores<T, 16>(S[c], sc, nullptr);
            mul = sc.cl;
        }
        if (near) {  // x itself takes S's place
            const int base = j0 + 4 * lh - qi - off;
#pragma unroll
            for (int c = 0; c < KT; ++c)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = 32 * c + 8 * (r >> 2) + (r & 3);
                    const float v = f.pack ? bias_at<T>(a, ok ? head : h0, base + j) : lut[base + j + a.radius + kReach];
                    S[c][r] = fmaf(S[c][r], mul, v);
                }
            mul = 1.f;
        }
        if (j0 + 32 * KT > wave_all) {  // some row does not see the whole tile
            const int left = lim - j0 - 4 * lh;
#pragma unroll
            for (int c = 0; c < KT; ++c)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * c + 8 * (r >> 2) + (r & 3) >= left) S[c][r] = -INFINITY;
        }
        float mt = S[0][0];
#pragma unroll
        for (int c = 0; c < KT; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) mt = fmaxf(mt, S[c][r]);
        mt = fmaxf(mt, __shfl_xor(mt, 32));
        const float mn = fmaxf(m, fmaf(mt, mul, add));
        // The maximum is moved up only when some row's grew by more than 2^8: the sums
        // stay far inside fp32, and most tiles leave the accumulators alone.
        if (__any(mn > m + 8.f)) {
            asm volatile("");  // a branch, not 16 ND products every time
            const float g = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.f : mn));
            l *= g;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) O[d][r] *= g;
            m = mn;
        }
        const float sub = add - (m == -INFINITY ? 0.f : m);
#pragma unroll
        for (int c = 0; c < KT; ++c) {
            float p[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[r] = __builtin_amdgcn_exp2f(fmaf(S[c][r], mul, sub));
                l += p[r];
            }
            if (EXTRA && x.thr) {
                const uint32_t bits = keep_bits(x.thr, j0 + 32 * c, lh, qi, b * a.heads + head, a);
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] = (bits >> r) & 1 ? p[r] : 0.f;
            }
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2) {
                const Frag<T> pf = pack8<T>(p + 8 * k2);
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    O[d] = mma(TL::frag_col(Vs, kw + 32 * c + 16 * k2, 32 * d, lane), pf, O[d]);
            }
        }
    }
    l += __shfl_xor(l, 32);

    if (WK > 1) {  // the key waves' results meet in LDS
        float* J = (float*)smem;
        __syncthreads();
        if (wk > 0) {
            float* mine = J + ((wk - 1) * WQ + wq) * 32 * (DP + 2);
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(d * 16 + r) * 64 + lane] = O[d][r];
            if (lh == 0) mine[32 * DP + lr] = m, mine[32 * DP + 32 + lr] = l;
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int k = 0; k < WK - 1; ++k) {
            const float* its = J + (k * WQ + wq) * 32 * (DP + 2);
            const float m2 = its[32 * DP + lr], l2 = its[32 * DP + 32 + lr], mn = fmaxf(m, m2);
            const float m0 = mn == -INFINITY ? 0.f : mn;
            const float g1 = __builtin_amdgcn_exp2f(m - m0), g2 = __builtin_amdgcn_exp2f(m2 - m0);
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) O[d][r] = O[d][r] * g1 + its[(d * 16 + r) * 64 + lane] * g2;
            l = l * g1 + l2 * g2;
            m = mn;
        }
    }
    if (!ok) return;
    if (f.splits > 1) {  // this slice's sums, unnormalised, for the joining kernel
        const int64_t at = ((int64_t)split * a.heads + head) * a.q_rows + s.q0 + qi;
        if (l > 0.f) store_row<float, DP>(f.part + at * D, O, 1.f, lh, D, (D & 3) == 0);
        if (lh == 0) f.ml[2 * at] = m, f.ml[2 * at + 1] = l;
        return;
    }
    const float inv = l > 0.f ? x.keep_scale / l : 0.f;
    store_row<T, DP>((T*)x.out + (int64_t)(s.q0 + qi) * a.out_ld + head * a.out_hs, O, inv, lh, D, VEC);
    if (x.lse && lh == 0)
        x.lse[(int64_t)head * a.q_rows + s.q0 + qi] = l > 0.f ? m + __builtin_amdgcn_logf(l) : -INFINITY;
}

// (defined for every type and width in a file of its own)
template <class T, int DP>
fo_status attn_fwd_launch(const AttnArgs& x, const FwdShape& f, hipStream_t s) {
    const fo_attn& a = x.a;
    const dim3 n = f.pack ? dim3((unsigned)(f.row_tiles * a.kv_heads * f.splits), a.batch)
                          : dim3((unsigned)(a.heads * f.splits), a.batch, f.row_tiles);
    const bool cap = a.cap > 0.f;
    const unsigned lds = a.table && !f.pack ? 4 * lut_floats(a) : 0;
    const bool extra = a.table || x.thr;
#define FO_FWD(WQ, CAP, EXTRA, VEC) attn_fwd_kernel<T, DP, WQ, CAP, EXTRA, VEC><<<n, 256, lds, s>>>(x, f)
#define FO_FWD_W(CAP, EXTRA)                                   \
    {                                                          \
        if (!f.vec) {  /* 33 to 64 rows: one tile either way */ \
            if (f.wq == 1) FO_FWD(1, CAP, EXTRA, false);       \
            else FO_FWD(4, CAP, EXTRA, false);                 \
        } else {                                               \
            if (f.wq == 1) FO_FWD(1, CAP, EXTRA, true);        \
            else if (f.wq == 2) FO_FWD(2, CAP, EXTRA, true);   \
            else FO_FWD(4, CAP, EXTRA, true);                  \
        }                                                      \
    }
    if (extra) {
        if (cap) FO_FWD_W(true, true) else FO_FWD_W(false, true)
    } else {
        if (cap) FO_FWD_W(true, false) else FO_FWD_W(false, false)
    }
#undef FO_FWD_W
#undef FO_FWD
    FO_LAUNCHED();
    return FO_OK;
}

}  // namespace fo
