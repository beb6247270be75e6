// Matrix-core building blocks of the attention operators: 32x32 products,
// LDS tiles and their operand fragments, and what a score is made of.
//
// Transposed orientation: a wave owns 32 rows (queries, or keys in the key
// kernel) which sit on the accumulator columns, one row per lane pair (l, l +
// 32).  Accumulator register r of lane l is column-of-the-other-side
//   8 (r / 4) + 4 (l / 32) + r % 4,
// so statistics over the other side reduce within a lane plus one exchange
// between the half-waves, and 16 of a tile's 32 entries (registers 8 kb .. 8 kb
// + 7) already are the B operand of a product that sums over them, provided the
// A operand takes its k index in the same order (frag_col).
#pragma once

#include "ops.h"

namespace fo {

constexpr float kLog2e = 1.4426950408889634f;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// Orders LDS accesses of a wave's lanes that read what another lane has written (the
// hardware keeps a wave's order; the compiler only a lane's own).
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// An operand of one step of 16 k values: lane l holds row l % 32 and k = 8 (l / 32) + e, e = 0..7.
template <class T>
struct Frag;
template <>
struct Frag<bf16_t> {
    bf16x8_t v;
};
template <>
struct Frag<float> {
    float v[8];
};

// c += A B over 16 k values.  fp32 takes eight 32x32x2 products, the e-th over k = e and 8 + e.
__device__ __forceinline__ f32x16 mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
    return c;
}

// Eight accumulator values as an operand: probabilities and score gradients, which
// bf16 calls round once here so that their products run at the bf16 rate, sixteen
// times fp32's.  Each rounding is independent and below 2^-9 in the root mean square,
// as large as that of a result; sums over them stay fp32.
template <class T>
__device__ __forceinline__ Frag<T> pack8(const float* x);
template <>
__device__ __forceinline__ Frag<bf16_t> pack8<bf16_t>(const float* x) {
    const u32x4_t u = {f2bf2(x[0], x[1]), f2bf2(x[2], x[3]), f2bf2(x[4], x[5]), f2bf2(x[6], x[7])};
    return {__builtin_bit_cast(bf16x8_t, u)};
}
template <>
__device__ __forceinline__ Frag<float> pack8<float>(const float* x) {
    Frag<float> f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = x[e];
    return f;
}

// An LDS tile of rows of DP values.  bf16: 16-byte chunks XOR-swizzled by row so
// that neither the row reads (16 rows, one chunk each) nor the transpose reads
// (four consecutive rows of 64 bytes) share banks.  fp32: rows padded by one
// 16-byte chunk, which spreads the row reads; column reads are consecutive.
template <class T, int DP>
struct Tile;
template <int DP>
struct Tile<bf16_t, DP> {
    static constexpr int LD = DP, CHUNK = 8;
    static __device__ __forceinline__ int idx(int row, int col) {
        int x;
        if (DP == 128) x = ((row & 3) << 2) | ((row >> 2) & 3);
        else if (DP == 64) x = (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
        else x = (row >> 2) & 3;
        return row * DP + ((((col >> 3) ^ x) << 3) | (col & 7));
    }
    // Lane rows are tile rows row0 + l % 32, k runs along the row.
    static __device__ __forceinline__ Frag<bf16_t> frag_row(const bf16_t* t, int row0, int col0, int lane) {
        return {*reinterpret_cast<const bf16x8_t*>(&t[idx(row0 + (lane & 31), col0 + 8 * (lane >> 5))])};
    }
    // Lane rows are tile columns col0 + l % 32, k are 16 tile rows from row0, in the
    // accumulators' order or in their own (PLAIN): two transpose reads (ds_read_b64_tr_b16: within each group
    // of 16 lanes, lane i receives element i mod 4 of the 8 bytes addressed by lane
    // 4 j + i / 4, j = 0..3).
    template <bool PLAIN = false>
    static __device__ __forceinline__ Frag<bf16_t> frag_col(const bf16_t* t, int row0, int col0, int lane) {
        const int g = lane >> 4, s = lane & 15, col = col0 + 16 * (g & 1) + 4 * (s & 3);
        s16x4_t v[2];
#pragma unroll
        for (int r = 0; r < 2; ++r)
            v[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4_t*)(t + idx(row0 + (PLAIN ? 8 : 4) * (lane >> 5) + (PLAIN ? 4 : 8) * r + (s >> 2), col)));
        const s16x8_t o = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
        return {__builtin_bit_cast(bf16x8_t, o)};
    }
};
template <int DP>
struct Tile<float, DP> {
    static constexpr int LD = DP + 4, CHUNK = 4;
    static __device__ __forceinline__ int idx(int row, int col) { return row * LD + col; }
    static __device__ __forceinline__ Frag<float> frag_row(const float* t, int row0, int col0, int lane) {
        const f32x4* p = reinterpret_cast<const f32x4*>(&t[idx(row0 + (lane & 31), col0 + 8 * (lane >> 5))]);
        const f32x4 a = p[0], b = p[1];
        return {{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
    }
    template <bool PLAIN = false>
    static __device__ __forceinline__ Frag<float> frag_col(const float* t, int row0, int col0, int lane) {
        Frag<float> f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            f.v[e] = t[idx(row0 + (PLAIN ? 8 * (lane >> 5) + e : 4 * (lane >> 5) + (e & 3) + 8 * (e >> 2)),
                           col0 + (lane & 31))];
        return f;
    }
};

// 16 bytes at p, aligned as T is: one load (the hardware takes any address).
template <class T>
__device__ __forceinline__ u32x4_t ld16(const T* p) {
    u32x4_t u;
    __builtin_memcpy(&u, p, 16);
    return u;
}
// Columns d .. of a row of D, in two steps so that the load can fly: raw_any reads the
// chunk that D ends in as the row's last 16 bytes (rows shorter than that go element by
// element), whole_any shifts it down and clears what lies past D.  32 heads of 77, two
// causal sequences of 2500 rows with dropout: 1293 us a training pass, 1039 us for heads
// of 80 in aligned rows, 2065 us when 77 was read element by element.
template <class T>
__device__ __forceinline__ u32x4_t raw_any(const T* row, int d, int D) {
    constexpr int N = 16 / sizeof(T);
    if (D >= N) return ld16(row + min(d, D - N));
    T v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < D ? row[e] : T(0);
    u32x4_t u;
    __builtin_memcpy(&u, v, 16);
    return u;
}
template <class T>
__device__ __forceinline__ u32x4_t whole_any(u32x4_t u, int d, int D) {
    constexpr int N = 16 / sizeof(T);
    if (D > N && D % N) {
        unsigned __int128 w;
        __builtin_memcpy(&w, &u, 16);
        w >>= 8 * (int)sizeof(T) * (N - D % N);  // the same for every lane
        u32x4_t t;
        __builtin_memcpy(&t, &w, 16);
        u = d + N > D ? t : u;
    }
    return d < D ? u : u32x4_t{0u, 0u, 0u, 0u};
}
// 16 bytes of a row from column d on, zeros past D or where !ok.  VEC: every row starts 16-byte aligned, D is a whole
// number of chunks and a row stride is below 2^24 bytes.
template <bool VEC, class T>
__device__ __forceinline__ u32x4_t ld_chunk(const T* row, int d, int D, bool ok) {
    u32x4_t u = {0u, 0u, 0u, 0u};
    if (VEC) {
        if (ok && d < D) u = *reinterpret_cast<const u32x4_t*>(row + d);
    } else if (ok) {
        u = whole_any<T>(raw_any(row, d, D), d, D);
    }
    return u;
}
template <bool VEC, class T>
__device__ __forceinline__ Frag<T> ld_frag(const T* row, int d, int D, bool ok) {
    Frag<T> f;
#pragma unroll
    for (int c = 0; c < (int)sizeof(T) / 2; ++c) {
        const u32x4_t u = ld_chunk<VEC>(row, d + c * (16 / (int)sizeof(T)), D, ok);
        __builtin_memcpy((char*)&f.v + 16 * c, &u, 16);
    }
    return f;
}

// ROWS rows of a [rows][ld] operand through registers into an LDS tile, all
// loads of a tile issued together so that they fly while the
// previous tile is in use.  Aligned rows (VEC) are read without a branch at 32-bit
// offsets from a base that the scalar unit moves on; rows past the last one and
// columns past D repeat the last row and chunk, which no result uses: their
// probabilities are masked to zero, the other operand's columns are zero.
template <class T, int DP, int ROWS, bool VEC, int THREADS = 256>
struct Stage {
    static constexpr int CPR = DP * (int)sizeof(T) / 16, N = ROWS * CPR / THREADS, EPC = 16 / (int)sizeof(T);
    static constexpr int RS = THREADS / CPR;  // rows between a thread's chunks
    static_assert(ROWS * CPR % THREADS == 0, "whole chunks per thread");
    u32x4_t u[N];
    // Rows r0 .. of which those below n (more than r0) exist.
    __device__ __forceinline__ void load(const T* base, int64_t ld, int r0, int n, int D, int tid) {
        if constexpr (VEC) {
            const char* p = (const char*)(base + r0 * ld);
            const uint32_t step = (uint32_t)(ld * sizeof(T)), last = (uint32_t)(n - 1 - r0);
            const uint32_t col = 16 * min(tid % CPR, (D - 1) / EPC);
#pragma unroll
            for (int i = 0; i < N; ++i)
                u[i] = *reinterpret_cast<const u32x4_t*>(
                    p + (__umul24(min((uint32_t)(tid / CPR + i * RS), last), step) + col));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = min(r0 + tid / CPR + i * RS, n - 1);
                u[i] = raw_any(base + r * ld, (tid % CPR) * EPC, D);
            }
        }
    }
    // Zeros in the columns past D, for tiles that meet another tile's there.
    __device__ __forceinline__ void clear_past(int D, int tid) {
        const bool out = (tid % CPR) * EPC >= D;
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = out ? u32x4_t{0u, 0u, 0u, 0u} : u[i];
    }
    __device__ __forceinline__ void store(T* t, int tid, int D) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int x = tid + THREADS * i, d = (tid % CPR) * EPC;
            *reinterpret_cast<u32x4_t*>(&t[Tile<T, DP>::idx(x / CPR, d)]) = VEC ? u[i] : whole_any<T>(u[i], d, D);
        }
    }
};

// A row's DP accumulated values times s: register 4 q + e of accumulator t is column 32 t + 8 q + 4 (l / 32) + e.
template <class T, int DP>
__device__ __forceinline__ void store_row(T* row, const f32x16* acc, float s, int lh, int D, bool vec) {
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = 32 * t + 8 * q + 4 * lh;
            const float v[4] = {acc[t][4 * q] * s, acc[t][4 * q + 1] * s, acc[t][4 * q + 2] * s, acc[t][4 * q + 3] * s};
            if (c + 4 <= D) {
                if constexpr (sizeof(T) == 2) {
                    const uint2 u = make_uint2(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]));
                    __builtin_memcpy(row + c, &u, 8);
                } else {
                    __builtin_memcpy(row + c, v, 16);
                }
            } else if (!vec) {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (c + e < D) row[c + e] = from_f<T>(v[e]);
            }
        }
}

// ------------------------------------------------------------------ scores, base 2
// u log2(e) = S mul + add, or with a cap cl tanh(cs S) + add.  tanh(y) = 1 - 2 / (e^2y
// + 1), off by up to 2^-21 where y is far below zero and the quotient near 2: far below
// a bf16 probability's rounding.  fp32 takes |y| there, whose quotient is small (2^-22
// at 0.35, less above), and below 0.35, where this form would lose the leading digits,
// the series of tanh.
struct ScoreK {
    float mul;   // |scale| log2(e), not 0 so that it orders the scores and keeps -infinity
    float cs;    // scale / cap
    float cl;    // cap log2(e)
};
__device__ __forceinline__ ScoreK score_k(const fo_attn& a) {
    ScoreK k;
    k.mul = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);  // the least normal number
    k.cs = a.cap > 0.f ? a.scale / a.cap : 0.f;
    k.cl = a.cap * kLog2e;
    return k;
}
// Without a cap the sign of a negative scale goes into the row operand.
template <class T>
__device__ __forceinline__ void negate(Frag<T>& f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = -f.v[e];
}
// Scores -> tanh(cs S), slope = du / ds (or NULL).  A wave
// whose arguments all stay below 0.35, as scores usually do under their cap, takes
// the series alone: 9 instructions (fp32) against 16 with two at quarter rate.
template <class T, int N, class V>
__device__ __forceinline__ void cap_scores(V& S, const ScoreK& k, float* slope) {
    float top = 0.f;
#pragma unroll
    for (int r = 0; r < N; ++r) top = fmaxf(top, fabsf(S[r]));
    const bool high = __any(top * fabsf(k.cs) >= 0.35f);
    auto series = [&](float y) {  // of tanh: below 0.35 to 2^-24 in fp32, to 2^-17 in bf16
        const float y2 = y * y;
        float c = -17.f / 315.f;
        if (sizeof(T) == 4) c = fmaf(y2, fmaf(y2, fmaf(y2, -1382.f / 155925.f, 62.f / 2835.f), -17.f / 315.f), 2.f / 15.f);
        else c = fmaf(y2, c, 2.f / 15.f);
        c = fmaf(y2, c, -1.f / 3.f);
        return fmaf(y * y2, c, y);
    };
    auto put = [&](int r, float t) {
        if (slope) slope[r] = fmaf(-t, t, 1.f);
        S[r] = t;
    };
    if (!high) {
#pragma unroll
        for (int r = 0; r < N; ++r) put(r, series(S[r] * k.cs));
    } else {
#pragma unroll
        for (int r = 0; r < N; ++r) {
            const float y = S[r] * k.cs;
            const float z = sizeof(T) == 4 ? fabsf(y) : y;
            float t = fmaf(__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * (2.f * kLog2e)) + 1.f), -2.f, 1.f);
            if (sizeof(T) == 4) t = z < 0.35f ? series(y) : copysignf(t, y);
            put(r, t);
        }
    }
}

// The bias of distance n (clamped to the radius) in base 2; -infinity where it hides.
template <class T>
__device__ __forceinline__ float bias_at(const fo_attn& a, int h, int n) {
    const int g = min(max(a.bucket[min(max(n, -a.radius), a.radius) + a.radius], 0), a.n_buckets - 1);
    const float t = to_f(((const T*)a.table)[(int64_t)g * a.heads + h]);
    return t <= -1e30f ? -INFINITY : t * kLog2e;
}
// Distances of a 32-row by up to 64-column tile reach at most kReach past the
// radius before the whole tile lies beyond it, where its bias is one value.
constexpr int kReach = 96;
__host__ __device__ inline int lut_floats(const fo_attn& a) { return 2 * (a.radius + kReach) + 1; }
// Calls f(n) for n = t, t + step, .. < count, in a loop that no lane leaves early:
// one that lanes leave one by one had the compiler copy registers behind it
// before it turned the lanes on again.
template <class F>
__device__ __forceinline__ void each(int t, int step, int count, F f) {
    for (int n0 = 0; n0 < count; n0 += step)
        if (n0 + t < count) f(n0 + t);
}
template <class T>
__device__ __forceinline__ void fill_lut(float* lut, const fo_attn& a, int h, int tid, int step = 256) {
    each(tid, step, lut_floats(a), [&](int x) { lut[x] = bias_at<T>(a, h, x - a.radius - kReach); });
}

// One past the last key that query i sees: a prefix of the keys for every mask.
__device__ __forceinline__ int limit_of(const fo_attn& a, const Span& s, int pre, int i) {
    if (a.mask == FO_ATTN_FULL) return s.nk;
    return max(0, min(max(i + (s.nk - s.nq) + 1, pre), s.nk));
}

// keep factors of the 16 keys of a 32-key subtile from key j0 (a multiple of 32)
// on that this lane holds for query i: two generator calls.
__device__ __forceinline__ uint32_t keep_bits(uint32_t thr, int j0, int lh, int i, int bh, const fo_attn& a) {
    uint32_t bits = 0;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const uint4 w = philox7(2 * ((j0 >> 4) + m) + lh, i, bh, a.offset, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
#pragma unroll
        for (int e = 0; e < 8; ++e) bits |= (half_of(w, e) >= thr ? 1u : 0u) << (8 * m + e);
    }
    return bits;
}

}  // namespace fo
