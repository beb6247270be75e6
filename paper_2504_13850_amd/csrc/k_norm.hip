// RMS norm with the residual's addition, forward and backward, and rows in 8 bits.
//
// Bound by HBM: every operand is read once and every result written once.  A row
// lies in the registers of its team of threads between the sum of its squares and
// its results, so that nothing is read twice.
#include <algorithm>

#include "lm.h"
#include "row8.h"

namespace fo {
namespace {

constexpr float kF8Max = 448.f;  // largest e4m3
constexpr float kTiny = 0x1p-100f;

// THREADS threads a workgroup, TPR of them on a row, NC times eight columns each.
template <int THREADS_, int TPR_, int NC_>
struct Shape {
    static constexpr int THREADS = THREADS_, TPR = TPR_, NC = NC_, RPW = THREADS_ / TPR_;
    static constexpr int64_t COLS = int64_t(TPR_) * NC_ * 8;
};

// The narrowest of the shapes that holds a row, up to `most` columns; false for rows that none holds.
template <class F>
bool with_shape(int32_t cols, int64_t most, F f) {
    if (cols > most) return false;
    if (cols <= Shape<256, 16, 1>::COLS) f(Shape<256, 16, 1>{});
    else if (cols <= Shape<256, 64, 1>::COLS) f(Shape<256, 64, 1>{});
    else if (cols <= Shape<256, 64, 2>::COLS) f(Shape<256, 64, 2>{});
    else if (cols <= Shape<256, 256, 1>::COLS) f(Shape<256, 256, 1>{});
    else if (cols <= Shape<256, 256, 2>::COLS) f(Shape<256, 256, 2>{});
    else if (cols <= Shape<256, 256, 3>::COLS) f(Shape<256, 256, 3>{});
    else if (cols <= Shape<1024, 1024, 1>::COLS) f(Shape<1024, 1024, 1>{});
    else if (cols <= Shape<1024, 1024, 2>::COLS) f(Shape<1024, 1024, 2>{});
    else if (cols <= Shape<1024, 1024, 4>::COLS) f(Shape<1024, 1024, 4>{});
    else return false;
    return true;
}

// Four or eight e4m3 to a word or two, round to nearest even.
__device__ __forceinline__ uint2 pack_f8(const float* x) {
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}
__device__ __forceinline__ void store_f8(uint8_t* p, const float* x, int n) {
    const uint2 u = pack_f8(x);
    if (n == 8) {
        __builtin_memcpy(p, &u, 8);
    } else {
        uint8_t v[8];
        __builtin_memcpy(v, &u, 8);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = v[e];
    }
}

// eps = 0 and a row of zeros: y = 0.
__device__ __forceinline__ float rstd_of(float squares, int cols, float eps) {
    const float m = squares / (float)cols + eps;
    return m > 0.f || m != m ? 1.f / sqrtf(m) : 0.f;
}
// scale = top / 448, and its reciprocal.
__device__ __forceinline__ float2 f8_scale(float top) {
    return make_float2((top > 0.f && top < kTiny ? kTiny : top) / kF8Max, kF8Max / fmaxf(top, kTiny));
}

// h = x + residual of one chunk, stored where it is asked for.
template <class T, bool NT>
__device__ __forceinline__ void load_h(const NormArgs& a, int64_t row, int c0, int n, float* h) {
    Eight<T, NT> x, r;
    x.load((const T*)a.x + row * a.x_ld + c0, n, n == 8);
    if (a.res) r.load((const T*)a.res + row * a.res_ld + c0, n, n == 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = a.res ? x.at(e) + r.at(e) : x.at(e);
}
// w of one chunk; zeros past the row's end, so that what lies there takes no part.
template <class T>
__device__ __forceinline__ void load_w(const void* w, int c0, int n, float* f) {
    Eight<T, false> u;
    if (w) u.load((const T*)w + c0, n, n == 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = e < n ? (w ? u.at(e) : 1.f) : 0.f;
}

// NT: operands past the caches.
template <class T, class S, int OUT, bool NT>
__global__ void __launch_bounds__(S::THREADS) norm_kernel(NormArgs a) {
    __shared__ float lds[32];
    const int t = threadIdx.x % S::TPR;
    const int64_t row = (int64_t)block_of() * S::RPW + threadIdx.x / S::TPR;
    if (row >= a.rows) return;  // whole teams, and whole workgroups where a team needs a barrier
    float h[S::NC][8], w[S::NC][8], ss = 0.f, top = 0.f;
    Eight<T, NT> x[S::NC], res[S::NC];
    Eight<T, false> u[S::NC];
#pragma unroll
    for (int c = 0; c < S::NC; ++c) {
        const int c0 = (t + c * S::TPR) * 8;
        if (c0 >= a.cols) continue;
        x[c].load_row((const T*)a.x + row * a.x_ld, c0, a.cols);
        if (a.res) res[c].load_row((const T*)a.res + row * a.res_ld, c0, a.cols);
        if (OUT != kQuantF8 && a.w) u[c].load_row((const T*)a.w, c0, a.cols);
    }
#pragma unroll
    for (int c = 0; c < S::NC; ++c) {
        const int n = min(8, a.cols - (t + c * S::TPR) * 8);
        x[c].fit(n, a.cols);
        if (a.res) res[c].fit(n, a.cols);
        if (OUT != kQuantF8 && a.w) u[c].fit(n, a.cols);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[c][e] = n <= 0 ? 0.f : a.res ? x[c].at(e) + res[c].at(e) : x[c].at(e);
            w[c][e] = n <= 0 ? 0.f : OUT != kQuantF8 && a.w ? u[c].at(e) : 1.f;
        }
    }
#pragma unroll
    for (int c = 0; c < S::NC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += h[c][e] * h[c][e];
    float r = 1.f;
    if (OUT != kQuantF8) r = rstd_of(team<S::TPR>(ss, lds, Add()), a.cols, a.eps);
    // the largest of y itself: h w may leave fp32's range where y does not
#pragma unroll
    for (int c = 0; c < S::NC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(OUT == kQuantF8 ? h[c][e] : h[c][e] * r * w[c][e]));
    float2 f8 = make_float2(0.f, 0.f);
    if (OUT != kNorm) f8 = f8_scale(team<S::TPR>(top, lds + 16, Max()));
    if (t == 0) {
        if (OUT == kNorm && a.rstd) a.rstd[row] = r;
        if (OUT != kNorm) a.y_scale[row] = f8.x;
    }
#pragma unroll
    for (int c = 0; c < S::NC; ++c) {
        const int c0 = (t + c * S::TPR) * 8, n = min(8, a.cols - c0);
        if (n <= 0) continue;
        if (a.h) Eight<T, false>::store((T*)a.h + row * a.h_ld + c0, h[c], n, n == 8);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e] = OUT == kQuantF8 ? h[c][e] : h[c][e] * r * w[c][e];
            if (OUT != kNorm) y[e] *= f8.y;
        }
        if (OUT == kNorm) Eight<T, false>::store((T*)a.y + row * a.y_ld + c0, y, n, n == 8);
        else store_f8((uint8_t*)a.y + row * a.y_ld + c0, y, n);
    }
}

// Rows longer than the registers hold: read twice.  A thread writes only what it read itself, so in place works too.
template <class T, int OUT>
__global__ void __launch_bounds__(1024) norm_long_kernel(NormArgs a) {
    __shared__ float lds[32];
    const int64_t row = block_of();
    if (row >= a.rows) return;
    float ss = 0.f;
    double top = 0.0;  // |h w| before the row's factor is known: within range in 64 bits
    for (int64_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += 8192) {
        const int n = (int)min((int64_t)8, a.cols - c0);
        float h[8], w[8];
        load_h<T, false>(a, row, (int)c0, n, h);
        if (OUT == kNormF8) load_w<T>(a.w, (int)c0, n, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            ss += h[e] * h[e];
            top = fmax(top, fabs(OUT == kNormF8 ? (double)h[e] * w[e] : (double)h[e]));
        }
    }
    float r = 1.f;
    if (OUT != kQuantF8) r = rstd_of(team<1024>(ss, lds, Add()), a.cols, a.eps);
    float2 f8 = make_float2(0.f, 0.f);
    if (OUT != kNorm) f8 = f8_scale(team<1024>((float)(top * r), lds + 16, Max()));
    if (threadIdx.x == 0) {
        if (OUT == kNorm && a.rstd) a.rstd[row] = r;
        if (OUT != kNorm) a.y_scale[row] = f8.x;
    }
    for (int64_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += 8192) {
        const int n = (int)min((int64_t)8, a.cols - c0);
        float h[8], w[8], y[8];
        load_h<T, false>(a, row, (int)c0, n, h);
        if (OUT != kQuantF8) load_w<T>(a.w, (int)c0, n, w);
        if (a.h) Eight<T, false>::store((T*)a.h + row * a.h_ld + c0, h, n, n == 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e] = OUT == kQuantF8 ? h[e] : h[e] * r * w[e];
            if (OUT != kNorm) y[e] *= f8.y;
        }
        if (OUT == kNorm) Eight<T, false>::store((T*)a.y + row * a.y_ld + c0, y, n, n == 8);
        else store_f8((uint8_t*)a.y + row * a.y_ld + c0, y, n);
    }
}

// Operands that no cache keeps: 16384 rows of 4096 bf16, a pass forward and backward 166 us with the loads and
// dx past the caches, which leaves h and y to the launches that read them, 203 through them (stores of h and y past them
// too cost another 14).
template <class T>
bool past_caches(int64_t rows, int32_t cols) { return 4 * rows * cols * (int64_t)sizeof(T) > int64_t(256) << 20; }

template <class T, int OUT>
fo_status fwd(const NormArgs& a, hipStream_t s) {
    const bool held = with_shape(a.cols, INT32_MAX, [&](auto shape) {
        using S = decltype(shape);
        const dim3 g = grid_of(cdiv(a.rows, S::RPW));
        if (OUT == kNorm && past_caches<T>(a.rows, a.cols)) norm_kernel<T, S, OUT, OUT == kNorm><<<g, S::THREADS, 0, s>>>(a);
        else norm_kernel<T, S, OUT, false><<<g, S::THREADS, 0, s>>>(a);
    });
    if (!held) norm_long_kernel<T, OUT><<<grid_of(a.rows), 1024, 0, s>>>(a);
    FO_LAUNCHED();
    return FO_OK;
}
template <class T>
fo_status fwd_any(NormOut out, const NormArgs& a, hipStream_t s) {
    return out == kNorm ? fwd<T, kNorm>(a, s) : out == kNormF8 ? fwd<T, kNormF8>(a, s) : fwd<T, kQuantF8>(a, s);
}

// ------------------------------------------------------------------ backward
// Columns that the registers of a workgroup hold with the weight's gradient (3000 rows of 20000 bf16: 153 us through the
// long rows' kernels, 320 with what spills; fp32, 2000 rows without residual: 192 and 316).
constexpr int64_t kBwdCols = Shape<1024, 1024, 2>::COLS;

// Workgroups, and parts of the weight's gradient: each takes every so many-th row.  As many as the chip has room for:
// parts are written and read once more (bf16 with residual: 2048 rows of 16384 58 us with 256 parts, 75 with 512, 104
// with 1024; 4096 of 4096 31 with 512, 36 with 1024).  Of short rows more, two rows a team (100000 of 64: 19 us with
// 1024, 26 with 512).  Long rows: 1024 workgroups along rows and columns.
int64_t bwd_parts(int64_t rows, int32_t cols) {
    int64_t rpw = 1, most = std::max<int64_t>(1, 1024 / cdiv(cols, 2048));
    with_shape(cols, kBwdCols, [&](auto shape) { rpw = decltype(shape)::RPW, most = decltype(shape)::THREADS == 1024 ? 256 : 512; });
    const int64_t n = cdiv(rows, rpw);
    return std::max<int64_t>(1, std::min(n, cols > 512 ? most : std::min<int64_t>(1024, std::max(most, n / 2))));
}

// 64 columns of dw, all rows: eight threads along the columns, the others' sums joined in order.
template <class T, int THREADS>
__device__ void dw_columns(const NormBwdArgs& a, int64_t id, float* sums) {
    constexpr int TEAMS = THREADS / 8;
    const int tx = threadIdx.x % 8, ty = threadIdx.x / 8;
    const int64_t c0 = id * 64 + tx * 8;
    const int n = (int)min((int64_t)8, a.cols - c0);
    float dw[8] = {};
    if (n > 0) {
#pragma unroll 4
        for (int64_t row = ty; row < a.rows; row += TEAMS) {
            Eight<T, false> g, x;
            g.load((const T*)a.dy + row * a.dy_ld + c0, n, n == 8);
            x.load((const T*)a.h + row * a.h_ld + c0, n, n == 8);
            const float r = a.rstd[row];
#pragma unroll
            for (int e = 0; e < 8; ++e) dw[e] += g.at(e) * (x.at(e) * r);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[ty * 64 + tx * 8 + e] = dw[e];
    __syncthreads();
    const int64_t c = id * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || c >= a.cols) return;
    float s = 0.f;
#pragma unroll 8
    for (int k = 0; k < TEAMS; ++k) s += sums[k * 64 + threadIdx.x];
    ((T*)a.dw)[c] = from_f<T>(s);
}

// NT: operands past the caches, and dx.  FEW: workgroups past `rows_wgs` write dw, from dy and h read once more, in the
// same launch; else each leaves its rows' part of it.
template <class T, class S, bool NT, bool FEW>
__global__ void __launch_bounds__(S::THREADS) norm_bwd_kernel(NormBwdArgs a, int rows_wgs) {
    __shared__ float lds[2][16];
    __shared__ float sums[S::RPW > 1 || FEW ? 8 * S::THREADS : 1];
    if (FEW && (int)blockIdx.x >= rows_wgs) {
        dw_columns<T, S::THREADS>(a, (int)blockIdx.x - rows_wgs, sums);
        return;
    }
    // Where a whole workgroup of 1024 has a row, the next one's loads are in flight if the registers hold both.
    constexpr bool NEXT = S::TPR == 1024 && S::NC == 1;
    // Row's ends by load_row in 16 bits (5247 rows of 6845 87 us, 109 by single elements); in 32 the registers that fit()
    // needs cost more (12020 rows of 753 34 and 31).
    constexpr bool FIT = sizeof(T) == 2;
    const int t = threadIdx.x % S::TPR, ty = threadIdx.x / S::TPR;
    float w[S::NC][8], dw[S::NC][8] = {};
#pragma unroll
    for (int c = 0; c < S::NC; ++c) load_w<T>(a.w, (t + c * S::TPR) * 8, min(8, a.cols - (t + c * S::TPR) * 8), w[c]);
    struct Operands {
        Eight<T, NT> dy[S::NC], h[S::NC], dr[S::NC];
        float r;
    };
    const auto load = [&](int64_t row, Operands& o) {
        o.r = a.rstd[row];
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const int c0 = (t + c * S::TPR) * 8, n = min(8, a.cols - c0);
            const auto get = [&](const void* p, int64_t ld, Eight<T, NT>& x) {
                if (FIT) x.load_row((const T*)p + row * ld, c0, a.cols);
                else x.load((const T*)p + row * ld + c0, n, n == 8);
            };
            if (FIT && n <= 0) continue;
            get(a.dy, a.dy_ld, o.dy[c]);
            get(a.h, a.h_ld, o.h[c]);
            if (a.dres) get(a.dres, a.dres_ld, o.dr[c]);
        }
    };
    const int64_t row0 = (int64_t)blockIdx.x * S::RPW + ty, each = (int64_t)rows_wgs * S::RPW;
    Operands o, next;
    if (NEXT && row0 < a.rows) load(row0, o);
    int turn = 0;
    for (int64_t row = row0; row < a.rows; row += each) {
        if (!NEXT) load(row, o);
        else if (row + each < a.rows) load(row + each, next);
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const int n = min(8, a.cols - (t + c * S::TPR) * 8);
            if (FIT) {
                o.dy[c].fit(n, a.cols);
                o.h[c].fit(n, a.cols);
                if (a.dres) o.dr[c].fit(n, a.cols);
            }
            if (!FIT || n > 0)
#pragma unroll
                for (int e = 0; e < 8; ++e) dot += o.dy[c].at(e) * w[c][e] * o.h[c].at(e);
        }
        dot = team<S::TPR>(dot, lds[turn & 1], Add());
        ++turn;
        const float r = o.r, k = r * r * (dot / (float)a.cols);
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const int c0 = (t + c * S::TPR) * 8, n = min(8, a.cols - c0);
            float dx[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = o.dy[c].at(e), x = o.h[c].at(e);
                dx[e] = r * (g * w[c][e] - x * k);
                if (a.dres) dx[e] += o.dr[c].at(e);
                dw[c][e] += g * (x * r);
            }
            if (n > 0) Eight<T, NT>::store((T*)a.dx + row * a.dx_ld + c0, dx, n, n == 8);
        }
        if (NEXT) o = next;
    }
    if (FEW || !a.part) return;
#pragma unroll
    for (int c = 0; c < S::NC; ++c) {
        if constexpr (S::RPW > 1) {  // the teams' sums, in order
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[e * S::THREADS + threadIdx.x] = dw[c][e];
            __syncthreads();
            for (int x = threadIdx.x; x < S::TPR * 8; x += S::THREADS) {
                const int e = x % 8, u = x / 8, col = (u + c * S::TPR) * 8 + e;
                float s = 0.f;
#pragma unroll
                for (int q = 0; q < S::RPW; ++q) s += sums[e * S::THREADS + q * S::TPR + u];
                if (col < a.cols) a.part[(int64_t)blockIdx.x * a.cols + col] = s;
            }
        } else {
            const int c0 = (t + c * S::TPR) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c0 + e < a.cols) a.part[(int64_t)blockIdx.x * a.cols + c0 + e] = dw[c][e];
        }
    }
}

// Rows longer than the registers hold: read twice, the weight's gradient by a kernel of its own before that (dx may
// lie over what it reads).
template <class T>
__global__ void __launch_bounds__(1024) norm_bwd_long_kernel(NormBwdArgs a) {
    __shared__ float lds[16];
    const int64_t row = block_of();
    if (row >= a.rows) return;
    const T *dy = (const T*)a.dy + row * a.dy_ld, *h = (const T*)a.h + row * a.h_ld;
    const float r = a.rstd[row];
    float dot = 0.f;
    for (int64_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += 8192) {
        const int n = (int)min((int64_t)8, a.cols - c0);
        Eight<T, false> g, x;
        float w[8];
        g.load(dy + c0, n, n == 8);
        x.load(h + c0, n, n == 8);
        load_w<T>(a.w, (int)c0, n, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot += g.at(e) * w[e] * x.at(e);
    }
    const float k = r * r * (team<1024>(dot, lds, Add()) / (float)a.cols);
    for (int64_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += 8192) {
        const int n = (int)min((int64_t)8, a.cols - c0);
        Eight<T, false> g, x, d;
        float w[8], dx[8];
        g.load(dy + c0, n, n == 8);
        x.load(h + c0, n, n == 8);
        if (a.dres) d.load((const T*)a.dres + row * a.dres_ld + c0, n, n == 8);
        load_w<T>(a.w, (int)c0, n, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dx[e] = r * (g.at(e) * w[e] - x.at(e) * k);
            if (a.dres) dx[e] += d.at(e);
        }
        Eight<T, false>::store((T*)a.dx + row * a.dx_ld + c0, dx, n, n == 8);
    }
}
// A thread's eight columns down every parts-th row.
template <class T>
__global__ void __launch_bounds__(256) norm_dw_long_kernel(NormBwdArgs a, int parts) {
    const int64_t c0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    const int n = (int)min((int64_t)8, a.cols - c0);
    if (n <= 0) return;
    float dw[8] = {};
    for (int64_t row = blockIdx.y; row < a.rows; row += parts) {
        Eight<T, false> g, x;
        g.load((const T*)a.dy + row * a.dy_ld + c0, n, n == 8);
        x.load((const T*)a.h + row * a.h_ld + c0, n, n == 8);
        const float r = a.rstd[row];
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[e] += g.at(e) * (x.at(e) * r);
    }
    for (int e = 0; e < n; ++e) a.part[blockIdx.y * (int64_t)a.cols + c0 + e] = dw[e];
}

// Up to 512 rows dw is cheaper read for than joined in a second launch (a pass forward and backward, bf16: 4 rows of 768
// 7.6 us and 10.3, 512 of 8192 23 and 32; 1024 of 768 14 and 12), unless dx lies over what it reads.
constexpr int64_t kFewRows = 512;
template <class T>
fo_status bwd(const NormBwdArgs& args, void* dw, hipStream_t s) {
    NormBwdArgs a = args;
    const int parts = (int)bwd_parts(a.rows, a.cols);
    const bool few = dw && a.rows <= kFewRows && a.rows > 0 && a.cols <= kBwdCols && a.dx != a.dy && a.dx != a.h;
    if (a.rows) {
        const bool held = with_shape(a.cols, kBwdCols, [&](auto shape) {
            using S = decltype(shape);
            if (few) {
                a.dw = dw;
                norm_bwd_kernel<T, S, false, true><<<parts + (int)cdiv(a.cols, 64), S::THREADS, 0, s>>>(a, parts);
            } else if (past_caches<T>(a.rows, a.cols)) {
                norm_bwd_kernel<T, S, true, false><<<parts, S::THREADS, 0, s>>>(a, parts);
            } else {
                norm_bwd_kernel<T, S, false, false><<<parts, S::THREADS, 0, s>>>(a, parts);
            }
        });
        if (!held) {
            if (a.part) {
                norm_dw_long_kernel<T><<<dim3((unsigned)cdiv(a.cols, 2048), parts), 256, 0, s>>>(a, parts);
                FO_LAUNCHED();
            }
            norm_bwd_long_kernel<T><<<grid_of(a.rows), 1024, 0, s>>>(a);
        }
        FO_LAUNCHED();
    }
    return dw && !few ? column_sums<T>(a.part, a.rows ? parts : 0, a.cols, (T*)dw, s) : FO_OK;
}

}  // namespace

int64_t norm_workspace(int64_t rows, int32_t cols) { return bwd_parts(rows, cols) * cols * 4; }

fo_status launch_norm_fwd(int32_t dtype, NormOut out, const NormArgs& a, hipStream_t s) {
    return dtype == FO_DT_BF16 ? fwd_any<bf16_t>(out, a, s) : fwd_any<float>(out, a, s);
}

fo_status launch_norm_bwd(int32_t dtype, const NormBwdArgs& a, void* dw, hipStream_t s) {
    return dtype == FO_DT_BF16 ? bwd<bf16_t>(a, dw, s) : bwd<float>(a, dw, s);
}

}  // namespace fo
