// Dropout with bias and residual; the mask is drawn from the generator wherever
// it is needed and never stored.
//
// Bound by HBM: per element two or three reads and writes against 1/8 of a
// generator call (about 70 instructions, a third of them at quarter rate: the
// chip draws some 2e12 numbers a second, 13 TB/s of bf16 input, residual and
// output).  65536 x 768 bf16 with residual, 302 MB: 53 us, 5.7 TB/s; a copy of a
// GiB runs at 5.15.  That is for rows that all start 16-byte aligned; one operand whose
// rows do not (a dense bf16 width that is no multiple of 8) puts the whole call on
// element by element loads and stores.
#include <algorithm>

#include "row8.h"

namespace fo {
namespace {

// A workgroup is 2^tx threads along the columns, eight columns (one generator
// call) each, by 256 / 2^tx rows; a thread takes `steps` rows that many apart.
// Up to 32 threads on a row make 512-byte (bf16) runs; wider workgroups would
// leave more threads past the last column.
struct DropShape {
    int tx, rows, steps;  // log2 of the threads per row, rows side by side, rows per thread
    int xb, parts;        // workgroups along the columns, along the rows
};
// Rows per thread grow until about `most` workgroups are left: 8192 (302 MB in 53
// us, with 2048 in 56), or 2048 where a column sum over the parts follows.
DropShape drop_shape(int64_t rows, int32_t cols, int64_t most) {
    DropShape f;
    const int64_t calls = cdiv(cols, 8);
    f.tx = 0;
    while (f.tx < 5 && (1 << f.tx) < calls) ++f.tx;
    f.rows = 256 >> f.tx;
    f.xb = (int)cdiv(calls, 1 << f.tx);
    const int64_t wgs = f.xb * cdiv(rows, f.rows);
    f.steps = (int)std::min<int64_t>(std::max<int64_t>(1, wgs / most), 1 << 20);
    f.parts = (int)cdiv(rows, (int64_t)f.rows * f.steps);
    return f;
}
constexpr int64_t kFwdWgs = 8192, kBwdWgs = 2048;

constexpr int FLY = 4;  // rows of a thread in flight

// BWD: x is dy and y is dx; part (may be NULL) receives the workgroup's column sums.
template <class T, bool BWD, bool NT>
__global__ void __launch_bounds__(256) dropout_kernel(DropArgs d, DropShape f, bool vec, float* __restrict__ part) {
    __shared__ float sums[BWD ? 256 * 8 : 1];
    const int calls = (d.cols + 7) / 8, tid = threadIdx.x;
    const int cc = blockIdx.x * (1 << f.tx) + (tid & ((1 << f.tx) - 1)), ty = tid >> f.tx;
    const int c0 = cc * 8, n = min(8, d.cols - c0);
    const bool v8 = vec && n == 8, in = cc < calls;
    const T *x = (const T*)d.x + c0, *res = (const T*)d.res + c0;
    T* y = (T*)d.y + c0;
    float b[8] = {}, sum[8] = {};
    if (!BWD && d.bias && in) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) b[e] = to_f(((const T*)d.bias)[c0 + e]);
    }
    if (in) {
        const int64_t r0 = (int64_t)blockIdx.y * f.rows * f.steps + ty;
        // this thread's rows: r0, r0 + f.rows, ..
        const int left = r0 < d.rows ? (int)min((d.rows - 1 - r0) / f.rows + 1, (int64_t)f.steps) : 0;
        const int64_t dx = f.rows * d.x_ld, dr = f.rows * d.res_ld, dy = f.rows * d.y_ld;
        x += r0 * d.x_ld;
        res += r0 * d.res_ld;
        y += r0 * d.y_ld;
        int64_t call = r0 * calls + cc;
        for (int st = 0; st < left; st += FLY) {
            Eight<T, NT> xv[FLY], rv[FLY];
#pragma unroll
            for (int u = 0; u < FLY; ++u)
                if (st + u < left) {
                    xv[u].load(x + u * dx, n, v8);
                    if (!BWD && d.res) rv[u].load(res + u * dr, n, v8);
                }
#pragma unroll
            for (int u = 0; u < FLY; ++u)
                if (st + u < left) {
                    const uint4 w = philox7((uint32_t)call, (uint32_t)(call >> 32), 0u, d.offset, d.k0, d.k1);
                    float out[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float v = xv[u].at(e);
                        if (!BWD) v += b[e];
                        v = half_of(w, e) >= d.thr ? v * d.keep_scale : 0.f;
                        if (BWD) sum[e] += v;
                        else if (d.res) v += rv[u].at(e);
                        out[e] = v;
                    }
                    Eight<T, NT>::store(y, out, n, v8);
                    y += dy;
                    call += (int64_t)f.rows * calls;
                }
            x += FLY * dx;
            res += FLY * dr;
        }
    }
    if (!BWD || !part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[e * 256 + tid] = sum[e];
    __syncthreads();
    // 8 << tx columns; column e of thread t: rows in order
    for (int x8 = tid; x8 < 8 << f.tx; x8 += 256) {
        const int t = x8 >> 3, e = x8 & 7, c = (blockIdx.x * (1 << f.tx) + t) * 8 + e;
        float s = 0.f;
        for (int q = 0; q < f.rows; ++q) s += sums[e * 256 + (q << f.tx) + t];
        if (c < d.cols) part[(int64_t)blockIdx.y * d.cols + c] = s;
    }
}

template <class T, bool BWD>
fo_status run(const DropArgs& d, const DropShape& f, float* part, hipStream_t s) {
    const bool vec = vec_rows<T>(d.x, d.x_ld) && vec_rows<T>(d.y, d.y_ld) && (!d.res || vec_rows<T>(d.res, d.res_ld));
    // What passes the 256 MB last-level cache by goes round the caches (302 MB: 53
    // us, 58 through them); less stays where the next kernel finds it.
    const bool nt = d.rows * d.cols * (int64_t)sizeof(T) * (d.res ? 3 : 2) > (int64_t(256) << 20);
    if (nt) dropout_kernel<T, BWD, true><<<dim3(f.xb, f.parts), 256, 0, s>>>(d, f, vec, part);
    else dropout_kernel<T, BWD, false><<<dim3(f.xb, f.parts), 256, 0, s>>>(d, f, vec, part);
    FO_LAUNCHED();
    return FO_OK;
}
template <class T>
fo_status bwd(const DropArgs& d, void* dbias, float* ws, hipStream_t s) {
    const DropShape f = drop_shape(d.rows, d.cols, kBwdWgs);
    if (d.rows) {
        const fo_status st = run<T, true>(d, f, dbias ? ws : nullptr, s);
        if (st != FO_OK) return st;
    }
    if (dbias) {
        return column_sums<T>(ws, f.parts, d.cols, (T*)dbias, s);
    }
    return FO_OK;
}

}  // namespace

int64_t dropout_workspace(int64_t rows, int32_t cols) { return (int64_t)drop_shape(rows, cols, kBwdWgs).parts * cols * 4; }

fo_status launch_dropout_fwd(int32_t dtype, const DropArgs& d, hipStream_t s) {
    const DropShape f = drop_shape(d.rows, d.cols, kFwdWgs);
    return dtype == FO_DT_BF16 ? run<bf16_t, false>(d, f, nullptr, s) : run<float, false>(d, f, nullptr, s);
}

fo_status launch_dropout_bwd(int32_t dtype, const DropArgs& d, void* dbias, float* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? bwd<bf16_t>(d, dbias, ws, s) : bwd<float>(d, dbias, ws, s);
}

}  // namespace fo
