// Dropout with bias and residual; the mask is drawn from the generator wherever
// it is needed and never stored.
#include "ops.h"

namespace fo {
namespace {

constexpr int kRowsPerPart = 64;  // rows of one partial column sum

// One thread per eight columns of a row: the eight numbers of one generator call.
template <class T, bool BWD>
__global__ void __launch_bounds__(256) dropout_kernel(DropArgs d, float* __restrict__ part) {
    const int calls = (d.cols + 7) / 8;
    const int cc = blockIdx.x * blockDim.x + threadIdx.x;
    if (cc >= calls) return;
    const int64_t r0 = (int64_t)blockIdx.y * kRowsPerPart, r1 = min(r0 + kRowsPerPart, d.rows);
    const int c0 = cc * 8, nc = min(8, d.cols - c0);
    const T *x = (const T*)d.x, *bias = (const T*)d.bias, *res = (const T*)d.res;
    T* y = (T*)d.y;
    float sum[8] = {};
    for (int64_t r = r0; r < r1; ++r) {
        const int64_t n = r * calls + cc;
        const uint4 w = philox7((uint32_t)n, (uint32_t)(n >> 32), 0u, d.offset, d.k0, d.k1);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e >= nc) continue;
            float v = to_f(x[r * d.x_ld + c0 + e]);
            if (!BWD && bias) v += to_f(bias[c0 + e]);
            v = half_of(w, e) >= d.thr ? v * d.keep_scale : 0.f;
            if (BWD) sum[e] += v;
            if (!BWD && res) v += to_f(res[r * d.res_ld + c0 + e]);
            y[r * d.y_ld + c0 + e] = from_f<T>(v);
        }
    }
    if (BWD && part)
        for (int e = 0; e < nc; ++e) part[(int64_t)blockIdx.y * d.cols + c0 + e] = sum[e];
}

template <class T>
__global__ void __launch_bounds__(256) dbias_kernel(const float* __restrict__ part, int parts, int cols,
                                                    T* __restrict__ out) {
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c >= cols) return;
    float s = 0.f;
    for (int p = 0; p < parts; ++p) s += part[(int64_t)p * cols + c];
    out[c] = from_f<T>(s);
}

}  // namespace

int64_t dropout_workspace(int64_t rows, int32_t cols) { return cdiv(rows, kRowsPerPart) * cols * 4; }

fo_status launch_dropout_fwd(int32_t dtype, const DropArgs& d, hipStream_t s) {
    const dim3 g((unsigned)cdiv(cdiv(d.cols, 8), 256), (unsigned)cdiv(d.rows, kRowsPerPart));
    if (dtype == FO_DT_BF16) dropout_kernel<bf16_t, false><<<g, 256, 0, s>>>(d, nullptr);
    else dropout_kernel<float, false><<<g, 256, 0, s>>>(d, nullptr);
    FO_LAUNCHED();
    return FO_OK;
}

fo_status launch_dropout_bwd(int32_t dtype, const DropArgs& d, void* dbias, float* ws, hipStream_t s) {
    const int parts = (int)cdiv(d.rows, kRowsPerPart);
    float* part = dbias ? ws : nullptr;
    if (parts) {
        const dim3 g((unsigned)cdiv(cdiv(d.cols, 8), 256), (unsigned)parts);
        if (dtype == FO_DT_BF16) dropout_kernel<bf16_t, true><<<g, 256, 0, s>>>(d, part);
        else dropout_kernel<float, true><<<g, 256, 0, s>>>(d, part);
        FO_LAUNCHED();
    }
    if (dbias) {
        const unsigned g = (unsigned)cdiv(d.cols, 256);
        if (dtype == FO_DT_BF16) dbias_kernel<bf16_t><<<g, 256, 0, s>>>(part, parts, d.cols, (bf16_t*)dbias);
        else dbias_kernel<float><<<g, 256, 0, s>>>(part, parts, d.cols, (float*)dbias);
        FO_LAUNCHED();
    }
    return FO_OK;
}

}  // namespace fo
