// Preference loss: a workgroup a pair, one launch.
//
// Twelve bytes a row and a handful of operations a pair: the call costs its launch
// and one pass of dependent loads.  Sums in fp64: answers are long, and the two
// sums of a pair nearly cancel.
#include "lm.h"

namespace fo {
namespace {

constexpr int THREADS = 256;

struct Rows {
    int64_t lo, hi;
};
__device__ __forceinline__ Rows answer(const PrefArgs& p, int64_t q) {
    const int64_t lo = min(max((int64_t)p.begin[q], (int64_t)0), p.rows);
    return {lo, min(max((int64_t)p.end[q], lo), p.rows)};
}

// log(1 + exp(x)) and 1 / (1 + exp(-x)), neither overflowing.
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.f) + log1pf(expf(-fabsf(x))); }
__device__ __forceinline__ float sigma(float x) {
    const float e = expf(-fabsf(x));
    return (x >= 0.f ? 1.f : e) / (1.f + e);
}

__global__ void __launch_bounds__(THREADS) pref_kernel(PrefArgs p) {
    __shared__ double part[2][THREADS / 64];
    const int64_t pair = block_of();
    if (pair >= p.pairs) return;
    const Rows at[2] = {answer(p, 2 * pair), answer(p, 2 * pair + 1)};
    double sum[2] = {0.0, 0.0};
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll 4
        for (int64_t r = at[q].lo + threadIdx.x; r < at[q].hi; r += THREADS)
            sum[q] += (double)p.logp[r] - (p.ref ? (double)p.ref[r] : 0.0);
#pragma unroll
        for (int m = 1; m < 64; m *= 2) sum[q] += __shfl_xor(sum[q], m);
        if ((threadIdx.x & 63) == 0) part[q][threadIdx.x >> 6] = sum[q];
    }
    __syncthreads();  // every row has been read: dlogp may lie over logp
    double reward[2];
    float each[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        reward[q] = 0.0;
#pragma unroll
        for (int k = 0; k < THREADS / 64; ++k) reward[q] += part[q][k];
        const int64_t n = at[q].hi - at[q].lo;
        const double b = p.mean && n > 1 ? (double)p.beta / (double)n : (double)p.beta;
        reward[q] *= b;
        each[q] = (float)b;
    }
    const float d = (float)(reward[0] - reward[1]);
    if (threadIdx.x == 0) {
        // a term without weight counts as 0 where it is infinite too
        p.loss[pair] = (p.smooth < 1.f ? (1.f - p.smooth) * softplus(-d) : 0.f) +
                       (p.smooth > 0.f ? p.smooth * softplus(d) : 0.f);
        p.reward[2 * pair] = (float)reward[0];
        p.reward[2 * pair + 1] = (float)reward[1];
    }
    if (!p.dlogp) return;
    const float slope = p.dloss * (p.smooth * sigma(d) - (1.f - p.smooth) * sigma(-d));
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const float g = (q ? -slope : slope) * each[q];
        for (int64_t r = at[q].lo + threadIdx.x; r < at[q].hi; r += THREADS) p.dlogp[r] = g;
    }
}

}  // namespace

fo_status launch_pref_loss(const PrefArgs& p, hipStream_t s) {
    pref_kernel<<<grid_of(p.pairs), THREADS, 0, s>>>(p);
    FO_LAUNCHED();
    return FO_OK;
}

}  // namespace fo
