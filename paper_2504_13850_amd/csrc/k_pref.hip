// Preference loss: a workgroup a pair, one launch.
//
// Twelve bytes a row and a handful of operations a pair: the call costs its launch
// and one pass of dependent loads.  All in fp64 up to the results' one rounding:
// answers are long, the two sums of a pair nearly cancel, and an error of d is a
// relative one of the loss and of its gradient.
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
    double reward[2], each[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        reward[q] = 0.0;
#pragma unroll
        for (int k = 0; k < THREADS / 64; ++k) reward[q] += part[q][k];
        const int64_t n = at[q].hi - at[q].lo;
        each[q] = p.mean && n > 1 ? (double)p.beta / (double)n : (double)p.beta;
        reward[q] *= each[q];
    }
    // log(1 + exp(+-d)) = max(+-d, 0) + log(1 + exp(-|d|)), 1 / (1 + exp(+-d)) from the same exponential: nothing overflows
    const double d = reward[0] - reward[1], smooth = p.smooth, e = exp(-fabs(d));
    if (threadIdx.x == 0) {
        const double both = log1p(e);
        // a term without weight counts as 0 where it is infinite too
        p.loss[pair] = (float)((smooth < 1.0 ? (1.0 - smooth) * (fmax(-d, 0.0) + both) : 0.0) +
                               (smooth > 0.0 ? smooth * (fmax(d, 0.0) + both) : 0.0));
        p.reward[2 * pair] = (float)reward[0];
        p.reward[2 * pair + 1] = (float)reward[1];
    }
    if (!p.dlogp) return;
    const double up = (d >= 0.0 ? 1.0 : e) / (1.0 + e), down = (d >= 0.0 ? e : 1.0) / (1.0 + e);
    const double slope = (double)p.dloss * (smooth * up - (1.0 - smooth) * down);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const float g = (float)((q ? -slope : slope) * each[q]);
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
