// Embedding: rows of a table by tokens, and the table's gradient.
#include "lm.h"
#include "row8.h"

namespace fo {
namespace {

// A thread takes eight columns of a row.
template <class T>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmbedArgs a) {
    const int chunks = (a.cols + 7) / 8;
    const int64_t id = (int64_t)block_of() * 256 + threadIdx.x, row = id / chunks;
    if (row >= a.rows) return;
    const int c0 = (int)(id % chunks) * 8, n = min(8, a.cols - c0), token = a.tokens[row];
    float y[8] = {};
    if (token >= 0 && token < a.vocab) {
        Eight<T, false> x;
        x.load((const T*)a.table + token * a.table_ld + c0, n, n == 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x.at(e) * a.scale;
    }
    Eight<T, false>::store((T*)a.out + row * a.out_ld + c0, y, n, n == 8);
}

// A workgroup owns a row of the table and looks through all tokens.
template <class T>
__global__ void __launch_bounds__(256) embed_bwd_kernel(EmbedArgs a) {
    __shared__ int tok[2048];
    const int64_t v = block_of();
    if (v >= a.vocab) return;
    for (int64_t b0 = 0; b0 < a.cols; b0 += 2048) {
        const int64_t c0 = b0 + threadIdx.x * 8;
        const int n = (int)min((int64_t)8, a.cols - c0);
        float sum[8] = {};
        for (int64_t r0 = 0; r0 < a.rows; r0 += 2048) {
            const int m = (int)min((int64_t)2048, a.rows - r0);
            __syncthreads();
            for (int i = threadIdx.x; i < m; i += 256) tok[i] = a.tokens[r0 + i];
            __syncthreads();
            for (int i = 0; i < m; ++i) {
                if (tok[i] != v || n <= 0) continue;
                Eight<T, false> x;
                x.load((const T*)a.dout + (r0 + i) * a.dout_ld + c0, n, n == 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += x.at(e);
            }
        }
        if (n <= 0) continue;
        T* y = (T*)a.dtable + v * a.dtable_ld + c0;
        if (a.accumulate) {
            Eight<T, false> old;
            old.load(y, n, n == 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = sum[e] * a.scale + old.at(e);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] *= a.scale;
        }
        Eight<T, false>::store(y, sum, n, n == 8);
    }
}

}  // namespace

fo_status launch_embed_fwd(int32_t dtype, const EmbedArgs& a, hipStream_t s) {
    const dim3 g = grid_of(cdiv(a.rows * cdiv(a.cols, 8), 256));
    if (dtype == FO_DT_BF16) embed_fwd_kernel<bf16_t><<<g, 256, 0, s>>>(a);
    else embed_fwd_kernel<float><<<g, 256, 0, s>>>(a);
    FO_LAUNCHED();
    return FO_OK;
}

int64_t embed_workspace(int64_t rows, int32_t cols, int32_t vocab) { return 0; }

fo_status launch_embed_bwd(int32_t dtype, const EmbedArgs& a, void* ws, hipStream_t s) {
    if (dtype == FO_DT_BF16) embed_bwd_kernel<bf16_t><<<grid_of(a.vocab), 256, 0, s>>>(a);
    else embed_bwd_kernel<float><<<grid_of(a.vocab), 256, 0, s>>>(a);
    FO_LAUNCHED();
    return FO_OK;
}

}  // namespace fo
