// Products of 8-bit rows with a scale each: c_mn = a_scale[m] b_scale[n] sum_k a_mk b_nk.
#include "lm.h"
#include "row8.h"

namespace fo {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// c += a b^T of 16 rows and columns over 128 of k.  Lane l holds 32 bytes of row l % 16 of either operand, those of
// k = 32 (l / 16) on (any order of k serves, the same for both); c: column l % 16, rows 4 (l / 16) ..
//
// For results in bf16 the 8-bit matrix instruction: it adds products by eights, cutting each below 2^-13 of the
// largest of its eight (measured; 1.4e-5 of the result's norm where the operands are normal, and at most 7 2^-13 of
// the terms' sizes), and what it adds up is fp32.  For results in fp32 that would be seen: there the bytes become bf16,
// which holds each of them exactly, at a fourth of the rate.
template <class T>
__device__ __forceinline__ f32x4 mfma_f8(i32x8 a, i32x8 b, f32x4 c);
template <>
__device__ __forceinline__ f32x4 mfma_f8<bf16_t>(i32x8 a, i32x8 b, f32x4 c) {
    constexpr int kOne = 0x7F7F7F7F;  // block scales of 1
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, kOne, 0, kOne);
}
__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
    const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)};
    return __builtin_bit_cast(bf16x8, v);
}
template <>
__device__ __forceinline__ f32x4 mfma_f8<float>(i32x8 a, i32x8 b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 8; i += 2)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(a[i], a[i + 1]), widen(b[i], b[i + 1]), c, 0, 0, 0);
    return c;
}

// Any sizes, strides and alignments: 64 rows by 64 columns a workgroup, 16 bytes at a time where a chunk lies inside
// the row, byte by byte in its tail.
template <class T>
__global__ void __launch_bounds__(256) gemm_f8_any_kernel(GemmF8Args g) {
    constexpr int BK = 128, LD = BK + 16;
    __shared__ __align__(16) uint8_t lds[2][64 * LD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t tiles_n = (g.N + 63) / 64, id = block_of();
    const int64_t m0 = id / tiles_n * 64;
    const int n0 = (int)(id % tiles_n) * 64;
    if (m0 >= g.M) return;
    f32x4 acc[4] = {};
    for (int64_t k0 = 0; k0 < g.K; k0 += BK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // 2 x 64 rows x 8 chunks
            const int x = tid + 256 * i, op = x >> 9, r = (x >> 3) & 63, c = (x & 7) * 16;
            const bool ok = op ? n0 + r < g.N : m0 + r < g.M;
            const uint8_t* p = op ? g.b + (int64_t)(n0 + r) * g.ldb : g.a + (m0 + r) * g.lda;
            uint8_t v[16] = {};
            if (ok && k0 + c + 16 <= g.K) {
                __builtin_memcpy(v, p + k0 + c, 16);
            } else if (ok) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k0 + c + e < g.K) v[e] = p[k0 + c + e];
            }
            __builtin_memcpy(&lds[op][r * LD + c], v, 16);
        }
        __syncthreads();
        i32x8 a;
        __builtin_memcpy(&a, &lds[0][(wave * 16 + (lane & 15)) * LD + (lane >> 4) * 32], 32);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            i32x8 b;
            __builtin_memcpy(&b, &lds[1][(j * 16 + (lane & 15)) * LD + (lane >> 4) * 32], 32);
            acc[j] = mfma_f8<T>(a, b, acc[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + j * 16 + (lane & 15);
        if (n >= g.N) continue;
        const float sb = g.b_scale ? g.b_scale[n] : 1.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t m = m0 + wave * 16 + (lane >> 4) * 4 + i;
            if (m >= g.M) continue;
            const float sa = g.a_scale ? g.a_scale[m] : 1.f;
            ((T*)g.c)[m * g.ldc + n] = from_f<T>(acc[j][i] * sa * sb);
        }
    }
}

}  // namespace

int64_t gemm_f8_workspace(int64_t M, int32_t N, int32_t K) { return 0; }

fo_status launch_gemm_f8(int32_t dtype, const GemmF8Args& g, void* ws, hipStream_t s) {
    const dim3 grid = grid_of(cdiv(g.M, 64) * cdiv(g.N, 64));
    if (dtype == FO_DT_BF16) gemm_f8_any_kernel<bf16_t><<<grid, 256, 0, s>>>(g);
    else gemm_f8_any_kernel<float><<<grid, 256, 0, s>>>(g);
    FO_LAUNCHED();
    return FO_OK;
}

}  // namespace fo
