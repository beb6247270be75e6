// Shared by the transformer operators (fedoptima_ops.h): argument records,
// launchers, and the dropout generator.
#pragma once

#include "../../include/fedoptima_ops.h"
#include "common.h"

namespace fo {

// p to the nearest multiple of 2^-16: an element is dropped when its 16-bit number is below the result.
inline uint32_t drop_threshold(float p) {
    const double t = (double)p * 65536.0 + 0.5;
    return t >= 65535.0 ? 65535u : (uint32_t)t;
}

// A grid of n workgroups in two dimensions: one dimension holds 2^32 threads, and a launch
// of more wraps round without an error.  Workgroups past n, in the last row, have no work.
constexpr int kGridBits = 20;  // workgroups of up to 1024 threads
inline dim3 grid_of(int64_t n) {
    return n <= int64_t(1) << kGridBits ? dim3((unsigned)n)
                                        : dim3(1u << kGridBits, (unsigned)cdiv(n, int64_t(1) << kGridBits));
}
__device__ __forceinline__ int block_of() { return (int)((blockIdx.y << kGridBits) + blockIdx.x); }

// Philox 4x32 (Salmon et al., 2011): four words out of four counter words and a
// two-word key.  Seven rounds, the fewest that the paper finds to pass every
// TestU01 battery; its usual ten cost 3/7 more of a pass that is bound by its
// 32-bit multiplies wherever it sits inside the attention.
__device__ __forceinline__ uint4 philox7(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                         uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}
// Number e (0..7) of a call's eight 16-bit numbers, low halves first.
__device__ __forceinline__ uint32_t half_of(const uint4& w, int e) {
    const uint32_t x = e < 4 ? (e < 2 ? w.x : w.y) : (e < 6 ? w.z : w.w);
    return (e & 1) ? x >> 16 : x & 0xFFFFu;
}

template <class T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<bf16_t>(bf16_t x) { return bf2f(x); }
template <class T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ bf16_t from_f<bf16_t>(float x) { return f2bf(x); }

// ------------------------------------------------------------------ attention
struct AttnArgs {
    fo_attn a;
    const void *q, *k, *v;
    void* out;
    float* lse;
    uint32_t thr;      // dropout threshold, 0: none
    float keep_scale;  // 1 / (1 - thr / 65536)
    // backward
    const void* dout;
    void *dq, *dk, *dv, *dtable;
    float* delta;      // [heads][q_rows]
    float* hist;       // sums of the bias gradient by distance
};

// Sequence b's rows, clamped to what there is.
struct Span {
    int q0, nq, k0, nk;
};
__device__ __forceinline__ Span span_of(const fo_attn& a, int b) {
    Span s;
    const int64_t q0 = min(max((int64_t)a.q_begin[b], (int64_t)0), a.q_rows);
    const int64_t q1 = min(min(max((int64_t)a.q_end[b], q0), a.q_rows), q0 + a.max_q);
    const int64_t k0 = min(max((int64_t)a.k_begin[b], (int64_t)0), a.k_rows);
    const int64_t k1 = min(min(max((int64_t)a.k_end[b], k0), a.k_rows), k0 + a.max_k);
    s.q0 = (int)q0; s.nq = (int)(q1 - q0); s.k0 = (int)k0; s.nk = (int)(k1 - k0);
    return s;
}

int64_t attn_workspace(const fo_attn& a, bool backward);
fo_status launch_attn_op_fwd(const AttnArgs& x, void* ws, hipStream_t s);
fo_status launch_attn_op_bwd(AttnArgs& x, void* ws, hipStream_t s);

// ------------------------------------------------------------------ dropout
struct DropArgs {
    int64_t rows;
    int32_t cols;
    const void *x, *bias, *res;
    int64_t x_ld, res_ld, y_ld;
    void* y;
    uint32_t thr, k0, k1, offset;
    float keep_scale;
};
fo_status launch_dropout_fwd(int32_t dtype, const DropArgs& d, hipStream_t s);
int64_t dropout_workspace(int64_t rows, int32_t cols);
fo_status launch_dropout_bwd(int32_t dtype, const DropArgs& d, void* dbias, float* ws, hipStream_t s);

}  // namespace fo
