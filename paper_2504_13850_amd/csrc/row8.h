// Rows of eight elements a thread: loads and stores for the operators that pass
// over matrices, and the sums of a matrix's columns over partial rows.
#pragma once

#include "ops.h"

namespace fo {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes at an address that only its elements are aligned to: one load or store, the hardware takes any address.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// Eight values of a row.  NT: past the caches, for what a 256 MB last-level cache would not keep.
template <class T, bool NT>
struct Eight {
    static constexpr int PIECES = sizeof(T) / 2, PER = 8 / PIECES;  // of 16 bytes
    u32x4 u[PIECES];
    // The first n of eight; vec: all of them.  `step`: where the second four of 32-bit values begin.
    __device__ __forceinline__ void load(const T* p, int n, bool vec, int step = 4) {
        if (vec) {
#pragma unroll
            for (int c = 0; c < PIECES; ++c) {
                const u32x4_any* q = reinterpret_cast<const u32x4_any*>(p + c * step);
                u[c] = NT ? __builtin_nontemporal_load(q) : *q;
            }
        } else {
            T v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e + (e / PER) * (step - 4)] : T(0);
            __builtin_memcpy(u, v, sizeof(u));
        }
    }
    // Eight of a row of `cols` from c0 on; of the row's end its last eight, which fit() moves to their place once they are
    // there.  So no thread branches to single elements and waits for them between one operand's loads and the next's
    // (RMS norm forward, 5247 rows of 6845 bf16 81 us so, 72 as here).  fit: n = cols - c0, eight at most.
    __device__ __forceinline__ void load_row(const T* row, int c0, int cols) {
        if (cols >= 8) load(row + min(c0, cols - 8), 8, true);
        else load(row, cols, false);
    }
    __device__ __forceinline__ void fit(int n, int cols) {
        if (n >= 8 || n <= 0 || cols < 8) return;
        uint32_t w[4 * PIECES + 4] = {};  // zeros come in
        __builtin_memcpy(w, u, sizeof(u));
        const int k = 8 - n;
#pragma unroll
        for (int m = 4; m; m /= 2) {
            if (!(k & m)) continue;
#pragma unroll
            for (int i = 0; i < 4 * PIECES; ++i)
                w[i] = m * PIECES >= 2 ? w[i + m * PIECES / 2] : w[i] >> 16 | w[i + 1] << 16;
        }
        __builtin_memcpy(u, w, sizeof(u));
    }
    __device__ __forceinline__ float at(int e) const {
        T v[8];
        __builtin_memcpy(v, u, sizeof(u));
        return to_f(v[e]);
    }
    __device__ __forceinline__ void put(int place, T x) {
        T v[8];
        __builtin_memcpy(v, u, sizeof(u));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e == place ? x : v[e];
        __builtin_memcpy(u, v, sizeof(u));
    }
    __device__ __forceinline__ static void store(T* p, const float* x, int n, bool vec, int step = 4) {
        u32x4 w[PIECES];
        if constexpr (sizeof(T) == 2)
            w[0] = u32x4{f2bf2(x[0], x[1]), f2bf2(x[2], x[3]), f2bf2(x[4], x[5]), f2bf2(x[6], x[7])};
        else
            __builtin_memcpy(w, x, sizeof(w));
        if (vec) {
#pragma unroll
            for (int c = 0; c < PIECES; ++c) {
                u32x4_any* q = reinterpret_cast<u32x4_any*>(p + c * step);
                if (NT) __builtin_nontemporal_store(w[c], q);
                else *q = w[c];
            }
        } else {
            T v[8];
            __builtin_memcpy(v, w, sizeof(w));
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) p[e + (e / PER) * (step - 4)] = v[e];
        }
    }
};

// Whether every row of a matrix starts 16-byte aligned.
template <class T>
bool vec_rows(const void* p, int64_t ld) {
    return ((uintptr_t)p & 15) == 0 && ld * (int64_t)sizeof(T) % 16 == 0;
}

// 32 columns a workgroup, the parts dealt to 32 rows of threads and joined in order.
template <class T>
__global__ void __launch_bounds__(1024) column_sums_kernel(const float* __restrict__ part, int parts, int cols,
                                                          T* __restrict__ out) {
    __shared__ float sums[32][32];
    const int t = threadIdx.x & 31, y = threadIdx.x >> 5, c = block_of() * 32 + t;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (int p = y; p < parts; p += 32) s += part[(int64_t)p * cols + c];
    }
    sums[y][t] = s;
    __syncthreads();
    if (y || c >= cols) return;
    for (int k = 1; k < 32; ++k) s += sums[k][t];
    out[c] = from_f<T>(s);
}

// out[c] = the sum of part[parts][cols] over the parts.
template <class T>
fo_status column_sums(const float* part, int parts, int cols, T* out, hipStream_t s) {
    column_sums_kernel<T><<<grid_of(cdiv(cols, 32)), 1024, 0, s>>>(part, parts, cols, out);
    FO_LAUNCHED();
    return FO_OK;
}

// ------------------------------------------------------------------ sums and maxima over a team of threads
// TPR threads of a workgroup share a row: a power of two up to a wave, or the whole
// workgroup, whose waves meet in `lds` (two floats for each).  Every thread gets the result.
struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
template <int TPR, class Op>
__device__ __forceinline__ float team(float v, float* lds, Op op) {
#pragma unroll
    for (int m = 1; m < (TPR < 64 ? TPR : 64); m *= 2) v = op(v, __shfl_xor(v, m));
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[threadIdx.x & (TPR / 64 - 1)];
#pragma unroll
        for (int m = 1; m < TPR / 64; m *= 2) v = op(v, __shfl_xor(v, m));
    }
    return v;
}

}  // namespace fo
