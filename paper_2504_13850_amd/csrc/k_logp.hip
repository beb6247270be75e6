// Log probabilities of target tokens, their gradient, and both in one pass.
//
// Bound by HBM: the logits are read once (forward), read and written once
// (gradient; cross-entropy where a row lies in the registers of a workgroup).
// Running maximum and sum leave the target's term out: with it, 1 - p and log p
// lose all but a few bits where p is near 1.
#include <algorithm>

#include "lm.h"
#include "row8.h"

namespace fo {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float exp_(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Maximum and sum of exp(z - maximum) over some terms, by raw logits: z = scale raw, scale > 0.
struct Part {
    float m, s;
};
// exp(scale raw - scale m) where m may be -infinity (no term, or none but -infinity).
__device__ __forceinline__ float term(float raw, float scale, float m) {
    return exp_(m == -INFINITY ? -INFINITY : (raw - m) * scale);
}
__device__ __forceinline__ Part join(Part a, Part b, float scale) {
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return {m, a.s + b.s};  // 0, or NaN
    return {m, a.s * exp_((a.m - m) * scale) + b.s * exp_((b.m - m) * scale)};
}
template <int TPR>
__device__ __forceinline__ Part team_join(Part p, float scale, Part* lds) {
#pragma unroll
    for (int m = 1; m < (TPR < 64 ? TPR : 64); m *= 2)
        p = join(p, Part{__shfl_xor(p.m, m), __shfl_xor(p.s, m)}, scale);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = p;
        __syncthreads();
        p = lds[threadIdx.x & (TPR / 64 - 1)];
#pragma unroll
        for (int m = 1; m < TPR / 64; m *= 2) p = join(p, Part{__shfl_xor(p.m, m), __shfl_xor(p.s, m)}, scale);
    }
    return p;
}

// logp and lse from the other terms and the target's logit; all: what the row's terms are divided by, as {m, 1 / s},
// and the target's 1 - p.
struct Row {
    float logp, lse, m, inv, rest;
};
__device__ __forceinline__ Row row_of(Part p, float zt, float scale) {
    Row r;
    r.m = fmaxf(p.m, zt);
    if (p.s != p.s || zt != zt) r.m = NAN;
    const float others = p.s * term(p.m, scale, r.m), own = term(zt, scale, r.m), all = others + own;
    r.inv = 1.f / all;
    r.rest = others * r.inv;
    r.logp = zt >= p.m ? -log1pf(others) : (zt - r.m) * scale - logf(all);
    r.lse = r.m * scale + logf(all);
    if (r.m == -INFINITY) {
        r.logp = r.lse = -INFINITY;
        r.rest = 0.f;
    }
    return r;
}

// The chunk's sum and maximum, the target's element (place t, if it lies here) left out.
template <class T>
__device__ __forceinline__ void add_chunk(const Eight<T, false>& x, int n, int t, float scale, Part& p) {
    float v[8], m = p.m;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = e < n && e != t ? x.at(e) : -INFINITY;
        m = fmaxf(m, v[e]);
    }
    float s = p.s * term(p.m, scale, m);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[e] != v[e] ? v[e] : term(v[e], scale, m);
    p = {m, s};
}

constexpr int FLY = 4;  // chunks of a thread in flight

// SLICED: workgroup (row, slice) leaves its part in `part`; else a team of TPR threads has a row.
template <class T, int TPR, bool SLICED>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) logp_fwd_kernel(LogpArgs a, Part* __restrict__ part, int slices) {
    constexpr int THREADS = TPR < 256 ? 256 : TPR, RPW = THREADS / TPR;
    __shared__ Part lds[TPR / 64 + 1];
    const int t = threadIdx.x % TPR;
    const int64_t id = block_of(), row = SLICED ? id / slices : id * RPW + threadIdx.x / TPR;
    if (row >= a.rows) return;
    const int target = a.targets[row];
    const bool there = target >= 0 && target < a.vocab;
    Part p = {-INFINITY, 0.f};
    if (there) {
        const T* x = (const T*)a.logits + row * a.ld;
        const int chunks = (a.vocab + 7) / 8, each = SLICED ? (chunks + slices - 1) / slices : chunks;
        const int first = SLICED ? (int)(id % slices) * each : 0, last = min(chunks, first + each);
        for (int c = first + t; c < last; c += FLY * TPR) {
            Eight<T, false> u[FLY];
#pragma unroll
            for (int k = 0; k < FLY; ++k) {
                const int c0 = (c + k * TPR) * 8, n = min(8, a.vocab - c0);
                if (c + k * TPR < last) u[k].load(x + c0, n, n == 8);
            }
#pragma unroll
            for (int k = 0; k < FLY; ++k) {
                const int c0 = (c + k * TPR) * 8;
                if (c + k * TPR < last) add_chunk(u[k], a.vocab - c0, target - c0, a.scale, p);
            }
        }
        p = team_join<TPR>(p, a.scale, lds);
    }
    if (t) return;
    if (SLICED) {
        part[id] = p;
        return;
    }
    Row r = {};
    if (there) r = row_of(p, to_f(((const T*)a.logits)[row * a.ld + target]), a.scale);
    a.logp[row] = r.logp;
    if (a.lse) a.lse[row] = r.lse;
}

// A wave a row: the slices in order of their lanes.
template <class T>
__global__ void __launch_bounds__(64) logp_join_kernel(LogpArgs a, const Part* __restrict__ part, int slices) {
    const int64_t row = block_of();
    if (row >= a.rows) return;
    const int target = a.targets[row];
    Row r = {};
    if (target >= 0 && target < a.vocab) {
        Part p = {-INFINITY, 0.f};
        for (int k = threadIdx.x; k < slices; k += 64) p = join(p, part[row * slices + k], a.scale);
        p = team_join<64>(p, a.scale, nullptr);
        r = row_of(p, to_f(((const T*)a.logits)[row * a.ld + target]), a.scale);
    }
    if (threadIdx.x) return;
    a.logp[row] = r.logp;
    if (a.lse) a.lse[row] = r.lse;
}

// XENT: weight is minus the gradient by logp, and logp becomes the loss.
template <class T, bool XENT>
__global__ void __launch_bounds__(256) logp_bwd_kernel(LogpArgs a, float* __restrict__ loss) {
    const int64_t row = block_of();
    if (row >= a.rows) return;
    const int target = a.targets[row], chunks = (a.vocab + 7) / 8;
    const bool there = target >= 0 && target < a.vocab;
    const float logp = a.logp[row], lse = a.lse[row];
    if (XENT && blockIdx.z == 0 && threadIdx.x == 0) loss[row] = there ? -logp : 0.f;
    const T* x = (const T*)a.logits + row * a.ld;
    T* y = (T*)a.dlogits + row * a.dlogits_ld;
    const bool none = !there || lse == -INFINITY;
    const float g = none ? 0.f : (XENT ? -a.weight[row] : a.weight[row]) * a.scale;
    const float own = none ? 0.f : g * -expm1f(logp);
    for (int c = blockIdx.z * 256 + threadIdx.x; c < chunks; c += gridDim.z * 256) {
        const int c0 = c * 8, n = min(8, a.vocab - c0);
        float d[8] = {};
        if (!none) {
            Eight<T, false> u;
            u.load(x + c0, n, n == 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[e] = -g * exp_(fmaf(u.at(e), a.scale, -lse));
                if (c0 + e == target) d[e] = own;
            }
        }
        Eight<T, false>::store(y + c0, d, n, n == 8);
    }
}

// Cross-entropy with the row in registers: maximum and sum of what is held, then the gradient from it.
template <class T, int TPR, int NC>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) xent_kernel(LogpArgs a) {
    constexpr int THREADS = TPR < 256 ? 256 : TPR, RPW = THREADS / TPR;
    __shared__ float lds[32];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)block_of() * RPW + threadIdx.x / TPR;
    if (row >= a.rows) return;
    const int target = a.targets[row];
    T* y = (T*)a.dlogits + row * a.dlogits_ld;
    if (target < 0 || target >= a.vocab) {
        const float zero[8] = {};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int c0 = (t + c * TPR) * 8, n = min(8, a.vocab - c0);
            if (n > 0) Eight<T, false>::store(y + c0, zero, n, n == 8);
        }
        if (t == 0) a.logp[row] = 0.f;
        return;
    }
    const T* x = (const T*)a.logits + row * a.ld;
    const float zt = to_f(x[target]);
    Eight<T, false> u[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int c0 = (t + c * TPR) * 8, n = min(8, a.vocab - c0);
        u[c].load(x + c0, n, n == 8);
    }
    float m = -INFINITY, s = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int c0 = (t + c * TPR) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c0 + e < a.vocab && c0 + e != target) m = fmaxf(m, u[c].at(e));
    }
    m = team<TPR>(m, lds, Max());
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int c0 = (t + c * TPR) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = u[c].at(e);
            if (c0 + e < a.vocab && c0 + e != target) s += v != v ? v : term(v, a.scale, m);
        }
    }
    s = team<TPR>(s, lds + 16, Add());  // every thread has read its logits: dlogits may lie over them
    const Row r = row_of(Part{m, s}, zt, a.scale);
    const bool none = r.m == -INFINITY;
    const float g = none ? 0.f : a.weight[row] * a.scale, k = g * r.inv;
    if (t == 0) a.logp[row] = -r.logp;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int c0 = (t + c * TPR) * 8, n = min(8, a.vocab - c0);
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            d[e] = none ? 0.f : k * term(u[c].at(e), a.scale, r.m);
            if (c0 + e == target) d[e] = -g * r.rest;
        }
        if (n > 0) Eight<T, false>::store(y + c0, d, n, n == 8);
    }
}

// Workgroups along a row so that few long rows fill the chip: about two workgroups a CU, 4096 logits each or more.
constexpr int64_t kWgs = 512;
int slices_of(int64_t rows, int32_t vocab) {
    if (rows >= kWgs || rows < 1) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(kWgs / rows, vocab / 4096));
}
int64_t part_bytes(int64_t rows, int32_t vocab) {
    const int n = slices_of(rows, vocab);
    return n > 1 ? cdiv(rows * n * (int64_t)sizeof(Part), 16) * 16 : 0;
}

template <class T>
fo_status fwd(const LogpArgs& a, void* ws, hipStream_t s) {
    const int n = slices_of(a.rows, a.vocab);
    if (n > 1) {
        logp_fwd_kernel<T, 256, true><<<grid_of(a.rows * n), 256, 0, s>>>(a, (Part*)ws, n);
        FO_LAUNCHED();
        logp_join_kernel<T><<<grid_of(a.rows), 64, 0, s>>>(a, (const Part*)ws, n);
    } else if (a.vocab <= 2048) {
        logp_fwd_kernel<T, 64, false><<<grid_of(cdiv(a.rows, 4)), 256, 0, s>>>(a, nullptr, 1);
    } else {
        logp_fwd_kernel<T, 256, false><<<grid_of(a.rows), 256, 0, s>>>(a, nullptr, 1);
    }
    FO_LAUNCHED();
    return FO_OK;
}

// Workgroups along the vocabulary: one for each 16384 logits of a row (2048 to a thread would be a long tail).
dim3 bwd_grid(const LogpArgs& a) {
    dim3 g = grid_of(a.rows);
    g.z = (unsigned)std::min<int64_t>(cdiv(a.vocab, 16384), 65535);
    return g;
}

template <class T>
fo_status bwd(const LogpArgs& a, hipStream_t s) {
    logp_bwd_kernel<T, false><<<bwd_grid(a), 256, 0, s>>>(a, nullptr);
    FO_LAUNCHED();
    return FO_OK;
}

// Rows that a workgroup holds in registers: 8 NC logits a thread.  A few rows longer than one workgroup's share go
// through the sliced forward pass and the gradient.
bool held(int64_t rows, int32_t vocab, int32_t size) {
    return slices_of(rows, vocab) == 1 && (int64_t)vocab * size <= 262144;
}

template <class T>
fo_status xent(const LogpArgs& a, void* ws, hipStream_t s) {
    if (!held(a.rows, a.vocab, sizeof(T))) {
        LogpArgs b = a;
        b.logp = (float*)((char*)ws + part_bytes(a.rows, a.vocab));
        b.lse = b.logp + a.rows;
        const fo_status st = fwd<T>(b, ws, s);
        if (st != FO_OK) return st;
        logp_bwd_kernel<T, true><<<bwd_grid(b), 256, 0, s>>>(b, a.logp);
    } else if (a.vocab <= 1024) {
        xent_kernel<T, 64, 2><<<grid_of(cdiv(a.rows, 4)), 256, 0, s>>>(a);
    } else if (a.vocab <= 8192) {
        xent_kernel<T, 256, 4><<<grid_of(a.rows), 256, 0, s>>>(a);
    } else if (a.vocab <= 32768) {
        xent_kernel<T, 1024, 4><<<grid_of(a.rows), 1024, 0, s>>>(a);
    } else if (a.vocab <= 65536) {
        xent_kernel<T, 1024, 8><<<grid_of(a.rows), 1024, 0, s>>>(a);
    } else if constexpr (sizeof(T) == 2) {
        xent_kernel<T, 1024, 16><<<grid_of(a.rows), 1024, 0, s>>>(a);
    }
    FO_LAUNCHED();
    return FO_OK;
}

}  // namespace

int64_t logp_workspace(int64_t rows, int32_t vocab) {
    // the type is not known here: cross-entropy's copy of logp and lse where either type needs it
    return part_bytes(rows, vocab) + (held(rows, vocab, 4) ? 0 : cdiv(rows * 8, 16) * 16);
}

fo_status launch_logp_fwd(int32_t dtype, const LogpArgs& a, void* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? fwd<bf16_t>(a, ws, s) : fwd<float>(a, ws, s);
}

fo_status launch_logp_bwd(int32_t dtype, const LogpArgs& a, hipStream_t s) {
    return dtype == FO_DT_BF16 ? bwd<bf16_t>(a, s) : bwd<float>(a, s);
}

fo_status launch_xent(int32_t dtype, const LogpArgs& a, void* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? xent<bf16_t>(a, ws, s) : xent<float>(a, ws, s);
}

}  // namespace fo
