// Log probabilities of target tokens, their gradient, and both in one pass.
//
// Bound by HBM: the logits are read once (forward), read and written once
// (gradient; cross-entropy where a row lies in the registers of a workgroup).
// 8192 rows of 32000 bf16, a tenth without a target, cross-entropy: 167 us, 6.0
// TB/s; forward and gradient of 5565 such rows 178 us, 6.0 TB/s (a copy of a GiB
// runs at 5.15).  Some ten instructions a logit and pass, the exponential at a
// quarter of the rate: half of that time, hidden where loads are not held up.
// Running maximum and sum leave the target's term out: with it, 1 - p and log p
// lose all but a few bits where p is near 1.
#include <algorithm>

#include "lm.h"
#include "row8.h"

namespace fo {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLeast = -3.402823466e38f;

// Maximum and sum of exp(scale (raw - maximum)) over some terms by their raw logits.  The maximum starts from the least
// finite number and not from -infinity, so that no difference of infinities arises: a sum of 0 has no terms, or none
// but -infinity.  A NaN goes by the maximum and into the sum.
struct Part {
    float m, s;
};
constexpr Part kNone = {kLeast, 0.f};
// scale log2(e) in two parts: with the first alone every term of a row is off the same way, log sum exp by some 1e-7,
// and a loss over whole answers adds that up.  Cross-entropy, whose rows nothing adds up before they are rounded, does
// with the first (167 us, 177 with both).
struct Factor {
    float hi, lo;
};
__device__ __forceinline__ Factor factor(float scale) {
    const double c = (double)scale * 1.4426950408889634;
    return {(float)c, (float)(c - (double)(float)c)};
}
__device__ __forceinline__ float term(float raw, float m, Factor c) {
    const float x = raw - m;
    return __builtin_amdgcn_exp2f(fmaf(x, c.hi, fmaxf(x, -1e4f) * c.lo));
}
__device__ __forceinline__ float term(float raw, float m, float c) { return __builtin_amdgcn_exp2f((raw - m) * c); }
__device__ __forceinline__ Part join(Part a, Part b, Factor c) {
    const float m = fmaxf(a.m, b.m);
    return {m, a.s * term(a.m, m, c) + b.s * term(b.m, m, c)};
}
template <int TPR>
__device__ __forceinline__ Part team_join(Part p, Factor c, Part* lds) {
#pragma unroll
    for (int m = 1; m < (TPR < 64 ? TPR : 64); m *= 2)
        p = join(p, Part{__shfl_xor(p.m, m), __shfl_xor(p.s, m)}, c);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = p;
        __syncthreads();
        p = lds[threadIdx.x & (TPR / 64 - 1)];
#pragma unroll
        for (int m = 1; m < TPR / 64; m *= 2) p = join(p, Part{__shfl_xor(p.m, m), __shfl_xor(p.s, m)}, c);
    }
    return p;
}

// What a row's gradient needs of the other terms and the target's logit zt: the maximum, 1 / the sum of all terms, and
// the other terms' share, which is the target's 1 - p.
struct Row {
    float m, inv, rest;
    bool none;  // every term is 0
};
__device__ __forceinline__ Row row_of(Part p, float zt, Factor c) {
    Row r;
    r.m = fmaxf(p.m, zt);
    const float others = p.s * term(p.m, r.m, c), all = others + term(zt, r.m, c);
    r.none = all == 0.f;
    r.inv = 1.f / all;
    r.rest = r.none ? 0.f : others * r.inv;
    return r;
}
// logp and lse, in 64 bits: a loss over whole answers adds up what they are off by.
__device__ __forceinline__ float2 logs_of(Part p, float zt, float scale) {
    const Factor c = factor(scale);
    const float m = fmaxf(p.m, zt);
    const double others = (double)p.s * term(p.m, m, c), all = others + term(zt, m, c);
    if (all == 0.0) return make_float2(-INFINITY, -INFINITY);
    const double away = ((double)zt - m) * scale;
    return make_float2((float)(zt >= p.m ? -log1p(others) : away - log(all)), (float)((double)m * scale + log(all)));
}

// -infinity in the target's place, if it lies in this chunk.
template <class T>
__device__ __forceinline__ void leave_out(Eight<T, false>& x, int chunk, int target) {
    if (target >> 3 == chunk) x.put(target & 7, from_f<T>(-INFINITY));
}
// What a row has past its last whole chunk, -infinity after it.
template <class T>
__device__ __forceinline__ Eight<T, false> last_chunk(const T* row, int vocab) {
    const int c0 = vocab & ~7, n = vocab & 7;
    Eight<T, false> x;
    x.load(row + c0, n, false);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e >= n) x.put(e, from_f<T>(-INFINITY));
    return x;
}
template <class T>
__device__ __forceinline__ void add_chunk(const Eight<T, false>& x, Factor c, Part& p) {
    float m = p.m;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, x.at(e));
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = term(x.at(e), m, c);
#pragma unroll
    for (int k = 4; k; k /= 2)  // one addition a chunk to what a thread has: a few threads' rows are as exact as many's
#pragma unroll
        for (int e = 0; e < k; ++e) s[e] += s[e + k];
    p = {m, fmaf(p.s, term(p.m, m, c), s[0])};
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
    const Factor c2 = factor(a.scale);
    Part p = kNone;
    float zt = 0.f;
    if (there) {
        const T* x = (const T*)a.logits + row * a.ld;
        if (!SLICED) zt = to_f(x[target]);
        const int chunks = a.vocab / 8, each = SLICED ? (chunks + slices - 1) / slices : chunks;
        const int slice = SLICED ? (int)(id % slices) : 0, first = min(chunks, slice * each), last = min(chunks, first + each);
        int c = first + t;
        for (; c + (FLY - 1) * TPR < last; c += FLY * TPR) {  // the loads first, without a branch between them
            Eight<T, false> u[FLY];
#pragma unroll
            for (int k = 0; k < FLY; ++k) u[k].load(x + (c + k * TPR) * 8, 8, true);
#pragma unroll
            for (int k = 0; k < FLY; ++k) {
                leave_out(u[k], c + k * TPR, target);
                add_chunk(u[k], c2, p);
            }
        }
        for (; c < last; c += TPR) {
            Eight<T, false> u;
            u.load(x + c * 8, 8, true);
            leave_out(u, c, target);
            add_chunk(u, c2, p);
        }
        if (a.vocab % 8 && t == 0 && slice == slices - 1) {
            Eight<T, false> u = last_chunk(x, a.vocab);
            leave_out(u, chunks, target);
            add_chunk(u, c2, p);
        }
        p = team_join<TPR>(p, c2, lds);
    }
    if (t) return;
    if (SLICED) {
        part[id] = p;
        return;
    }
    float2 r = make_float2(0.f, 0.f);
    if (there) r = logs_of(p, zt, a.scale);
    a.logp[row] = r.x;
    if (a.lse) a.lse[row] = r.y;
}

// A wave a row: the slices in order of their lanes.
template <class T>
__global__ void __launch_bounds__(64) logp_join_kernel(LogpArgs a, const Part* __restrict__ part, int slices) {
    const int64_t row = block_of();
    if (row >= a.rows) return;
    const int target = a.targets[row];
    float2 r = make_float2(0.f, 0.f);
    if (target >= 0 && target < a.vocab) {
        const Factor c = factor(a.scale);
        const float zt = to_f(((const T*)a.logits)[row * a.ld + target]);
        Part p = kNone;
        for (int k = threadIdx.x; k < slices; k += 64) p = join(p, part[row * slices + k], c);
        p = team_join<64>(p, c, nullptr);
        r = logs_of(p, zt, a.scale);
    }
    if (threadIdx.x) return;
    a.logp[row] = r.x;
    if (a.lse) a.lse[row] = r.y;
}

// Which of a row's chunks a launch of the gradient writes.  Over the logits themselves no other workgroup may lose the
// target's logit before it has read it: all but its chunk in one launch, that chunk in the next.
enum Chunks { kAll, kOthers, kTargets };

// scale (u - from) + at = z - lse.  By lse every term is off by what lse lost when it was rounded, up to |lse| 2^-24 of
// itself (logits around 100000: 3e-3); by the target's logit and logp, whose difference lse is, up to 2 |logp| 2^-24 where
// the terms are large.  No lse is too large for that, nor infinite where scale takes the maximum past fp32.
struct Origin {
    float from, at;
};
__device__ __forceinline__ Origin origin(float zt, float logp, float lse) {
    return 2.f * fabsf(logp) < fabsf(lse) ? Origin{zt, logp} : Origin{0.f, -lse};
}

// XENT: weight is minus the gradient by logp, and logp becomes the loss.  NT: past the caches.
template <class T, int TPR, bool XENT, bool NT>
__global__ void __launch_bounds__(256) logp_bwd_kernel(LogpArgs a, Chunks which, float* __restrict__ loss) {
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)block_of() * (256 / TPR) + threadIdx.x / TPR;
    if (row >= a.rows) return;
    const int target = a.targets[row], chunks = (a.vocab + 7) / 8;
    const bool there = target >= 0 && target < a.vocab;
    const float logp = a.logp[row], lse = a.lse[row];
    const T* x = (const T*)a.logits + row * a.ld;
    T* y = (T*)a.dlogits + row * a.dlogits_ld;
    const float zt = there ? to_f(x[target]) : 0.f;
    if (TPR > 64) __syncthreads();  // every wave has read it: dlogits may lie over the logits
    if (XENT && which != kTargets && blockIdx.z == 0 && t == 0) loss[row] = there ? -logp : 0.f;
    const bool none = !there || lse == -INFINITY;
    const float g = none ? 0.f : (XENT ? -a.weight[row] : a.weight[row]) * a.scale;
    const float own = none ? 0.f : g * -expm1f(logp);
    const Origin o = origin(zt, logp, lse);
    const int mine = there ? target >> 3 : -1;
    if (which == kTargets && (t || !there)) return;
    const int first = which == kTargets ? mine : (int)blockIdx.z * TPR + t, last = which == kTargets ? mine + 1 : chunks;
    for (int c = first; c < last; c += gridDim.z * TPR) {
        if (which == kOthers && c == mine) continue;
        const int c0 = c * 8, n = min(8, a.vocab - c0);
        float d[8] = {};
        if (!none) {
            Eight<T, NT> u;
            u.load(x + c0, n, n == 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[e] = -g * __builtin_amdgcn_exp2f(fmaf(u.at(e) - o.from, a.scale, o.at) * kLog2e);
                if (c0 + e == target) d[e] = own;
            }
        }
        Eight<T, NT>::store(y + c0, d, n, n == 8);
    }
}

// Cross-entropy with the row in registers: maximum and sum of what is held, then the gradient from it.  64 registers,
// two workgroups of 1024 on a CU, where a thread holds four chunks: one works while the other waits (8192 rows of 32000
// bf16 177 us, 224 with one).  Left alone the compiler takes 70 for four chunks, 56 for three, which fits without being
// told, and 83 for six, which never would.  NT: the gradient past the caches.
template <class T, int TPR, int NC, bool NT>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR, TPR * NC == 4096 ? 8 : 4) xent_kernel(LogpArgs a) {
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
            if (n > 0) Eight<T, NT>::store(y + c0, zero, n, n == 8);
        }
        if (t == 0) a.logp[row] = 0.f;
        return;
    }
    const T* x = (const T*)a.logits + row * a.ld;
    const float zt = to_f(x[target]);
    const Factor c2 = factor(a.scale);
    const int chunks = a.vocab / 8;  // one at least
    Eight<T, false> u[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) u[c].load(x + min(t + c * TPR, chunks - 1) * 8, 8, true);
    Part p = kNone;
#pragma unroll
    for (int c = 0; c < NC; ++c) {  // past the whole chunks: the row's end, or nothing
        if (t + c * TPR >= chunks) u[c] = last_chunk(x, t + c * TPR == chunks ? a.vocab : 0);
        leave_out(u[c], t + c * TPR, target);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) p.m = fmaxf(p.m, u[c].at(e));
    p.m = team<TPR>(p.m, lds, Max());
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) p.s += term(u[c].at(e), p.m, c2.hi);
    p.s = team<TPR>(p.s, lds + 16, Add());  // every thread has read its logits: dlogits may lie over them
    const Row r = row_of(p, zt, c2);
    const float g = r.none ? 0.f : a.weight[row] * a.scale, k = r.none ? 0.f : g * r.inv;
    if (t == 0) a.logp[row] = -logs_of(p, zt, a.scale).x;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int c0 = (t + c * TPR) * 8, n = min(8, a.vocab - c0);
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = k * term(u[c].at(e), r.m, c2.hi);
        if (target >> 3 == t + c * TPR)
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = e == (target & 7) ? -g * r.rest : d[e];
        if (n > 0) Eight<T, NT>::store(y + c0, d, n, n == 8);
    }
}

// Workgroups along a row so that few long rows fill the chip: about two workgroups a CU, 4096 logits each or more.  Up
// to 65536 logits one workgroup of 1024 threads a row is as fast in one launch (60 rows of 32000 bf16 8.0 us, 8.2 in
// two; 5 rows of 128000 fp32 12.7 and 7.7).
constexpr int64_t kWgs = 512;
constexpr int32_t kOneWg = 65536;
int slices_of(int64_t rows, int32_t vocab) {
    if (rows >= kWgs || rows < 1 || vocab <= kOneWg) return 1;
    return (int)std::min<int64_t>(kWgs / rows, vocab / 4096);
}
int64_t part_bytes(int64_t rows, int32_t vocab) {
    const int n = slices_of(rows, vocab);
    return n > 1 ? cdiv(rows * n * (int64_t)sizeof(Part), 16) * 16 : 0;
}

template <class T, int TPR>
void launch_fwd(const LogpArgs& a, hipStream_t s) {
    constexpr int THREADS = TPR < 256 ? 256 : TPR;
    logp_fwd_kernel<T, TPR, false><<<grid_of(cdiv(a.rows, THREADS / TPR)), THREADS, 0, s>>>(a, nullptr, 1);
}
// Short rows take few threads, for the logarithms in 64 bits take a wave as long whether one lane or 16 have a row
// (bf16, 165000 rows of 128: 4 threads 17 us, 16 30, 64 108; 12000 of 4096: 16 threads 22, 64 24, 256 33), unless there
// are too few rows to fill the chip so (500 rows of 1000: 4 threads 11.0, 64 6.0).
template <class T>
fo_status fwd(const LogpArgs& a, void* ws, hipStream_t s) {
    const int n = slices_of(a.rows, a.vocab);
    const auto narrow = [&](int team, int32_t most) { return a.vocab <= (a.rows * team >= 1 << 16 ? most : 16 * team); };
    if (n > 1) {
        logp_fwd_kernel<T, 256, true><<<grid_of(a.rows * n), 256, 0, s>>>(a, (Part*)ws, n);
        FO_LAUNCHED();
        logp_join_kernel<T><<<grid_of(a.rows), 64, 0, s>>>(a, (const Part*)ws, n);
    } else if (narrow(4, 512)) launch_fwd<T, 4>(a, s);
    else if (narrow(16, 4096)) launch_fwd<T, 16>(a, s);
    else if (narrow(64, 8192)) launch_fwd<T, 64>(a, s);
    else if (a.vocab <= 8192 || a.rows >= kWgs) launch_fwd<T, 256>(a, s);
    else launch_fwd<T, 1024>(a, s);
    FO_LAUNCHED();
    return FO_OK;
}

// Logits and gradient that no cache keeps: a step of 5565 rows of 32000 bf16 takes 182 us with the gradient's loads and
// stores past the caches, 232 through them.
bool past_caches(const LogpArgs& a, int size) { return 2 * a.rows * a.vocab * size > int64_t(256) << 20; }

template <class T, int TPR, bool XENT>
void launch_bwd(const LogpArgs& a, float* loss, hipStream_t s) {
    dim3 g = grid_of(cdiv(a.rows, 256 / TPR));
    g.z = (unsigned)std::min<int64_t>(cdiv(a.vocab, 16384), 65535);  // along the vocabulary: eight chunks a thread
    const Chunks which = g.z > 1 && a.dlogits == a.logits ? kOthers : kAll;
    if (past_caches(a, sizeof(T))) logp_bwd_kernel<T, TPR, XENT, true><<<g, 256, 0, s>>>(a, which, loss);
    else logp_bwd_kernel<T, TPR, XENT, false><<<g, 256, 0, s>>>(a, which, loss);
    if (which == kOthers) logp_bwd_kernel<T, 8, XENT, false><<<grid_of(cdiv(a.rows, 32)), 256, 0, s>>>(a, kTargets, loss);
}
// A team about as wide as a row: 165000 rows of 128 bf16 16 us with 8 threads a row, 122 with 256; 50000 of 1024 34 with
// 32 and 50.
template <class T, bool XENT>
fo_status bwd(const LogpArgs& a, float* loss, hipStream_t s) {
    const int64_t bytes = a.vocab * (int64_t)sizeof(T);
    if constexpr (XENT) {  // of rows that xent_kernel does not hold
        if (bytes <= 256) launch_bwd<T, 8, XENT>(a, loss, s);
        else launch_bwd<T, 256, XENT>(a, loss, s);
    } else {
        if (bytes <= 256) launch_bwd<T, 8, XENT>(a, loss, s);
        else if (bytes <= 2048) launch_bwd<T, 32, XENT>(a, loss, s);
        else if (bytes <= 4096) launch_bwd<T, 64, XENT>(a, loss, s);
        else launch_bwd<T, 256, XENT>(a, loss, s);
    }
    FO_LAUNCHED();
    return FO_OK;
}

// Rows that a workgroup holds in registers: 8 NC logits a thread, a whole chunk at least.  Others go through the forward
// pass and the gradient.
bool held(int32_t vocab) { return vocab >= 8 && vocab <= kOneWg; }

// The narrowest of the teams and chunks that holds a row: registers that hold nothing cost (bf16, 165000 rows of 128: 4
// threads 20 us, 8 30, 64 122; 16400 rows of 9000: 512 threads with three chunks 119, with four 158, 1024 with four 282).
template <class T, int TPR, int NC, int... REST>
void launch_xent(const LogpArgs& a, hipStream_t s) {
    if constexpr (sizeof...(REST) != 0)
        if (a.vocab > TPR * NC * 8) return launch_xent<T, REST...>(a, s);
    constexpr int THREADS = TPR < 256 ? 256 : TPR;
    const dim3 g = grid_of(cdiv(a.rows, THREADS / TPR));
    if (past_caches(a, sizeof(T))) xent_kernel<T, TPR, NC, true><<<g, THREADS, 0, s>>>(a);
    else xent_kernel<T, TPR, NC, false><<<g, THREADS, 0, s>>>(a);
}

template <class T>
fo_status xent(const LogpArgs& a, void* ws, hipStream_t s) {
    if (!held(a.vocab)) {
        LogpArgs b = a;
        b.logp = (float*)((char*)ws + part_bytes(a.rows, a.vocab));
        b.lse = b.logp + a.rows;
        const fo_status st = fwd<T>(b, ws, s);
        return st != FO_OK ? st : bwd<T, true>(b, a.logp, s);
    }
    launch_xent<T, 4, 4, 8, 4, 16, 4, 32, 4, 64, 4, 256, 2, 256, 3, 256, 4, 512, 3, 512, 4, 1024, 3, 1024, 4, 1024, 6, 1024, 7,
                1024, 8>(a, s);
    FO_LAUNCHED();
    return FO_OK;
}

}  // namespace

int64_t logp_workspace(int64_t rows, int32_t vocab) {
    return part_bytes(rows, vocab) + (held(vocab) ? 0 : cdiv(rows * 8, 16) * 16);  // and fo_xent's logp and lse
}

fo_status launch_logp_fwd(int32_t dtype, const LogpArgs& a, void* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? fwd<bf16_t>(a, ws, s) : fwd<float>(a, ws, s);
}

fo_status launch_logp_bwd(int32_t dtype, const LogpArgs& a, hipStream_t s) {
    return dtype == FO_DT_BF16 ? bwd<bf16_t, false>(a, nullptr, s) : bwd<float, false>(a, nullptr, s);
}

fo_status launch_xent(int32_t dtype, const LogpArgs& a, void* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? xent<bf16_t>(a, ws, s) : xent<float>(a, ws, s);
}

}  // namespace fo
