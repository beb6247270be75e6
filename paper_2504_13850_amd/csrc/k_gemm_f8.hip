// Products of 8-bit rows with a scale each: c_mn = a_scale[m] b_scale[n] sum_k a_mk b_nk.
//
// Large ones are bound by the matrix instructions: 8192^3 in 425 to 437 us, 2510 to 2590 TFLOP/s (the library's 2730;
// the instructions alone, from registers, 4330), at a clock that the load takes down to 1.95 GHz: 2990 in the loop over
// k, 40 us for the tiles' first copies and their rows' way out.  Few rows of a are bound by reading b: 1 x 128000 x
// 4096 in 88 us, 6.0 TB/s.  Between them the latency of copies, steps and stores that follow each other.
#include <algorithm>

#include "lm.h"
#include "row8.h"

namespace fo {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Sums over 32 bytes a lane: of 16 rows and columns over 128 of k, or of 32 over 64.  Lane l holds row l % 16 (32) of
// either operand and the bytes of block l / 16 (l / 32) of k: any order of k serves, the same for both.  c: column
// l % 16 (32) of the second operand; rows 4 (l / 16) + i of the first (8 (i / 4) + 4 (l / 32) + i % 4).
//
// For results in bf16 the 8-bit matrix instruction: it adds products by eights, cutting each below 2^-13 of the
// largest of its eight (measured; 1.4e-5 of the result's norm where the operands are normal, and at most 7 2^-13 of
// the terms' sizes), and what it adds up is fp32.  For results in fp32 that would be seen: there the bytes become bf16,
// which holds each of them exactly, at half of the rate and the price of the conversions.
constexpr int kOne = 0x7F7F7F7F;  // block scales of 1
__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
    const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)};
    return __builtin_bit_cast(bf16x8, v);
}
template <class T>
struct Frag;  // what a lane holds of an operand, ready for the matrix instruction
template <>
struct Frag<bf16_t> {
    i32x8 v;
    Frag() = default;
    __device__ __forceinline__ explicit Frag(i32x8 x) : v(x) {}
};
template <>
struct Frag<float> {
    bf16x8 v[4];
    Frag() = default;
    __device__ __forceinline__ explicit Frag(i32x8 x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = widen(x[2 * i], x[2 * i + 1]);
    }
};
__device__ __forceinline__ f32x4 mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, c, 0, 0, 0, kOne, 0, kOne);
}
__device__ __forceinline__ f32x16 mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a.v, b.v, c, 0, 0, 0, kOne, 0, kOne);
}
__device__ __forceinline__ f32x4 mma(const Frag<float>& a, const Frag<float>& b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x16 mma(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}

// Four neighbouring columns n .. of row m.
template <class T>
__device__ __forceinline__ void store4(const GemmF8Args& g, int64_t m, int n, const float* v) {
    T* p = (T*)g.c + m * g.ldc + n;
    T u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = from_f<T>(v[e]);
    if (n + 4 <= g.N) {
        __builtin_memcpy(p, u, sizeof(u));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < g.N) p[e] = u[e];
    }
}

// ------------------------------------------------------------------ any operands
// Small products of rows that no tile takes, and rows whose strides or starts alone are no multiple of 16: 64 rows by
// 64 columns a workgroup, 16 bytes at a time where a chunk lies inside the row, byte by byte in its tail.
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
        const auto frag = [&](int op, int row) {
            i32x8 x;
            __builtin_memcpy(&x, &lds[op][(row + (lane & 15)) * LD + (lane >> 4) * 32], 32);
            return Frag<T>(x);
        };
        const Frag<T> a = frag(0, wave * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = mma(frag(1, j * 16), a, acc[j]);
    }
    const int64_t m = m0 + wave * 16 + (lane & 15);
    if (m >= g.M) return;
    const float sa = g.a_scale ? g.a_scale[m] : 1.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + j * 16 + (lane >> 4) * 4;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = acc[j][i] * sa * (g.b_scale && n + i < g.N ? g.b_scale[n + i] : 1.f);
        store4<T>(g, m, n, v);
    }
}

// ------------------------------------------------------------------ tiles
// Rows that start 16-byte aligned, K a multiple of 16.  BM x BN of c a workgroup, WM x WN waves; 128 of k a step, in
// two to four stages of LDS that the copies fill without registers (lane l of a wave writes 16 bytes at the instruction's
// base + 16 l, so an instruction fills eight rows of 128 bytes).  Chunk c of row r lies at c ^ r % 8 ^ r / 8 % 8: eight
// neighbouring rows, and sixteen, read one chunk from distinct banks.
// As the compiler's own instruction the copy would be waited for before every read of LDS that it might write; here the
// kernel's waits alone count: each names the copies that the next step reads.  m0 is free: nothing else here uses it.
__device__ __forceinline__ uint32_t lds_at(const uint8_t* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)p;
}
__device__ __forceinline__ void copy16(const uint8_t* base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}

// At most N copies and no LDS operation in flight, and a barrier: unlike __syncthreads it does not wait for all copies.
template <int N>
__device__ __forceinline__ void stage_barrier() {
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int64_t kTileStride = int64_t(1) << 23;  // 256 rows have 32-bit offsets

// T: the type that chooses the arithmetic; Out: that of the elements of c, T or, for a slice of k, float.
template <class T, class Out, int BM, int BN, int WM, int WN, int STAGES>
__global__ void __launch_bounds__(64 * WM * WN) gemm_f8_tile_kernel(GemmF8Args g, int tiles_m, int tiles_n, int slice) {
    constexpr int WAVES = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, CA = BM / 8 / WAVES, CB = BN / 8 / WAVES;
    static_assert(BM % (WM * 32) == 0 && BN % (WN * 32) == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "tiles");
    __shared__ __align__(1024) uint8_t st0[(BM + BN) * 128], st1[(BM + BN) * 128];
    __shared__ __align__(1024) uint8_t st2[STAGES > 2 ? (BM + BN) * 128 : 16], st3[STAGES > 3 ? (BM + BN) * 128 : 16];
    uint8_t* const stage[4] = {st0, st1, st2, st3};
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // workgroups go to the eight XCDs in turn: each takes a run of tiles, in columns of eight tiles, so that tiles
    // that share rows of a or b share an L2
    const int tiles = tiles_m * tiles_n, id = blockIdx.x, run = (tiles + 7) / 8;
    const int t0 = id % 8 * run + id / 8;
    if (id / 8 >= run || t0 >= tiles) return;
    const int group = t0 / (8 * tiles_n), height = min(8, tiles_m - group * 8), in = t0 - group * 8 * tiles_n;
    const int64_t m0 = (int64_t)(group * 8 + in % height) * BM;
    const int n0 = in / height * BN;

    // this lane's part of a copy: row lane / 8 of eight, the chunk that belongs at lane % 8; rows past the last are the
    // last one again, their results are not stored
    const int64_t k0 = (int64_t)blockIdx.y * slice;  // the slice of k: a multiple of 128, all of it in one
    const int K = (int)min((int64_t)slice, g.K - k0);
    const uint8_t *a = g.a + m0 * g.lda + k0, *b = g.b + (int64_t)n0 * g.ldb + k0;
    const int last_a = (int)min(g.M - m0, (int64_t)BM) - 1, last_b = min(g.N - n0, BN) - 1;
    uint32_t off_a[CA], off_b[CB];
    const auto chunk = [&](int q) { return ((lane & 7) ^ (lane >> 3) ^ (q & 7)) * 16; };
#pragma unroll
    for (int i = 0; i < CA; ++i)
        off_a[i] = (uint32_t)(min((wave + i * WAVES) * 8 + (lane >> 3), last_a) * (int)g.lda + chunk(wave + i * WAVES));
#pragma unroll
    for (int i = 0; i < CB; ++i)
        off_b[i] = (uint32_t)(min((wave + i * WAVES) * 8 + (lane >> 3), last_b) * (int)g.ldb + chunk(BM / 8 + wave + i * WAVES));
    const auto copy = [&](uint8_t* st, int64_t k) {
        const uint32_t to = lds_at(st) + wave * 1024;
#pragma unroll
        for (int i = 0; i < CA; ++i) copy16(a + k, off_a[i], to + i * WAVES * 1024);
#pragma unroll
        for (int i = 0; i < CB; ++i) copy16(b + k, off_b[i], to + (BM / 8 + i * WAVES) * 1024);
    };

    f32x16 acc[TN][TM] = {};
    const int wm = wave % WM * (TM * 32), wn = BM + wave / WM * (TN * 32);
    // row base + 32 i + lane % 32, chunks 4 s + 2 (lane / 32) and the next: i and s flip one bit of the place alone
    const auto place = [&](int base, int e) {
        const int r = base + (lane & 31);
        return r * 128 + ((2 * (lane >> 5) + e) ^ (r & 7) ^ (r >> 3 & 7)) * 16;
    };
    const int pa[2] = {place(wm, 0), place(wm, 1)}, pb[2] = {place(wn, 0), place(wn, 1)};
    const auto frag = [&](const uint8_t* st, const int (&p)[2], int i, int s) {
        const int flip = (s ^ (i & 1)) * 64;
        const i32x4 lo = *(const i32x4*)(st + (p[0] ^ flip) + i * 4096), hi = *(const i32x4*)(st + (p[1] ^ flip) + i * 4096);
        return Frag<T>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const auto compute = [&](const uint8_t* st) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            Frag<T> fb[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = frag(st, pb, j, s);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const Frag<T> fa = frag(st, pa, i, s);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[j][i] = mma(fb[j], fa, acc[j][i]);
            }
        }
    };
    // a copy is issued STAGES - 1 steps ahead, also past the last (that one again), so that their number is known
    constexpr int AHEAD = STAGES - 1;
    const int steps = K / 128;
    if (steps) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) copy(stage[u], (int64_t)min(u, steps - 1) * 128);
        for (int t = 0; t < steps; t += STAGES) {
#pragma unroll
            for (int u = 0; u < STAGES; ++u) {
                if (t + u >= steps) break;
                stage_barrier<(CA + CB) * (AHEAD - 1)>();  // this step's stage is here, and the one before has been read
                copy(stage[(u + AHEAD) % STAGES], (int64_t)min(t + u + AHEAD, steps - 1) * 128);
                compute(stage[u]);
            }
        }
        stage_barrier<0>();
    }
    if (const int rest = K % 128) {  // chunks past K are zeros
        const int64_t k = (int64_t)steps * 128;
#pragma unroll
        for (int i = 0; i < CA + CB; ++i) {
            const int q = i < CA ? wave + i * WAVES : BM / 8 + wave + (i - CA) * WAVES;
            i32x4 v = {0, 0, 0, 0};
            if (chunk(q) < rest) v = *(const i32x4*)((i < CA ? a + off_a[i < CA ? i : 0] : b + off_b[i < CA ? 0 : i - CA]) + k);
            *(i32x4*)(st0 + q * 1024 + lane * 16) = v;
        }
        stage_barrier<0>();
        compute(st0);
        stage_barrier<0>();
    }

    // 32 rows of the wave at a time through its part of the LDS, so that rows are written 16 bytes a lane: straight from
    // the accumulators, which hold four columns of 32 rows, 8192^3 took 462 us and not 431
    constexpr int E = 16 / sizeof(Out), ROW = TN * 32 / E;  // elements of a chunk, chunks of a row
    uint8_t* mine = st0 + wave * (32 * TN * 32 * (int)sizeof(Out));
    static_assert(WAVES * 32 * TN * 32 * sizeof(Out) <= sizeof(st0), "the waves' rows fit a stage");
    const int nw = n0 + wn - BM;
    Out* c = (Out*)g.c + blockIdx.y * g.M * g.ldc;
    float sb[TN][16];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            sb[j][e] = g.b_scale ? g.b_scale[min(nw + j * 32 + e / 4 * 8 + (lane >> 5) * 4 + e % 4, g.N - 1)] : 1.f;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t mw = m0 + wm + i * 32;
        const float sa = g.a_scale ? g.a_scale[min(mw + (lane & 31), g.M - 1)] : 1.f;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                Out v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = from_f<Out>(acc[j][i][q * 4 + e] * sa * sb[j][q * 4 + e]);
                const int n = j * 32 + q * 8 + (lane >> 5) * 4, x = n / E;
                __builtin_memcpy(mine + ((lane & 31) * ROW + (x ^ (lane & (ROW - 1)))) * 16 + n % E * sizeof(Out), v, sizeof(v));
            }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
        for (int x = lane; x < 32 * ROW; x += 64) {
            const int r = x / ROW, q = x % ROW, n = nw + q * E;
            const u32x4 u = *(const u32x4*)(mine + (r * ROW + (q ^ (r & (ROW - 1)))) * 16);
            if (mw + r >= g.M) continue;
            Out* p = c + (mw + r) * g.ldc + n;
            if (n + E <= g.N) {
                *(u32x4_any*)p = u;
            } else {
                Out v[E];
                __builtin_memcpy(v, &u, 16);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (n + e < g.N) p[e] = v[e];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
}

// ------------------------------------------------------------------ few rows of a
// Up to 32 rows: b is read once, straight into registers; 16 columns a workgroup, whose waves take runs of k and join
// their sums in order.  b's rows are the matrix instruction's first operand, a's 16 TM rows its second.  Any strides,
// alignments and K.
template <class T, int TM, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) gemm_f8_few_kernel(GemmF8Args g) {
    constexpr int FLY = TM == 1 ? 8 : 4;  // steps of 128 in flight
    __shared__ f32x4 part[WAVES][TM][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)block_of() * 16;
    if (n0 >= g.N) return;
    const int steps = (g.K + 127) / 128, each = (steps + WAVES - 1) / WAVES;
    const int first = min(steps, wave * each), last = min(steps, first + each);
    const uint8_t* b = g.b + min(n0 + (lane & 15), (int64_t)g.N - 1) * g.ldb + (lane >> 4) * 32;
    const uint8_t* a[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) a[i] = g.a + min((int64_t)(i * 16 + (lane & 15)), g.M - 1) * g.lda + (lane >> 4) * 32;
    const auto load = [&](const uint8_t* p, int t) {  // zeros past K
        const int left = g.K - t * 128 - (lane >> 4) * 32;
        i32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        p += (int64_t)t * 128;
        if (left >= 32) {
            __builtin_memcpy(&v, p, 32);
        } else if (left > 0) {
            uint8_t u[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) u[e] = e < left ? p[e] : 0;
            __builtin_memcpy(&v, u, 32);
        }
        return v;
    };
    f32x4 acc[TM] = {};
    for (int t = first; t < last; t += FLY) {
        i32x8 vb[FLY], va[FLY][TM];
#pragma unroll
        for (int u = 0; u < FLY; ++u)
            if (t + u < last) {
                vb[u] = load(b, t + u);
#pragma unroll
                for (int i = 0; i < TM; ++i) va[u][i] = load(a[i], t + u);
            }
#pragma unroll
        for (int u = 0; u < FLY; ++u)
            if (t + u < last) {
                const Frag<T> fb(vb[u]);
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[i] = mma(fb, Frag<T>(va[u][i]), acc[i]);
            }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave >= TM) return;
    f32x4 sum = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += part[w][wave][lane];
    const int64_t m = wave * 16 + (lane & 15);
    const int n = (int)n0 + (lane >> 4) * 4;
    if (m >= g.M || n >= g.N) return;
    const float sa = g.a_scale ? g.a_scale[m] : 1.f;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = sum[e] * sa * (g.b_scale && n + e < g.N ? g.b_scale[n + e] : 1.f);
    store4<T>(g, m, n, v);
}

// ------------------------------------------------------------------ the launches
// c from the slices' sums, [slices][M][N], in order.  A thread has four columns.
template <class T>
__global__ void __launch_bounds__(256) gemm_f8_join_kernel(GemmF8Args g, const float* __restrict__ part, int slices) {
    const int64_t quads = (g.N + 3) / 4, id = (int64_t)block_of() * 256 + threadIdx.x, m = id / quads;
    if (m >= g.M) return;
    const int n = (int)(id - m * quads) * 4;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int at = min(n + e, g.N - 1);
        float sum = 0.f;
#pragma unroll 8
        for (int k = 0; k < slices; ++k) sum += part[(k * g.M + m) * g.N + at];
        v[e] = sum * (g.a_scale ? g.a_scale[m] : 1.f) * (g.b_scale ? g.b_scale[at] : 1.f);
    }
    store4<T>(g, m, n, v);
}

// Which kernel, by what each took (us) on one card:
//   M     N      K      few rows  64 x 64  128 x 128, 3 stages  2 stages  256 x 256
//   4     4096   4096   6.5       17.5
//   1     128000 4096   88        99
//   20    128000 1024   47        24
//   32    4096   4096   9.5       17.5
//   256   4096   4096             10.9     20.6                 23.9      43.9
//   600   4096   4096                      19.0                 23.8
//   1024  4096   4096             30       23.1                 27.1      47.2
//   2603  2304   768              16.3     14.3                 12.4      17.2
//   2048  4096   4096             56       42.6                 35.4      50.7
//   4096  4096   4096             104      82                   65.7      61.9
//   8192  8192   8192             858      615                  521       427
// Tiles of 64 hold four stages and of 128 three where a CU has a workgroup or two at a time: the copies then have the
// memory's latency for themselves, and a lone tile of 128 is shared by eight waves (600 x 4096 x 4096 21.3 us with
// four).  From two rounds of workgroups on, two stages and two workgroups a CU hide it better.
constexpr int kCUs = 256;
bool few_rows(int64_t M, int32_t N) { return M <= 16 || (M <= 32 && cdiv(N, 64) < kCUs); }
// Slices of k, of 2048 or more, where 64 x 64 tiles are few and k is long: 100 x 1024 x 8192 14.2 -> 11.8 us, 40 x 512 x
// 16384 23.6 -> 10.9; the launch that joins them eats the gain up where k is shorter (256 x 256 x 4096 9.2 -> 9.9).
int slices_of(int64_t M, int32_t N, int32_t K) {
    const int64_t tiles = cdiv(M, 64) * cdiv(N, 64);
    return tiles > kCUs / 4 || K < 8192 ? 1 : std::min(K / 2048, 16);
}

// Rows of K bytes to rows of `ld`, a multiple of 16 with zeros past K: chunks of a's rows, then of b's.
__global__ void __launch_bounds__(256) gemm_f8_align_kernel(GemmF8Args g, uint8_t* __restrict__ a, uint8_t* __restrict__ b, int64_t ld) {
    const int64_t chunks = ld / 16, id = (int64_t)block_of() * 256 + threadIdx.x, row = id / chunks, k = id % chunks * 16;
    if (row >= g.M + g.N) return;
    const bool first = row < g.M;
    const uint8_t* from = first ? g.a + row * g.lda : g.b + (row - g.M) * g.ldb;
    uint8_t v[16];
    if (k + 16 <= g.K) {
        __builtin_memcpy(v, from + k, 16);
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = k + e < g.K ? from[k + e] : 0;
    }
    __builtin_memcpy((first ? a + row * ld : b + (row - g.M) * ld) + k, v, 16);
}
// Whether a product whose rows have no multiple of 16 bytes is worth copies of its operands that have: with and without
// them 100 x 1000 x 1001 takes 10 and 14 us, 2048 x 2048 x 2047 27 and 41, 8000 x 8000 x 8001 483 and 1756.
bool copies_pay(int64_t M, int32_t N, int32_t K) { return K % 16 && M > 32 && (double)M * N * K >= 1e8; }

template <class T, class Out, int BM, int BN, int WM, int WN, int STAGES>
void launch_tiles(const GemmF8Args& g, int slices, hipStream_t s) {
    const int tm = (int)cdiv(g.M, BM), tn = (int)cdiv(g.N, BN), slice = (int)(cdiv(cdiv(g.K, 128), slices) * 128);
    const dim3 grid((unsigned)(cdiv((int64_t)tm * tn, 8) * 8), (unsigned)cdiv(g.K, slice));
    gemm_f8_tile_kernel<T, Out, BM, BN, WM, WN, STAGES><<<grid, 64 * WM * WN, 0, s>>>(g, tm, tn, slice);
}

template <class T>
fo_status run_tiles(const GemmF8Args& g, float* part, hipStream_t s) {
    const auto tiles = [&](int side) { return cdiv(g.M, side) * cdiv(g.N, side); };
    const int slices = slices_of(g.M, g.N, g.K);
    if (slices > 1) {
        GemmF8Args h = g;
        h.c = part;
        h.ldc = g.N;
        h.a_scale = h.b_scale = nullptr;
        launch_tiles<T, float, 64, 64, 2, 2, 4>(h, slices, s);
        FO_LAUNCHED();
        const int n = (int)cdiv(g.K, cdiv(cdiv(g.K, 128), slices) * 128);
        gemm_f8_join_kernel<T><<<grid_of(cdiv(g.M * cdiv(g.N, 4), 256)), 256, 0, s>>>(g, part, n);
    } else if (tiles(64) <= 2 * kCUs) {
        launch_tiles<T, T, 64, 64, 2, 2, 4>(g, 1, s);
    } else if (tiles(128) <= kCUs) {
        launch_tiles<T, T, 128, 128, 2, 4, 3>(g, 1, s);
    } else if (tiles(256) < kCUs * 3 / 4) {
        launch_tiles<T, T, 128, 128, 2, 2, 2>(g, 1, s);
    } else {
        launch_tiles<T, T, 256, 256, 2, 4, 2>(g, 1, s);
    }
    FO_LAUNCHED();
    return FO_OK;
}

int64_t part_bytes(int64_t M, int32_t N, int32_t K) {
    const int slices = slices_of(M, N, K);
    return slices > 1 ? cdiv((int64_t)slices * M * N * 4, 16) * 16 : 0;
}

template <class T>
fo_status run(const GemmF8Args& g, char* ws, hipStream_t s) {
    const bool whole = g.K % 16 == 0 && g.lda < kTileStride && g.ldb < kTileStride && g.lda % 16 == 0 &&
                       g.ldb % 16 == 0 && ((uintptr_t)g.a & 15) == 0 && ((uintptr_t)g.b & 15) == 0;
    const int64_t ld = cdiv(g.K, 16) * 16;
    if (few_rows(g.M, g.N)) {
        const dim3 grid = grid_of(cdiv(g.N, 16));
        // eight waves share k where columns are few (4 x 4096 x 4096: 6.5 us either way), else four (1 x 128000 x 4096:
        // 88 us, 108 with eight)
        if (g.M > 16) gemm_f8_few_kernel<T, 2, 8><<<grid, 512, 0, s>>>(g);
        else if (g.N < 16 * 4 * kCUs) gemm_f8_few_kernel<T, 1, 8><<<grid, 512, 0, s>>>(g);
        else gemm_f8_few_kernel<T, 1, 4><<<grid, 256, 0, s>>>(g);
    } else if (whole) {
        return run_tiles<T>(g, (float*)ws, s);
    } else if (copies_pay(g.M, g.N, g.K) && ld < kTileStride) {
        GemmF8Args h = g;
        uint8_t *a = (uint8_t*)ws + part_bytes(g.M, g.N, (int32_t)ld), *b = a + g.M * ld;
        gemm_f8_align_kernel<<<grid_of(cdiv((g.M + g.N) * (ld / 16), 256)), 256, 0, s>>>(g, a, b, ld);
        FO_LAUNCHED();
        h.a = a; h.b = b;
        h.lda = h.ldb = ld;
        h.K = (int32_t)ld;
        return run_tiles<T>(h, (float*)ws, s);
    } else {
        gemm_f8_any_kernel<T><<<grid_of(cdiv(g.M, 64) * cdiv(g.N, 64)), 256, 0, s>>>(g);
    }
    FO_LAUNCHED();
    return FO_OK;
}

}  // namespace

int64_t gemm_f8_workspace(int64_t M, int32_t N, int32_t K) {
    if (few_rows(M, N)) return 0;  // no rows among them
    const int64_t ld = cdiv(K, 16) * 16;
    if (copies_pay(M, N, K)) return part_bytes(M, N, (int32_t)ld) + (M + N) * ld;
    return K % 16 ? 0 : part_bytes(M, N, K);  // odd rows go to the kernel for any operands
}

fo_status launch_gemm_f8(int32_t dtype, const GemmF8Args& g, void* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? run<bf16_t>(g, (char*)ws, s) : run<float>(g, (char*)ws, s);
}

}  // namespace fo
