// Products of 8-bit rows with a scale each: c_mn = a_scale[m] b_scale[n] sum_k a_mk b_nk.
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
// Any strides, alignments and K: 64 rows by 64 columns a workgroup, 16 bytes at a time where a chunk lies inside the
// row, byte by byte in its tail.
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
// two stages of LDS that the copies fill without registers (lane l of a wave writes 16 bytes at the instruction's
// base + 16 l, so an instruction fills eight rows of 128 bytes).  Chunk c of row r lies at c ^ r % 8 ^ r / 8 % 8: eight
// neighbouring rows, and sixteen, read one chunk from distinct banks.  The stages are arrays of their own, so that the
// compiler knows a read of one from a copy into the other.
__device__ __forceinline__ void copy16(const uint8_t* base, uint32_t off, uint8_t* to) {
    __builtin_amdgcn_global_load_lds(base + off, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// No copy or LDS operation in flight; and a barrier that, unlike __syncthreads, does not wait for copies.
__device__ __forceinline__ void stage_barrier() {
    __builtin_amdgcn_s_waitcnt(7 << 4);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int64_t kTileStride = int64_t(1) << 23;  // 256 rows have 32-bit offsets

template <class T, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) gemm_f8_tile_kernel(GemmF8Args g, int tiles_m, int tiles_n) {
    constexpr int WAVES = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, CA = BM / 8 / WAVES, CB = BN / 8 / WAVES;
    static_assert(BM % (WM * 32) == 0 && BN % (WN * 32) == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "tiles");
    __shared__ __align__(1024) uint8_t st0[(BM + BN) * 128];
    __shared__ __align__(1024) uint8_t st1[(BM + BN) * 128];
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
    const uint8_t *a = g.a + m0 * g.lda, *b = g.b + (int64_t)n0 * g.ldb;
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
#pragma unroll
        for (int i = 0; i < CA; ++i) copy16(a + k, off_a[i], st + (wave + i * WAVES) * 1024);
#pragma unroll
        for (int i = 0; i < CB; ++i) copy16(b + k, off_b[i], st + (BM / 8 + wave + i * WAVES) * 1024);
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
    const int steps = g.K / 128;
    if (steps) {
        copy(st0, 0);
        stage_barrier();
        int t = 0;
        for (; t + 2 < steps; t += 2) {
            copy(st1, (int64_t)(t + 1) * 128);
            compute(st0);
            stage_barrier();  // st1 is here, and st0 has been read
            copy(st0, (int64_t)(t + 2) * 128);
            compute(st1);
            stage_barrier();
        }
        if (t + 1 < steps) copy(st1, (int64_t)(t + 1) * 128);
        compute(st0);
        stage_barrier();
        if (t + 1 < steps) {
            compute(st1);
            stage_barrier();
        }
    }
    if (const int rest = g.K % 128) {  // chunks past K are zeros
        const int64_t k = (int64_t)steps * 128;
#pragma unroll
        for (int i = 0; i < CA + CB; ++i) {
            const int q = i < CA ? wave + i * WAVES : BM / 8 + wave + (i - CA) * WAVES;
            i32x4 v = {0, 0, 0, 0};
            if (chunk(q) < rest) v = *(const i32x4*)((i < CA ? a + off_a[i < CA ? i : 0] : b + off_b[i < CA ? 0 : i - CA]) + k);
            *(i32x4*)(st0 + q * 1024 + lane * 16) = v;
        }
        stage_barrier();
        compute(st0);
        stage_barrier();
    }

    // 32 rows of the wave at a time through its part of the LDS, so that rows are written 16 bytes a lane: straight from
    // the accumulators, which hold four columns of 32 rows, 8192^3 took TIME_STRAIGHT us
    constexpr int E = 16 / sizeof(T), ROW = TN * 32 / E;  // elements of a chunk, chunks of a row
    uint8_t* mine = st0 + wave * (32 * TN * 32 * (int)sizeof(T));
    static_assert(WAVES * 32 * TN * 32 * sizeof(T) <= sizeof(st0), "the waves' rows fit a stage");
    const int nw = n0 + wn - BM;
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
                T v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = from_f<T>(acc[j][i][q * 4 + e] * sa * sb[j][q * 4 + e]);
                const int n = j * 32 + q * 8 + (lane >> 5) * 4, c = n / E;
                __builtin_memcpy(mine + ((lane & 31) * ROW + (c ^ (lane & (ROW - 1)))) * 16 + n % E * sizeof(T), v, sizeof(v));
            }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
        for (int x = lane; x < 32 * ROW; x += 64) {
            const int r = x / ROW, c = x % ROW, n = nw + c * E;
            const u32x4 u = *(const u32x4*)(mine + (r * ROW + (c ^ (r & (ROW - 1)))) * 16);
            if (mw + r >= g.M) continue;
            T* p = (T*)g.c + (mw + r) * g.ldc + n;
            if (n + E <= g.N) {
                *(u32x4_any*)p = u;
            } else {
                T v[E];
                __builtin_memcpy(v, &u, 16);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (n + e < g.N) p[e] = v[e];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
}

template <class T, int BM, int BN, int WM, int WN>
void launch_tiles(const GemmF8Args& g, hipStream_t s) {
    const int tm = (int)cdiv(g.M, BM), tn = (int)cdiv(g.N, BN);
    gemm_f8_tile_kernel<T, BM, BN, WM, WN><<<(unsigned)(cdiv((int64_t)tm * tn, 8) * 8), 64 * WM * WN, 0, s>>>(g, tm, tn);
}

template <class T>
fo_status run(const GemmF8Args& g, hipStream_t s) {
    const bool whole = g.K % 16 == 0 && g.lda < kTileStride && g.ldb < kTileStride && g.lda % 16 == 0 && g.ldb % 16 == 0 && ((uintptr_t)g.a & 15) == 0 && ((uintptr_t)g.b & 15) == 0;
#ifndef SHAPE
#define SHAPE 0
#endif
    if (!whole) gemm_f8_any_kernel<T><<<grid_of(cdiv(g.M, 64) * cdiv(g.N, 64)), 256, 0, s>>>(g);
    else if (SHAPE == 1 || (SHAPE == 0 && cdiv(g.M, 256) * cdiv(g.N, 256) >= 256)) launch_tiles<T, 256, 256, 2, 4>(g, s);
    else if (SHAPE == 2 || (SHAPE == 0 && cdiv(g.M, 128) * cdiv(g.N, 128) >= 256)) launch_tiles<T, 128, 128, 2, 2>(g, s);
    else launch_tiles<T, 64, 64, 2, 2>(g, s);
    FO_LAUNCHED();
    return FO_OK;
}

}  // namespace

int64_t gemm_f8_workspace(int64_t M, int32_t N, int32_t K) { return 0; }

fo_status launch_gemm_f8(int32_t dtype, const GemmF8Args& g, void* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? run<bf16_t>(g, s) : run<float>(g, s);
}

}  // namespace fo
