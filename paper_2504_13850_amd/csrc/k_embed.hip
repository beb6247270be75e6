// Embedding: rows of a table by tokens, and the table's gradient.
//
// Bound by HBM: the named rows in and out; the gradient's rows in and the table's
// gradient out, most of it zeros where the batch is small beside the vocabulary.
//
// The gradient's sums have to come in the same order every time, so there are no
// atomics on them: the rows are sorted by token (stable), the sorted list is cut
// into pieces of equal length whatever the tokens are, a team of threads sums a
// piece's rows and writes each token that begins and ends inside it, and the sums of
// tokens that cross pieces are joined by a last launch.  The zeros are written in
// shares beside the sort's launches, which leave the memory idle.
#include <algorithm>

#include "lm.h"
#include "row8.h"

namespace fo {
namespace {

// A team of 2^tx threads takes 8 << tx columns of a row (all of them, up to 2048), 256 >> tx teams a workgroup.
int team_bits(int32_t cols) {
    int tx = 2;  // 64 teams at most: their entries have to fit the LDS
    while (tx < 8 && (8 << tx) < cols) ++tx;
    return tx;
}

// The eight columns of a team's thread.  32-bit values as two fours half a row apart, so that a wave's stores are whole
// lines: past the caches each instruction's stores leave by themselves, and half lines go at half the rate.  A pass with
// the forward, fp32: 8192 rows of 2048 over 32000 tokens 169 us with eight in a run (zeros too), 100 as here; 60170 rows
// of 1480 over 48577 tokens 353 and 271.
struct Mine {
    int64_t c0;
    int n, step;
};
template <class T>
__device__ __forceinline__ Mine mine_of(int32_t cols, int tx) {
    const int t = threadIdx.x & ((1 << tx) - 1), w = min(2048, cols - (int)blockIdx.z * 2048);
    const int64_t c = (int64_t)blockIdx.z * 2048;
    if (sizeof(T) == 2) return {c + t * 8, min(8, w - t * 8), 4};
    const int step = (w + 7) / 8 * 4, second = w - step - t * 4;
    return {c + t * 4, t * 4 >= step ? 0 : second > 0 ? 4 + min(4, second) : min(4, w - t * 4), step};
}

// A thread's columns of a row, in two steps: the loads of several rows, then the row's end put in place (16 bits).
template <class T, bool NT>
__device__ __forceinline__ void load_mine(Eight<T, NT>& x, const T* row, Mine m, int32_t cols) {
    if (sizeof(T) == 2) x.load_row(row, (int)m.c0, cols);
    else x.load(row + m.c0, m.n, m.n == 8, m.step);
}
template <class T, bool NT>
__device__ __forceinline__ void fit_mine(Eight<T, NT>& x, Mine m, int32_t cols) {
    if (sizeof(T) == 2) x.fit(m.n, cols);
}

constexpr int64_t kPastCaches = int64_t(256) << 20;

// ------------------------------------------------------------------ forward
constexpr int FWD_FLY = 4;  // rows of a team in flight

template <class T, bool NT>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmbedArgs a, int tx) {
    const int ty = threadIdx.x >> tx, teams = 256 >> tx;
    const Mine m = mine_of<T>(a.cols, tx);
    const int64_t r0 = (int64_t)block_of() * teams * FWD_FLY + ty;
    if (m.n <= 0) return;
    int token[FWD_FLY];
    Eight<T, false> x[FWD_FLY];
#pragma unroll
    for (int k = 0; k < FWD_FLY; ++k) token[k] = r0 + k * teams < a.rows ? a.tokens[r0 + k * teams] : -1;
#pragma unroll
    for (int k = 0; k < FWD_FLY; ++k) {
        if ((uint32_t)token[k] < (uint32_t)a.vocab)
            load_mine(x[k], (const T*)a.table + token[k] * a.table_ld, m, a.cols);
        else
            x[k] = {};
    }
#pragma unroll
    for (int k = 0; k < FWD_FLY; ++k) {
        if (r0 + k * teams >= a.rows) continue;
        float y[8];
        fit_mine(x[k], m, a.cols);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[k].at(e) * a.scale;
        if ((uint32_t)token[k] >= (uint32_t)a.vocab)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = 0.f;
        Eight<T, NT>::store((T*)a.out + (r0 + k * teams) * a.out_ld + m.c0, y, m.n, m.n == 8, m.step);
    }
}

template <class T>
fo_status fwd(const EmbedArgs& a, hipStream_t s) {
    const int tx = team_bits(a.cols);
    dim3 g = grid_of(cdiv(a.rows, (256 >> tx) * FWD_FLY));
    g.z = (unsigned)cdiv(a.cols, 2048);
    // past the caches: see Eight
    if (a.rows * a.cols * (int64_t)sizeof(T) >= kPastCaches) embed_fwd_kernel<T, true><<<g, 256, 0, s>>>(a, tx);
    else embed_fwd_kernel<T, false><<<g, 256, 0, s>>>(a, tx);
    FO_LAUNCHED();
    return FO_OK;
}

// ------------------------------------------------------------------ zeros
// The zeros are written in shares, one beside each launch of the sort that has
// workgroups of some length: they leave the memory idle.  NT: past the caches.
constexpr int64_t kFillWgs = 1024;
struct Fill {
    int wgs;          // workgroups of a launch
    int share, of;    // which of how many shares
};

template <class T, bool NT, int THREADS>
__device__ void fill_zeros(const EmbedArgs& a, Fill f, int id) {
    constexpr int PER = 16 / sizeof(T);  // a store's
    const auto zero = [](T* y, int64_t left) {
        if (left >= PER) {
            u32x4_any* q = reinterpret_cast<u32x4_any*>(y);
            if (NT) __builtin_nontemporal_store(u32x4{}, q);
            else *q = u32x4{};
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (e < left) y[e] = T(0);
        }
    };
    T* y = (T*)a.dtable;
    if (a.dtable_ld == a.cols) {  // one run
        const int64_t all = (int64_t)a.vocab * a.cols, chunks = (all + PER - 1) / PER, each = (chunks + f.of - 1) / f.of;
        const int64_t last = min(chunks, (f.share + 1) * each);
        for (int64_t c = f.share * each + (int64_t)id * THREADS + threadIdx.x; c < last; c += (int64_t)f.wgs * THREADS)
            zero(y + c * PER, all - c * PER);
        return;
    }
    for (int64_t v = (int64_t)id * f.of + f.share; v < a.vocab; v += (int64_t)f.wgs * f.of)
        for (int64_t c0 = threadIdx.x * PER; c0 < a.cols; c0 += THREADS * PER) zero(y + v * a.dtable_ld + c0, a.cols - c0);
}

// ------------------------------------------------------------------ sort
// An entry of the sorted list: token (as unsigned: those outside the vocabulary come last) and row.
typedef uint2 Entry;

// Few rows: an entry's place is the number of entries that come before it, counted.
// 16 rows a workgroup, 64 threads with every 64th four of the tokens for each; n^2
// comparisons of two instructions, spread over all CUs: 4096 rows and 49 MB of zeros
// 11 us (64 rows a workgroup, tokens by scalar loads: 19).
constexpr int64_t kCountRows = 8192;
constexpr int COUNT_THREADS = 1024, COUNT_ROWS = 16, COUNT_SHARES = COUNT_THREADS / COUNT_ROWS;

template <class T, bool NT>
__global__ void __launch_bounds__(COUNT_THREADS) embed_count_kernel(EmbedArgs a, Entry* __restrict__ out, int wgs, Fill f) {
    if ((int)blockIdx.x >= wgs) {
        fill_zeros<T, NT, COUNT_THREADS>(a, f, (int)blockIdx.x - wgs);
        return;
    }
    __shared__ __align__(16) uint32_t tok[kCountRows];
    __shared__ int part[COUNT_THREADS / 64][COUNT_ROWS];
    const int n = (int)a.rows, padded = (n + 3) & ~3, first = blockIdx.x * COUNT_ROWS;
    for (int i = threadIdx.x; i < padded; i += COUNT_THREADS)
        tok[i] = i < n ? min((uint32_t)a.tokens[i], (uint32_t)a.vocab) : ~0u;
    __syncthreads();
    const int i = first + (int)(threadIdx.x % COUNT_ROWS), share = threadIdx.x / COUNT_ROWS;
    const uint32_t mine = i < n ? tok[i] : 0u;
    int before = 0;
#pragma unroll 4
    for (int j = share * 4; j < padded; j += COUNT_SHARES * 4) {
        const uint4 k = *(const uint4*)&tok[j];
        if (j >= first && j < first + COUNT_ROWS) {
            before += (k.x < mine || (k.x == mine && j < i)) + (k.y < mine || (k.y == mine && j + 1 < i)) +
                      (k.z < mine || (k.z == mine && j + 2 < i)) + (k.w < mine || (k.w == mine && j + 3 < i));
        } else {  // rows of earlier workgroups come first on a tie, rows of later ones do not
            const uint32_t most = mine + (j < first);
            before += (k.x < most) + (k.y < most) + (k.z < most) + (k.w < most);
        }
    }
    before += __shfl_xor(before, 16);
    before += __shfl_xor(before, 32);
    if ((threadIdx.x & 63) < COUNT_ROWS) part[threadIdx.x >> 6][threadIdx.x & 63] = before;
    __syncthreads();
    if (threadIdx.x >= COUNT_ROWS || i >= n) return;
    before = 0;
#pragma unroll
    for (int k = 0; k < COUNT_THREADS / 64; ++k) before += part[k][threadIdx.x];
    out[before] = make_uint2(mine, (uint32_t)i);
}

// More rows: digits of up to ten bits, lowest first.  A workgroup has a tile of
// entries, a wave of it a run of them.  counts: [digit][tile].  Tiles of 1024 entries
// spread few rows over many CUs (65536 rows: placing a digit 7 us, 15 with 4096); with more rows
// larger tiles keep the counts small.
constexpr int SORT_THREADS = 256, SORT_WAVES = SORT_THREADS / 64, MAX_BITS = 10;
int tile_of(int64_t rows) { return rows <= int64_t(1) << 20 ? 1024 : 4096; }

struct Digit {
    int shift, bits;
};
__device__ __forceinline__ Entry entry_of(const EmbedArgs& a, const Entry* in, int64_t i) {
    return in ? in[i] : make_uint2(min((uint32_t)a.tokens[i], (uint32_t)a.vocab), (uint32_t)i);
}

template <class T, bool NT>
__global__ void __launch_bounds__(SORT_THREADS) embed_digits_kernel(EmbedArgs a, const Entry* __restrict__ in, Digit d,
                                                                     int tile, int* __restrict__ counts, int tiles, Fill f) {
    if ((int)blockIdx.x >= tiles) {
        fill_zeros<T, NT, SORT_THREADS>(a, f, (int)blockIdx.x - tiles);
        return;
    }
    __shared__ int sum[1 << MAX_BITS];
    for (int k = threadIdx.x; k < 1 << d.bits; k += SORT_THREADS) sum[k] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * tile, i1 = min(i0 + tile, a.rows);
#pragma unroll 4
    for (int64_t i = i0 + threadIdx.x; i < i1; i += SORT_THREADS)
        atomicAdd(&sum[entry_of(a, in, i).x >> d.shift & ((1u << d.bits) - 1u)], 1);
    __syncthreads();
    for (int k = threadIdx.x; k < 1 << d.bits; k += SORT_THREADS) counts[(int64_t)k * tiles + blockIdx.x] = sum[k];
}

__device__ __forceinline__ int wave_scan(int v) {  // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int u = __shfl_up(v, m);
        if (lane >= m) v += u;
    }
    return v;
}

// A digit's counts become the sums of those before them; totals[digit] their sum.  A wave a digit.
__global__ void __launch_bounds__(64) embed_scan_kernel(int* __restrict__ counts, int* __restrict__ totals, int tiles) {
    int* row = counts + (int64_t)blockIdx.x * tiles;
    int before = 0;
    for (int t0 = 0; t0 < tiles; t0 += 64) {
        const int t = t0 + (int)threadIdx.x, v = t < tiles ? row[t] : 0, up = wave_scan(v);
        if (t < tiles) row[t] = before + up - v;
        before += __shfl(up, 63);
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

template <class T, bool NT, int TILE>
__global__ void __launch_bounds__(SORT_THREADS) embed_place_kernel(EmbedArgs a, const Entry* __restrict__ in, Digit d,
                                                                    const int* __restrict__ counts, const int* __restrict__ totals,
                                                                    int tiles, Entry* __restrict__ out, Fill f) {
    if ((int)blockIdx.x >= tiles) {
        fill_zeros<T, NT, SORT_THREADS>(a, f, (int)blockIdx.x - tiles);
        return;
    }
    constexpr int PER_THREAD = TILE / SORT_THREADS;
    __shared__ int seen[SORT_WAVES][1 << MAX_BITS];  // a wave's entries of each digit so far
    __shared__ int base[1 << MAX_BITS];
    __shared__ int carry[SORT_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, digits = 1 << d.bits;
    for (int k = threadIdx.x; k < SORT_WAVES << MAX_BITS; k += SORT_THREADS) (&seen[0][0])[k] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * TILE + wave * (TILE / SORT_WAVES) + lane;
    Entry e[PER_THREAD];
    int place[PER_THREAD];
#pragma unroll
    for (int k = 0; k < PER_THREAD; ++k) e[k] = i0 + k * 64 < a.rows ? entry_of(a, in, i0 + k * 64) : make_uint2(0u, 0u);
#pragma unroll
    for (int k = 0; k < PER_THREAD; ++k) {
        const bool there = i0 + k * 64 < a.rows;
        const uint32_t digit = e[k].x >> d.shift & (uint32_t)(digits - 1);
        uint64_t same = __ballot(there);
        for (int b = 0; b < d.bits; ++b) {
            const bool one = digit >> b & 1u;
            const uint64_t ones = __ballot(one);
            same &= one ? ones : ~ones;
        }
        const int earlier = __popcll(same & ((1ull << lane) - 1ull)), all = __popcll(same);
        place[k] = seen[wave][digit] + earlier;
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");  // every lane has read before the first of its digit adds
        if (there && earlier == 0) seen[wave][digit] += all;
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
    __syncthreads();
    // where each digit begins: the totals of smaller digits, and this digit's entries in earlier tiles
    int before = 0;
    for (int k0 = 0; k0 < digits; k0 += SORT_THREADS) {
        const int k = k0 + (int)threadIdx.x, v = k < digits ? totals[k] : 0, up = wave_scan(v);
        if (lane == 63) carry[wave] = up;
        __syncthreads();
        int add = before;
        for (int w = 0; w < wave; ++w) add += carry[w];
        if (k < digits) {
            int at = add + up - v + counts[(int64_t)k * tiles + blockIdx.x];
            base[k] = at;
            int sum = 0;  // and in earlier waves
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) {
                const int c = seen[w][k];
                seen[w][k] = sum;
                sum += c;
            }
        }
        for (int w = 0; w < SORT_WAVES; ++w) before += carry[w];
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < PER_THREAD; ++k) {
        if (i0 + k * 64 >= a.rows) continue;
        const uint32_t digit = e[k].x >> d.shift & (uint32_t)(digits - 1);
        out[base[digit] + seen[wave][digit] + place[k]] = e[k];
    }
}

// ------------------------------------------------------------------ sums
// Entries of a piece: short pieces where rows are few or narrow, so that teams fill the chip.  Each piece takes a
// workgroup of the join, so pieces grow up to 64 entries, which keeps some thousand of them up to 100000 or 260000 rows;
// with more rows there are more, one for 64 rows (the gradient, bf16: 56548 rows of 101 in pieces of 16 35 us, of 64 54;
// 65536 of 2048 197 and 187, of 768 69 and 63; 200000 of 128 76 and 50).
int piece_of(int64_t rows, int32_t cols) {
    const int64_t most = 256 >> team_bits(cols) >= 8 ? 4096 : 1536;
    int piece = 8;
    while (piece < 64 && cdiv(rows, piece) > most) piece *= 2;
    return piece;
}
constexpr int SUM_FLY = 8;  // rows of a team in flight

template <class T, bool NT>
__device__ __forceinline__ void write_row(const EmbedArgs& a, uint32_t token, Mine m, const float* sum) {
    T* y = (T*)a.dtable + token * a.dtable_ld + m.c0;
    float v[8];
    if (a.accumulate) {
        Eight<T, false> old;
        old.load(y, m.n, m.n == 8, m.step);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(sum[e], a.scale, old.at(e));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sum[e] * a.scale;
    }
    Eight<T, NT>::store(y, v, m.n, m.n == 8, m.step);
}
__device__ __forceinline__ void write_part(float* p, Mine m, const float* sum) {
    Eight<float, false>::store(p, sum, m.n, m.n == 8, m.step);
}

// A team sums a piece's rows.  part: [piece][2][cols], of the token that a piece goes on with ([0]) and of the one that
// goes on past it ([1]).
template <class T, bool NT>
__global__ void __launch_bounds__(256) embed_sum_kernel(EmbedArgs a, const Entry* __restrict__ sorted, int piece, int tx,
                                                         float* __restrict__ part) {
    const int ty = threadIdx.x >> tx, teams = 256 >> tx;
    const Mine m = mine_of<T>(a.cols, tx);
    extern __shared__ Entry entry[];  // the workgroup's, between the one before and the one after
    const int64_t first = (int64_t)block_of() * teams * piece;
    for (int k = threadIdx.x; k < teams * piece + 2; k += 256) {
        const int64_t i = first + k - 1;
        entry[k] = i >= 0 && i < a.rows ? sorted[i] : make_uint2(~0u, 0u);
    }
    __syncthreads();
    const int64_t p = (int64_t)block_of() * teams + ty, i0 = p * piece, i1 = min(a.rows, i0 + piece);
    if (i0 >= a.rows || m.n <= 0) return;
    const uint32_t vocab = (uint32_t)a.vocab;
    const auto own = [&](int64_t i) { return entry[(int)(i - first) + 1]; };
    const uint32_t before = own(i0 - 1).x, after = own(i1).x;
    float sum[8] = {};
    uint32_t token = own(i0).x;
    bool head = before == token;  // the present token began in an earlier piece
    float* mine = part + p * 2 * a.cols + m.c0;
    for (int64_t i = i0; i < i1; i += SUM_FLY) {
        Entry e[SUM_FLY];
        Eight<T, NT> x[SUM_FLY];
#pragma unroll
        for (int u = 0; u < SUM_FLY; ++u) e[u] = i + u < i1 ? own(i + u) : make_uint2(~0u, 0u);
#pragma unroll
        for (int u = 0; u < SUM_FLY; ++u)
            if (e[u].x < vocab) load_mine(x[u], (const T*)a.dout + (int64_t)e[u].y * a.dout_ld, m, a.cols);
#pragma unroll
        for (int u = 0; u < SUM_FLY; ++u) {
            if (i + u >= i1 || e[u].x >= vocab) break;
            if (e[u].x != token) {
                if (head) write_part(mine, m, sum);
                else write_row<T, NT>(a, token, m, sum);
                head = false;
                token = e[u].x;
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] = 0.f;
            }
            fit_mine(x[u], m, a.cols);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += x[u].at(k);
        }
    }
    if (token >= vocab) return;
    const bool tail = after == token;
    if (head) write_part(mine, m, sum);
    else if (tail) write_part(mine + a.cols, m, sum);
    else write_row<T, NT>(a, token, m, sum);
}

// The token that begins in a piece and goes on past it: its sums there and in the pieces after.  256 columns a
// workgroup, eight teams that take every eighth of the pieces, joined in order.
template <class T>
__global__ void __launch_bounds__(256) embed_join_kernel(EmbedArgs a, const Entry* __restrict__ sorted, int piece,
                                                          int64_t pieces, const float* __restrict__ part) {
    __shared__ float sums[8][32][9];
    const int64_t p = block_of();
    if (p + 1 >= pieces) return;
    const uint32_t token = sorted[(p + 1) * piece].x;
    if (token >= (uint32_t)a.vocab || sorted[(p + 1) * piece - 1].x != token) return;
    if (p && sorted[p * piece].x == token && sorted[p * piece - 1].x == token) return;  // it began before
    int64_t more = 0;  // pieces after p that begin with it
    for (;;) {
        const int64_t q = p + 1 + more + (threadIdx.x & 63);  // the same in every wave
        const uint64_t on = __ballot(q < pieces && sorted[q * piece].x == token);
        const int run = on == ~0ull ? 64 : __ffsll((unsigned long long)~on) - 1;
        more += run;
        if (run < 64) break;
    }
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int64_t c0 = ((int64_t)blockIdx.z * 32 + tx) * 8;
    const int n = (int)min((int64_t)8, a.cols - c0);
    float sum[8] = {};
    if (n > 0) {
#pragma unroll 4
        for (int64_t k = ty; k <= more; k += 8) {
            Eight<float, false> x;
            x.load(part + ((p + k) * 2 + (k == 0)) * a.cols + c0, n, n == 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x.at(e);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[ty][tx][e] = sum[e];
    __syncthreads();
    if (ty || n <= 0) return;
    for (int k = 1; k < 8; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += sums[k][tx][e];
    write_row<T, false>(a, token, {c0, n, 4}, sum);
}

template <class T, bool NT>
__global__ void __launch_bounds__(256) embed_zero_kernel(EmbedArgs a, Fill f) {
    fill_zeros<T, NT, 256>(a, f, (int)blockIdx.x);
}

// ------------------------------------------------------------------ few rows
// Up to 512 rows in one launch: a workgroup owns `per` tokens of the vocabulary and 128 columns, looks through all rows
// for its tokens, orders what it finds by token and row in LDS, and writes its part of dtable, zeros among it.  Sixteen
// teams of sixteen threads: a token of up to 16 rows is one team's, a longer one is shared by all and joined in order.
// A pass with the forward, bf16: 30 rows of 768 over 1000 tokens 7.8 us, 13.0 by the sort; 250 over 5000 10.1 and 15.4;
// 500 of 2048, all of one token, 20 and 15.  Where the zeros take most of the time (200 rows of 2048 over 64000 tokens
// 56 us and 46) the sort's launches write them better.
constexpr int64_t kFewRows = 512, kFewElements = int64_t(1) << 25;
bool few_rows(int64_t rows, int32_t cols, int32_t vocab) {
    return rows > 0 && rows <= kFewRows && (int64_t)vocab * cols <= kFewElements;
}
constexpr int FEW_TOKENS = 64, FEW_TEAMS = 16, FEW_ONE_TEAM = 16, FEW_PER_THREAD = (int)kFewRows / 256;

template <class T>
__global__ void __launch_bounds__(256) embed_few_kernel(EmbedArgs a, int per) {
    __shared__ __align__(16) uint32_t found[kFewRows];  // token - first and row, in the order of the rows
    __shared__ uint16_t rows_of[kFewRows];              // rows by token
    __shared__ int count[FEW_TOKENS], start[FEW_TOKENS], wave_found[4];
    __shared__ float sums[FEW_TEAMS][16][9];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, tx = tid & 15, ty = tid >> 4;
    const int64_t v0 = (int64_t)block_of() * per, c0 = (int64_t)blockIdx.z * 128 + tx * 8;
    const int tokens = (int)min((int64_t)per, a.vocab - v0), n = (int)min((int64_t)8, a.cols - c0);
    if (tokens <= 0) return;
    if (tid < FEW_TOKENS) count[tid] = 0;
    uint32_t mine[FEW_PER_THREAD];
    int hits = 0;
#pragma unroll
    for (int k = 0; k < FEW_PER_THREAD; ++k) {
        const int64_t i = tid * FEW_PER_THREAD + k;
        mine[k] = i < a.rows ? (uint32_t)a.tokens[i] - (uint32_t)v0 : ~0u;
        hits += mine[k] < (uint32_t)tokens;
    }
    const int up = wave_scan(hits);
    if (lane == 63) wave_found[wave] = up;
    __syncthreads();
    int at = up - hits, m = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) at += wave_found[w];
        m += wave_found[w];
    }
#pragma unroll
    for (int k = 0; k < FEW_PER_THREAD; ++k)
        if (mine[k] < (uint32_t)tokens) {
            found[at++] = mine[k] << 16 | (uint32_t)(tid * FEW_PER_THREAD + k);
            atomicAdd(&count[mine[k]], 1);
        }
    __syncthreads();
    if (wave == 0) start[lane] = wave_scan(count[lane]) - count[lane];
    __syncthreads();
    // an entry's place is behind the earlier ones of its token
    for (int j = tid; j < m; j += 256) {
        const uint32_t e = found[j], token = e >> 16;
        int place = start[token], q = 0;
#pragma unroll 4
        for (; q + 4 <= j; q += 4) {
            const uint4 f = *(const uint4*)&found[q];
            place += (f.x >> 16 == token) + (f.y >> 16 == token) + (f.z >> 16 == token) + (f.w >> 16 == token);
        }
        for (; q < j; ++q) place += found[q] >> 16 == token;
        rows_of[place] = (uint16_t)e;
    }
    __syncthreads();
    const auto add = [&](float* sum, int first, int last, int step) {
        for (int i = first; i < last; i += SUM_FLY * step) {
            Eight<T, false> x[SUM_FLY];
#pragma unroll
            for (int u = 0; u < SUM_FLY; ++u)
                if (i + u * step < last) x[u].load((const T*)a.dout + (int64_t)rows_of[i + u * step] * a.dout_ld + c0, n, n == 8);
#pragma unroll
            for (int u = 0; u < SUM_FLY; ++u)
                if (i + u * step < last)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += x[u].at(e);
        }
    };
    for (int r = ty; r < tokens; r += FEW_TEAMS) {
        const int rows = count[r];
        if (n <= 0 || rows > FEW_ONE_TEAM || (rows == 0 && a.accumulate)) continue;
        float sum[8] = {};
        add(sum, start[r], start[r] + rows, 1);
        write_row<T, false>(a, (uint32_t)(v0 + r), {c0, n, 4}, sum);
    }
    if (m <= FEW_ONE_TEAM) return;
    for (int r = 0; r < tokens; ++r) {
        if (count[r] <= FEW_ONE_TEAM) continue;
        float sum[8] = {};
        if (n > 0) add(sum, start[r] + ty, start[r] + count[r], FEW_TEAMS);
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[ty][tx][e] = sum[e];
        __syncthreads();
        if (ty == 0 && n > 0) {
#pragma unroll
            for (int k = 1; k < FEW_TEAMS; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += sums[k][tx][e];
            write_row<T, false>(a, (uint32_t)(v0 + r), {c0, n, 4}, sum);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ the launches
struct Room {
    int64_t sorted, other, counts, totals, part, bytes;  // offsets
    int64_t pieces;
    int tile, tiles;
};
Room room_of(int64_t rows, int32_t cols) {
    Room r{};
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t was = at;
        at += cdiv(bytes, 16) * 16;
        return was;
    };
    r.sorted = take(rows * (int64_t)sizeof(Entry));
    r.tile = tile_of(rows);
    r.tiles = (int)cdiv(rows, r.tile);
    if (rows > kCountRows) {
        r.other = take(rows * (int64_t)sizeof(Entry));
        r.counts = take((int64_t)r.tiles << MAX_BITS << 2);
        r.totals = take(int64_t(4) << MAX_BITS);
    }
    r.pieces = cdiv(rows, piece_of(rows, cols));
    r.part = take(r.pieces * 2 * cols * 4);
    r.bytes = at;
    return r;
}

template <class T, bool NT, int TILE>
fo_status sort_by_digits(const EmbedArgs& a, const Room& r, char* ws, Entry* sorted, Fill f, hipStream_t s) {
    Entry* other = (Entry*)(ws + r.other);
    int *counts = (int*)(ws + r.counts), *totals = (int*)(ws + r.totals);
    int bits = 1;
    while (bits < 31 && (int64_t(1) << bits) <= a.vocab) ++bits;  // tokens and, for the others, vocab
    const int passes = (int)cdiv(bits, MAX_BITS);
    const Entry* in = nullptr;
    Entry* to = passes % 2 ? sorted : other;
    f.of = 2 * passes;
    for (int k = 0, shift = 0; k < passes; ++k) {
        const Digit d = {shift, (int)cdiv(bits - shift, passes - k)};
        f.share = 2 * k;
        embed_digits_kernel<T, NT><<<r.tiles + f.wgs, SORT_THREADS, 0, s>>>(a, in, d, TILE, counts, r.tiles, f);
        FO_LAUNCHED();
        embed_scan_kernel<<<1 << d.bits, 64, 0, s>>>(counts, totals, r.tiles);
        FO_LAUNCHED();
        f.share = 2 * k + 1;
        embed_place_kernel<T, NT, TILE><<<r.tiles + f.wgs, SORT_THREADS, 0, s>>>(a, in, d, counts, totals, r.tiles, to, f);
        FO_LAUNCHED();
        in = to;
        to = to == sorted ? other : sorted;
        shift += d.bits;
    }
    return FO_OK;
}

template <class T, bool NT>
fo_status bwd(const EmbedArgs& a, char* ws, hipStream_t s) {
    if (few_rows(a.rows, a.cols, a.vocab)) {
        const int64_t slices = cdiv(a.cols, 128);  // about 1024 workgroups
        const int per = (int)std::min<int64_t>(FEW_TOKENS, std::max<int64_t>(1, a.vocab * slices / 1024));
        dim3 g = grid_of(cdiv(a.vocab, per));
        g.z = (unsigned)slices;
        embed_few_kernel<T><<<g, 256, 0, s>>>(a, per);
        FO_LAUNCHED();
        return FO_OK;
    }
    const Room r = room_of(a.rows, a.cols);
    Entry* sorted = (Entry*)(ws + r.sorted);
    Fill f = {a.accumulate ? 0 : (int)std::min(kFillWgs, cdiv((int64_t)a.vocab * a.cols, 8 * 256)), 0, 1};
    if (a.rows == 0) {
        embed_zero_kernel<T, NT><<<f.wgs, 256, 0, s>>>(a, f);
        FO_LAUNCHED();
        return FO_OK;
    }
    if (a.rows <= kCountRows) {
        const int wgs = (int)cdiv(a.rows, COUNT_ROWS);
        f.wgs = (int)cdiv(f.wgs, COUNT_THREADS / 256);
        embed_count_kernel<T, NT><<<wgs + f.wgs, COUNT_THREADS, 0, s>>>(a, sorted, wgs, f);
        FO_LAUNCHED();
    } else {
        const fo_status st = r.tile == 1024 ? sort_by_digits<T, NT, 1024>(a, r, ws, sorted, f, s)
                                            : sort_by_digits<T, NT, 4096>(a, r, ws, sorted, f, s);
        if (st != FO_OK) return st;
    }
    float* part = (float*)(ws + r.part);
    const int tx = team_bits(a.cols), piece = piece_of(a.rows, a.cols);
    dim3 g = grid_of(cdiv(r.pieces, 256 >> tx));
    g.z = (unsigned)cdiv(a.cols, 2048);
    embed_sum_kernel<T, NT><<<g, 256, ((256 >> tx) * piece + 2) * sizeof(Entry), s>>>(a, sorted, piece, tx, part);
    FO_LAUNCHED();
    if (r.pieces > 1) {
        g = grid_of(r.pieces - 1);
        g.z = (unsigned)cdiv(a.cols, 256);
        embed_join_kernel<T><<<g, 256, 0, s>>>(a, sorted, piece, r.pieces, part);
        FO_LAUNCHED();
    }
    return FO_OK;
}
// Gradients that no cache keeps go past the caches, in and out: 65536 rows of 2048 over
// 128000 tokens, 800 MB: 273 us a pass with the forward, 302 through them.
template <class T>
fo_status bwd_any(const EmbedArgs& a, char* ws, hipStream_t s) {
    const bool past = (a.rows + a.vocab) * a.cols * (int64_t)sizeof(T) >= kPastCaches;
    return past ? bwd<T, true>(a, ws, s) : bwd<T, false>(a, ws, s);
}

}  // namespace

fo_status launch_embed_fwd(int32_t dtype, const EmbedArgs& a, hipStream_t s) {
    return dtype == FO_DT_BF16 ? fwd<bf16_t>(a, s) : fwd<float>(a, s);
}

int64_t embed_workspace(int64_t rows, int32_t cols, int32_t vocab) { return rows && !few_rows(rows, cols, vocab) ? room_of(rows, cols).bytes : 0; }

fo_status launch_embed_bwd(int32_t dtype, const EmbedArgs& a, void* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? bwd_any<bf16_t>(a, (char*)ws, s) : bwd_any<float>(a, (char*)ws, s);
}

}  // namespace fo
