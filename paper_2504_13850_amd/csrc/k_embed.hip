// Embedding: rows of a table by tokens, and the table's gradient.
//
// Bound by HBM: the named rows in and out; the gradient's rows in and the table's
// gradient out, most of it zeros where the batch is small beside the vocabulary.
//
// The gradient's sums have to come in the same order every time, so there are no
// atomics on them: the rows are sorted by token (stable), the sorted list is cut
// into pieces of equal length whatever the tokens are, a team of threads sums a
// piece's rows and writes each token that begins and ends inside it, and the sums of
// tokens that cross pieces are joined by a last launch.  The zeros are written beside
// the first launch of the sort, which leaves the memory idle.
#include <algorithm>

#include "lm.h"
#include "row8.h"

namespace fo {
namespace {

// A team of 2^tx threads takes 8 << tx columns of a row (all of them, up to 2048), 256 >> tx teams a workgroup.
int team_bits(int32_t cols) {
    int tx = 0;
    while (tx < 8 && (8 << tx) < cols) ++tx;
    return tx;
}

constexpr int64_t kPastCaches = int64_t(256) << 20;

// ------------------------------------------------------------------ forward
constexpr int FWD_FLY = 4;  // rows of a team in flight

template <class T, bool NT>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmbedArgs a, int tx) {
    const int ty = threadIdx.x >> tx, teams = 256 >> tx;
    const int64_t c0 = ((int64_t)blockIdx.z * 256 + (threadIdx.x & ((1 << tx) - 1))) * 8;
    const int n = (int)min((int64_t)8, a.cols - c0);
    const int64_t r0 = (int64_t)block_of() * teams * FWD_FLY + ty;
    if (n <= 0) return;
    int token[FWD_FLY];
    Eight<T, false> x[FWD_FLY];
#pragma unroll
    for (int k = 0; k < FWD_FLY; ++k) token[k] = r0 + k * teams < a.rows ? a.tokens[r0 + k * teams] : -1;
#pragma unroll
    for (int k = 0; k < FWD_FLY; ++k) {
        if ((uint32_t)token[k] < (uint32_t)a.vocab)
            x[k].load((const T*)a.table + token[k] * a.table_ld + c0, n, n == 8);
        else
            x[k] = {};
    }
#pragma unroll
    for (int k = 0; k < FWD_FLY; ++k) {
        if (r0 + k * teams >= a.rows) continue;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[k].at(e) * a.scale;
        if ((uint32_t)token[k] >= (uint32_t)a.vocab)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = 0.f;
        Eight<T, NT>::store((T*)a.out + (r0 + k * teams) * a.out_ld + c0, y, n, n == 8);
    }
}

template <class T>
fo_status fwd(const EmbedArgs& a, hipStream_t s) {
    const int tx = team_bits(a.cols);
    dim3 g = grid_of(cdiv(a.rows, (256 >> tx) * FWD_FLY));
    g.z = (unsigned)cdiv(a.cols, 2048);
    // past the caches: see Eight
    if (a.rows * a.cols * (int64_t)sizeof(T) > kPastCaches) embed_fwd_kernel<T, true><<<g, 256, 0, s>>>(a, tx);
    else embed_fwd_kernel<T, false><<<g, 256, 0, s>>>(a, tx);
    FO_LAUNCHED();
    return FO_OK;
}

// ------------------------------------------------------------------ zeros
constexpr int64_t kFillWgs = 1024;

// Workgroup `id` of `of` writes zeros to its share of dtable.
template <class T>
__device__ void fill_zeros(const EmbedArgs& a, int64_t id, int64_t of, int threads) {
    const float zero[8] = {};
    const int64_t step = of * threads;
    T* y = (T*)a.dtable;
    if (a.dtable_ld == a.cols) {  // one run
        const int64_t all = (int64_t)a.vocab * a.cols, chunks = (all + 7) / 8;
        for (int64_t c = id * threads + threadIdx.x; c < chunks; c += step) {
            const int n = (int)min((int64_t)8, all - c * 8);
            Eight<T, false>::store(y + c * 8, zero, n, n == 8);
        }
        return;
    }
    for (int64_t v = id; v < a.vocab; v += of)
        for (int64_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += threads * 8) {
            const int n = (int)min((int64_t)8, a.cols - c0);
            Eight<T, false>::store(y + v * a.dtable_ld + c0, zero, n, n == 8);
        }
}

// ------------------------------------------------------------------ sort
// An entry of the sorted list: token (as unsigned: those outside the vocabulary come last) and row.
typedef uint2 Entry;

// Few rows: an entry's place is the number of entries that come before it, counted.
// 64 rows a workgroup, 16 waves with a sixteenth of the tokens each; n^2 comparisons,
// two instructions each: 8192 rows 3.4 us of the vector units, beside the zeros.
constexpr int64_t kCountRows = 8192;
constexpr int COUNT_WAVES = 16;

template <class T>
__global__ void __launch_bounds__(64 * COUNT_WAVES) embed_count_kernel(EmbedArgs a, Entry* __restrict__ out, int wgs, int fill) {
    if ((int)blockIdx.x >= wgs) {
        fill_zeros<T>(a, blockIdx.x - wgs, fill, 64 * COUNT_WAVES);
        return;
    }
    __shared__ int part[COUNT_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = (int)a.rows;
    const int first = blockIdx.x * 64, i = first + lane;
    const uint32_t* __restrict__ tok = (const uint32_t*)a.tokens;
    const uint32_t mine = i < n ? tok[i] : 0u;
    const int each = (n + COUNT_WAVES - 1) / COUNT_WAVES, lo = min(n, wave * each), hi = min(n, lo + each);
    int before = 0;
    // rows of earlier workgroups come first on a tie, rows of later ones do not
    const int own = min(max(first, lo), hi), past = min(max(first + 64, lo), hi);
#pragma unroll 16
    for (int j = lo; j < own; ++j) before += tok[j] <= mine;
    for (int j = own; j < past; ++j) before += tok[j] < mine || (tok[j] == mine && j < i);
#pragma unroll 16
    for (int j = past; j < hi; ++j) before += tok[j] < mine;
    part[wave][lane] = before;
    __syncthreads();
    if (wave || i >= n) return;
    for (int k = 1; k < COUNT_WAVES; ++k) before += part[k][lane];
    out[before] = make_uint2(mine, (uint32_t)i);
}

// More rows: digits of up to ten bits, lowest first.  A tile is TILE entries, a wave
// has a run of them.  counts: [digit][tile].
constexpr int TILE = 4096, SORT_THREADS = 256, SORT_WAVES = SORT_THREADS / 64, PER_THREAD = TILE / SORT_THREADS;
constexpr int MAX_BITS = 10;

struct Digit {
    int shift, bits;
};
__device__ __forceinline__ Entry entry_of(const EmbedArgs& a, const Entry* in, int64_t i) {
    return in ? in[i] : make_uint2(min((uint32_t)a.tokens[i], (uint32_t)a.vocab), (uint32_t)i);
}

template <class T>
__global__ void __launch_bounds__(SORT_THREADS) embed_digits_kernel(EmbedArgs a, const Entry* __restrict__ in, Digit d,
                                                                     int* __restrict__ counts, int tiles, int fill) {
    if ((int)blockIdx.x >= tiles) {
        fill_zeros<T>(a, blockIdx.x - tiles, fill, SORT_THREADS);
        return;
    }
    __shared__ int sum[1 << MAX_BITS];
    for (int k = threadIdx.x; k < 1 << d.bits; k += SORT_THREADS) sum[k] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * TILE;
#pragma unroll
    for (int k = 0; k < PER_THREAD; ++k) {
        const int64_t i = i0 + k * SORT_THREADS + threadIdx.x;
        if (i < a.rows) atomicAdd(&sum[entry_of(a, in, i).x >> d.shift & ((1u << d.bits) - 1u)], 1);
    }
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

__global__ void __launch_bounds__(SORT_THREADS) embed_place_kernel(EmbedArgs a, const Entry* __restrict__ in, Digit d,
                                                                    const int* __restrict__ counts, const int* __restrict__ totals,
                                                                    int tiles, Entry* __restrict__ out) {
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
// Entries of a piece: short pieces where rows are few, so that they fill the chip.
int piece_of(int64_t rows) { return rows <= 16384 ? 16 : 32; }
constexpr int SUM_FLY = 8;  // rows of a team in flight

template <class T>
__device__ __forceinline__ void write_row(const EmbedArgs& a, uint32_t token, int64_t c0, int n, const float* sum) {
    T* y = (T*)a.dtable + token * a.dtable_ld + c0;
    float v[8];
    if (a.accumulate) {
        Eight<T, false> old;
        old.load(y, n, n == 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(sum[e], a.scale, old.at(e));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sum[e] * a.scale;
    }
    Eight<T, false>::store(y, v, n, n == 8);
}
__device__ __forceinline__ void write_part(float* p, int n, const float* sum) {
    Eight<float, false>::store(p, sum, n, n == 8);
}

// A team sums a piece's rows.  part: [piece][2][cols], of the token that a piece goes on with ([0]) and of the one that
// goes on past it ([1]).
template <class T>
__global__ void __launch_bounds__(256) embed_sum_kernel(EmbedArgs a, const Entry* __restrict__ sorted, int piece, int tx,
                                                         float* __restrict__ part) {
    const int ty = threadIdx.x >> tx, teams = 256 >> tx;
    const int64_t c0 = ((int64_t)blockIdx.z * 256 + (threadIdx.x & ((1 << tx) - 1))) * 8;
    const int n = (int)min((int64_t)8, a.cols - c0);
    const int64_t p = (int64_t)block_of() * teams + ty, i0 = p * piece, i1 = min(a.rows, i0 + piece);
    if (i0 >= a.rows || n <= 0) return;
    const uint32_t vocab = (uint32_t)a.vocab;
    const uint32_t before = i0 ? sorted[i0 - 1].x : ~0u, after = i1 < a.rows ? sorted[i1].x : ~0u;
    float sum[8] = {};
    uint32_t token = sorted[i0].x;
    bool head = i0 && before == token;  // the present token began in an earlier piece
    float* mine = part + p * 2 * a.cols + c0;
    for (int64_t i = i0; i < i1; i += SUM_FLY) {
        Entry e[SUM_FLY];
        Eight<T, false> x[SUM_FLY];
#pragma unroll
        for (int u = 0; u < SUM_FLY; ++u) e[u] = i + u < i1 ? sorted[i + u] : make_uint2(~0u, 0u);
#pragma unroll
        for (int u = 0; u < SUM_FLY; ++u)
            if (e[u].x < vocab) x[u].load((const T*)a.dout + (int64_t)e[u].y * a.dout_ld + c0, n, n == 8);
#pragma unroll
        for (int u = 0; u < SUM_FLY; ++u) {
            if (i + u >= i1 || e[u].x >= vocab) break;
            if (e[u].x != token) {
                if (head) write_part(mine, n, sum);
                else write_row<T>(a, token, c0, n, sum);
                head = false;
                token = e[u].x;
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += x[u].at(k);
        }
    }
    if (token >= vocab) return;
    const bool tail = i1 < a.rows && after == token;
    if (head) write_part(mine, n, sum);
    else if (tail) write_part(mine + a.cols, n, sum);
    else write_row<T>(a, token, c0, n, sum);
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
    write_row<T>(a, token, c0, n, sum);
}

template <class T>
__global__ void __launch_bounds__(256) embed_zero_kernel(EmbedArgs a) {
    fill_zeros<T>(a, blockIdx.x, gridDim.x, 256);
}

// ------------------------------------------------------------------ the launches
struct Room {
    int64_t sorted, other, counts, totals, part, bytes;  // offsets
    int64_t pieces;
    int tiles;
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
    r.tiles = (int)cdiv(rows, TILE);
    if (rows > kCountRows) {
        r.other = take(rows * (int64_t)sizeof(Entry));
        r.counts = take((int64_t)r.tiles << MAX_BITS << 2);
        r.totals = take(int64_t(4) << MAX_BITS);
    }
    r.pieces = cdiv(rows, piece_of(rows));
    r.part = take(r.pieces * 2 * cols * 4);
    r.bytes = at;
    return r;
}

template <class T>
fo_status bwd(const EmbedArgs& a, char* ws, hipStream_t s) {
    const int64_t zeros = cdiv((int64_t)a.vocab * a.cols, 8);
    const auto fill_wgs = [&](int threads) { return a.accumulate ? 0 : (int)std::min(kFillWgs, cdiv(zeros, threads)); };
    if (a.rows == 0) {
        embed_zero_kernel<T><<<fill_wgs(256), 256, 0, s>>>(a);
        FO_LAUNCHED();
        return FO_OK;
    }
    const Room r = room_of(a.rows, a.cols);
    Entry *sorted = (Entry*)(ws + r.sorted), *other = (Entry*)(ws + r.other);
    if (a.rows <= kCountRows) {
        const int wgs = (int)cdiv(a.rows, 64), fill = fill_wgs(64 * COUNT_WAVES);
        embed_count_kernel<T><<<wgs + fill, 64 * COUNT_WAVES, 0, s>>>(a, sorted, wgs, fill);
        FO_LAUNCHED();
    } else {
        int *counts = (int*)(ws + r.counts), *totals = (int*)(ws + r.totals);
        int bits = 1;
        while (bits < 31 && (int64_t(1) << bits) <= a.vocab) ++bits;  // tokens and, for the others, vocab
        const int passes = (int)cdiv(bits, MAX_BITS);
        const Entry* in = nullptr;
        Entry* to = passes % 2 ? sorted : other;
        for (int k = 0, shift = 0; k < passes; ++k) {
            const Digit d = {shift, (int)cdiv(bits - shift, passes - k)};
            const int fill = k ? 0 : fill_wgs(SORT_THREADS);
            embed_digits_kernel<T><<<r.tiles + fill, SORT_THREADS, 0, s>>>(a, in, d, counts, r.tiles, fill);
            FO_LAUNCHED();
            embed_scan_kernel<<<1 << d.bits, 64, 0, s>>>(counts, totals, r.tiles);
            FO_LAUNCHED();
            embed_place_kernel<<<r.tiles, SORT_THREADS, 0, s>>>(a, in, d, counts, totals, r.tiles, to);
            FO_LAUNCHED();
            in = to;
            to = to == sorted ? other : sorted;
            shift += d.bits;
        }
    }
    float* part = (float*)(ws + r.part);
    const int tx = team_bits(a.cols), piece = piece_of(a.rows);
    dim3 g = grid_of(cdiv(r.pieces, 256 >> tx));
    g.z = (unsigned)cdiv(a.cols, 2048);
    embed_sum_kernel<T><<<g, 256, 0, s>>>(a, sorted, piece, tx, part);
    FO_LAUNCHED();
    if (r.pieces > 1) {
        g = grid_of(r.pieces - 1);
        g.z = (unsigned)cdiv(a.cols, 256);
        embed_join_kernel<T><<<g, 256, 0, s>>>(a, sorted, piece, r.pieces, part);
        FO_LAUNCHED();
    }
    return FO_OK;
}

}  // namespace

fo_status launch_embed_fwd(int32_t dtype, const EmbedArgs& a, hipStream_t s) {
    return dtype == FO_DT_BF16 ? fwd<bf16_t>(a, s) : fwd<float>(a, s);
}

int64_t embed_workspace(int64_t rows, int32_t cols, int32_t vocab) { return rows ? room_of(rows, cols).bytes : 0; }

fo_status launch_embed_bwd(int32_t dtype, const EmbedArgs& a, void* ws, hipStream_t s) {
    return dtype == FO_DT_BF16 ? bwd<bf16_t>(a, (char*)ws, s) : bwd<float>(a, (char*)ws, s);
}

}  // namespace fo
