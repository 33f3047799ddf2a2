// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Lookup: bound by the rows it copies.  A thread moves 16 bytes of a row.  Outputs
// larger than the L2s together (32 MB) are written past them: 8192 rows of 6144 of a
// text 34.7 -> 24.2 us (8.3 TB/s in and out, many rows read again from a cache), 16384
// random rows 76.8 -> 68.3, 34 MB 12.2 -> 11.9.
//
// Gradient: dE[v] = scale·Σ_{tokens[n] = v} dX[n], in the order of n so that the
// same call gives the same bits: no atomics on sums.
//  * sort: the tokens' numbers n in the order of (token, n), and where each entry's
//    run starts.  A workgroup owns a range of the vocabulary and reads all tokens:
//    first counting (those below its range: where its runs begin; those in it: by
//    entry and by which of its 16 waves' shares of the tokens), then placing them.
//    No workgroup waits for another.  A token's place among equal ones in its wave's
//    64 is found from ballots of the entry's bits.
//  * reduce: blocks of sorted places; the entries that begin and end in a block are
//    written.  An entry that goes on in the next block (a frequent token, half the
//    batch's padding) leaves a float32 partial row per block; further workgroups write
//    the zeros of the entries without a token.
//  * join: the partial rows of each such entry, added in order.
// Up to 64 tokens need no sorting: few_tokens_kernel.
#include <algorithm>

#include "common.hpp"
#include "train.hpp"

namespace espace {

namespace {

__device__ __forceinline__ uint16_t to_elem(float v, uint16_t) { return (uint16_t)bf16_rne(v); }
__device__ __forceinline__ float to_elem(float v, float) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ float to_f32(float v) { return v; }

// 16 bytes of a row
template <typename E> struct Piece {
    static constexpr int W = 16 / sizeof(E);
    E v[W];
};
template <typename E>
__device__ __forceinline__ Piece<E> load_piece(const E* p) {
    return __builtin_bit_cast(Piece<E>, *reinterpret_cast<const u32x4_t*>(p));
}
// the elements of columns below C, of the W from column c on
template <typename E, bool STREAM = false>
__device__ __forceinline__ void store_piece(E* row, int64_t c, int64_t C, const Piece<E>& v) {
    if (c + Piece<E>::W <= C) {
        u32x4_t* p = reinterpret_cast<u32x4_t*>(row + c);
        if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), p);
        else *p = __builtin_bit_cast(u32x4_t, v);
    } else {
#pragma unroll
        for (int e = 0; e < Piece<E>::W; ++e)
            if (c + e < C) row[c + e] = v.v[e];
    }
}

constexpr int64_t L2_BYTES = (int64_t)32 << 20, INFINITY_CACHE_BYTES = (int64_t)256 << 20;

template <typename E, bool STREAM>
__global__ __launch_bounds__(256) void embedding_kernel(const int64_t* __restrict__ tokens, const E* __restrict__ table,
                                                        int64_t lde, E* __restrict__ X, int64_t ldx, int64_t N,
                                                        int64_t K, int64_t V, float scale) {
    constexpr int W = Piece<E>::W;
    const int64_t pieces = (K + W - 1) / W, total = N * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / pieces, c = (i - n * pieces) * W;
        const int64_t t = tokens[n];
        Piece<E> v;
        if (t >= 0 && t < V) {
            // a row is padded to 16 bytes
            v = load_piece(table + t * lde + c);
            if (scale != 1.f) {
#pragma unroll
                for (int e = 0; e < W; ++e) v.v[e] = to_elem(to_f32(v.v[e]) * scale, E());
            }
        } else {
            const float f = t < 0 ? 0.f : __builtin_nanf("");
#pragma unroll
            for (int e = 0; e < W; ++e) v.v[e] = to_elem(f, E());
        }
        store_piece<E, STREAM>(X + n * ldx, c, K, v);
    }
}

// ---- gradient ------------------------------------------------------------------

constexpr int SORT_WAVES = 16;
constexpr int SORT_BINS = 1024;           // entries per workgroup, at most

// AHEAD: groups of 64 tokens whose loads are in flight; a share of no more is read once.
template <int AHEAD>
__global__ __launch_bounds__(SORT_WAVES * 64) void sort_tokens_kernel(const int64_t* __restrict__ tokens, int N, int V,
                                                                      int bins, int bits, int* __restrict__ order,
                                                                      int* __restrict__ start) {
    __shared__ int count[SORT_WAVES][SORT_BINS];
    __shared__ int sums[SORT_WAVES];
    __shared__ int wave_total[SORT_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lo = blockIdx.x * bins;
    const int nb = V - lo < bins ? V - lo : bins;
    for (int w = 0; w < SORT_WAVES; ++w)
        for (int i = threadIdx.x; i < nb; i += SORT_WAVES * 64) count[w][i] = 0;
    __syncthreads();
    // this wave's share of the tokens, whole groups of 64
    const int groups = (N + 63) / 64, per = (groups + SORT_WAVES - 1) / SORT_WAVES;
    const int g0 = wave * per, g1 = g0 + per < groups ? g0 + per : groups;
    // entries of AHEAD groups, relative to lo; -1 for a token outside the range or this
    // wave's share
    int rel[AHEAD];
    int below = 0;
    auto load = [&](int g) {
        int64_t t[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int n = (g + u) * 64 + lane;
            t[u] = g + u < g1 && n < N ? tokens[n] : -1;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            below += t[u] >= 0 && t[u] < lo;
            rel[u] = t[u] >= lo && t[u] < lo + nb ? (int)(t[u] - lo) : -1;
        }
    };
    for (int g = g0; g < g1; g += AHEAD) {
        load(g);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (rel[u] >= 0) atomicAdd(&count[wave][rel[u]], 1);
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) below += __shfl_xor(below, m);
    if (lane == 0) sums[wave] = below;
    __syncthreads();
    // thread b: entry lo + b; its tokens in all shares, where its run starts, and
    // where each share's part of it does
    const int b = threadIdx.x;
    int own = 0;
    if (b < nb)
        for (int w = 0; w < SORT_WAVES; ++w) own += count[w][b];
    int incl = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(incl, d);
        if (lane >= d) incl += up;
    }
    if (lane == 63) wave_total[wave] = incl;
    __syncthreads();
    int at = incl - own;
    for (int w = 0; w < SORT_WAVES; ++w) {
        at += sums[w];
        if (w < wave) at += wave_total[w];
    }
    if (b < nb) {
        start[lo + b] = at;
        if (lo + b == V - 1) start[V] = at + own;
        for (int w = 0; w < SORT_WAVES; ++w) {
            const int c = count[w][b];
            count[w][b] = at;
            at += c;
        }
    }
    __syncthreads();
    for (int g = g0; g < g1; g += AHEAD) {
        if (per > AHEAD) load(g);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const bool in = rel[u] >= 0;
            unsigned long long same = __ballot(in);
            if (same == 0) continue;
            const int bin = in ? rel[u] : 0;
            // lanes with the same entry
            for (int bit = 0; bit < bits; ++bit) {
                const unsigned long long on = __ballot((bin >> bit) & 1);
                same &= ((bin >> bit) & 1) ? on : ~on;
            }
            if (in) {
                const int rank = __popcll(same & ((1ull << lane) - 1));
                const int place = count[wave][bin] + rank;
                order[place] = (g + u) * 64 + lane;
                // the last of the equal lanes moves the place on; the wave's lanes
                // have all read it (one wave, in order)
                __builtin_amdgcn_wave_barrier();
                if ((same >> lane) == 1ull) count[wave][bin] = place + 1;
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// How the rows' columns lie on a workgroup's threads: `per_row` threads (a power of
// two) of 16 bytes each, workgroup y taking the per_row · W columns from y on; so
// narrow rows leave room for several at a time.
constexpr int RUN_MOST = 32;              // sorted places of a block of runs, at most
constexpr int ZERO_GROUPS = 1 << 22;      // workgroups that write zeros, at most
constexpr int ROWS_AHEAD = 8;             // rows whose loads are in flight

// Sums of the runs in blocks of `places` sorted places, a block for every `per_row`
// threads.  A run that goes on in the next block, or comes from the one before, leaves
// its sum in the block's part 1, or 0 (one that does both: 0).  Workgroups from
// run_groups on write the zeros of the entries without a token, RUN_MOST at a time.
template <typename E, bool STREAM>
__global__ __launch_bounds__(256) void reduce_runs_kernel(const int64_t* __restrict__ tokens,
                                                          const E* __restrict__ dX, int64_t lddx, E* __restrict__ dE,
                                                          int64_t ldde, int64_t K, int V, float scale, int accumulate,
                                                          const int* __restrict__ order, const int* __restrict__ start,
                                                          float* __restrict__ part, int64_t ldpart, int run_groups,
                                                          int places, int per_row) {
    constexpr int W = Piece<E>::W;
    const int group = threadIdx.x / per_row, groups = 256 / per_row;
    const int64_t c = ((int64_t)blockIdx.y * per_row + threadIdx.x % per_row) * W;
    if ((int)blockIdx.x >= run_groups) {
        const int lane = threadIdx.x & 63;
        Piece<E> z;
#pragma unroll
        for (int e = 0; e < W; ++e) z.v[e] = to_elem(0.f, E());
        for (int64_t v0 = ((int)blockIdx.x - run_groups) * (int64_t)RUN_MOST; v0 < V;
             v0 += ((int)gridDim.x - run_groups) * (int64_t)RUN_MOST) {
            // one bit an entry, in every wave
            const int64_t mine = v0 + (lane < RUN_MOST ? lane : RUN_MOST - 1);
            const bool none = lane < RUN_MOST && mine < V && start[mine] == start[mine + 1];
            const unsigned long long empty = __ballot(none);
            if (c < K)
                for (int k = group; k < RUN_MOST; k += groups)
                    if ((empty >> k) & 1) store_piece<E, STREAM>(dE + (v0 + k) * ldde, c, K, z);
        }
        return;
    }
    // rows of the workgroup's places, and the entries of those and their neighbours
    // (-1 before the first and past the last)
    __shared__ int row[256 / 8 * RUN_MOST], entry[256 / 8 * RUN_MOST + 2];
    const int total = start[V];
    const int all = groups * places, first = blockIdx.x * all;
    for (int i = threadIdx.x; i < all + 2; i += 256) {
        const int p = first + i - 1;
        int n = -1, v = -1;
        if (p >= 0 && p < total) {
            n = order[p];
            v = (int)tokens[n];
        }
        entry[i] = v;
        if (i >= 1 && i <= all) row[i - 1] = n;
    }
    __syncthreads();
    const int q0 = group * places;
    const int np = min(places, total - first - q0);
    if (np <= 0 || c >= K) return;
    const int block = blockIdx.x * groups + group;
    float sum[W];
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e] = 0.f;
    bool from_before = entry[q0] == entry[q0 + 1];
    for (int q = 0; q < np; q += ROWS_AHEAD) {
        Piece<E> x[ROWS_AHEAD];
#pragma unroll
        for (int u = 0; u < ROWS_AHEAD; ++u)
            x[u] = load_piece(dX + (int64_t)row[q0 + min(q + u, np - 1)] * lddx + c);
#pragma unroll
        for (int u = 0; u < ROWS_AHEAD; ++u) {
            if (q + u >= np) break;
#pragma unroll
            for (int e = 0; e < W; ++e) sum[e] += to_f32(x[u].v[e]);
            const int v = entry[q0 + q + u + 1];
            const bool goes_on = entry[q0 + q + u + 2] == v;
            if (goes_on && q + u + 1 < np) continue;
            // the run's last place in this block
            if (!from_before && !goes_on) {
                E* out = dE + (int64_t)v * ldde;
                Piece<E> o;
                if (accumulate) o = load_piece(out + c);
#pragma unroll
                for (int e = 0; e < W; ++e)
                    o.v[e] = to_elem(accumulate ? to_f32(o.v[e]) + scale * sum[e] : scale * sum[e], E());
                store_piece(out, c, K, o);
            } else {
                float* o = part + ((int64_t)block * 2 + (from_before ? 0 : 1)) * ldpart + c;
#pragma unroll
                for (int e = 0; e < W; e += 4)
                    *reinterpret_cast<f32x4_t*>(o + e) = f32x4_t{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
            }
            from_before = false;
#pragma unroll
            for (int e = 0; e < W; ++e) sum[e] = 0.f;
        }
    }
}

// The entry whose run starts in block blockIdx.x and goes on in the next ones: each
// per_row threads add a contiguous share of its parts, in order; the shares are added
// in order through LDS.
constexpr int JOIN_THREADS = 1024;

template <typename E>
__global__ __launch_bounds__(JOIN_THREADS) void join_runs_kernel(const int64_t* __restrict__ tokens,
                                                                 E* __restrict__ dE, int64_t ldde, int64_t K, int V,
                                                                 float scale, int accumulate,
                                                                 const int* __restrict__ order,
                                                                 const int* __restrict__ start,
                                                                 const float* __restrict__ part, int64_t ldpart,
                                                                 int places, int per_row) {
    constexpr int W = Piece<E>::W;
    __shared__ float shares[JOIN_THREADS * W];
    const int p1 = ((int)blockIdx.x + 1) * places;
    if (p1 >= start[V]) return;
    const int v = (int)tokens[order[p1 - 1]];
    const int s = start[v], t = start[v + 1];
    if (s < p1 - places || t <= p1) return;
    const int group = threadIdx.x / per_row, groups = JOIN_THREADS / per_row;
    const int64_t c = ((int64_t)blockIdx.y * per_row + threadIdx.x % per_row) * W;
    // part 1 of this block, part 0 of the next ones
    const int parts = (t - 1) / places - (int)blockIdx.x + 1;
    const int share = (parts + groups - 1) / groups;
    const int k0 = group * share, k1 = min(k0 + share, parts);
    float sum[W];
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e] = 0.f;
    if (c < K)
        for (int k = k0; k < k1; k += ROWS_AHEAD) {
            f32x4_t x[ROWS_AHEAD][W / 4];
#pragma unroll
            for (int u = 0; u < ROWS_AHEAD; ++u) {
                const int q = min(k + u, k1 - 1);
                const float* p = part + (((int64_t)blockIdx.x + q) * 2 + (q == 0 ? 1 : 0)) * ldpart + c;
#pragma unroll
                for (int e = 0; e < W / 4; ++e) x[u][e] = reinterpret_cast<const f32x4_t*>(p)[e];
            }
#pragma unroll
            for (int u = 0; u < ROWS_AHEAD; ++u)
                if (k + u < k1)
#pragma unroll
                    for (int e = 0; e < W; ++e) sum[e] += x[u][e / 4][e % 4];
        }
#pragma unroll
    for (int e = 0; e < W; ++e) shares[threadIdx.x * W + e] = sum[e];
    __syncthreads();
    if (group != 0 || c >= K) return;
    for (int g = 1; g < groups && g * share < parts; ++g)
#pragma unroll
        for (int e = 0; e < W; ++e) sum[e] += shares[(g * per_row + threadIdx.x) * W + e];
    E* out = dE + (int64_t)v * ldde;
    Piece<E> o;
    if (accumulate) o = load_piece(out + c);
#pragma unroll
    for (int e = 0; e < W; ++e)
        o.v[e] = to_elem(accumulate ? to_f32(o.v[e]) + scale * sum[e] : scale * sum[e], E());
    store_piece(out, c, K, o);
}

// A few tokens in one launch: a workgroup of RUN_MOST entries notes which tokens are of
// each, one bit a token, writes the zeros of those without, and then each per_row threads
// add an entry's rows in the tokens' order.
constexpr int FEW_TOKENS = 64;

template <typename E, bool STREAM>
__global__ __launch_bounds__(256) void few_tokens_kernel(const int64_t* __restrict__ tokens, int N,
                                                         const E* __restrict__ dX, int64_t lddx, E* __restrict__ dE,
                                                         int64_t ldde, int64_t K, int V, float scale, int accumulate,
                                                         int per_row) {
    constexpr int W = Piece<E>::W;
    static_assert(FEW_TOKENS == 64 && RUN_MOST <= 64, "a bit a token");
    __shared__ unsigned long long of[RUN_MOST];
    const int v0 = blockIdx.x * RUN_MOST, lane = threadIdx.x & 63;
    if (threadIdx.x < RUN_MOST) of[threadIdx.x] = 0;
    const int64_t t = (int)threadIdx.x < N ? tokens[threadIdx.x] : -1;
    __syncthreads();
    if (t >= v0 && t < v0 + RUN_MOST && t < V) atomicOr(&of[(int)t - v0], 1ull << threadIdx.x);
    __syncthreads();
    const int group = threadIdx.x / per_row, groups = 256 / per_row;
    const int64_t c = ((int64_t)blockIdx.y * per_row + threadIdx.x % per_row) * W;
    // one bit an entry, in every wave
    const unsigned long long named = __ballot(lane < RUN_MOST && of[lane < RUN_MOST ? lane : 0] != 0);
    if (c >= K) return;
    if (!accumulate) {
        Piece<E> z;
#pragma unroll
        for (int e = 0; e < W; ++e) z.v[e] = to_elem(0.f, E());
        for (int k = group; k < RUN_MOST && v0 + k < V; k += groups)
            if (!((named >> k) & 1)) store_piece<E, STREAM>(dE + (int64_t)(v0 + k) * ldde, c, K, z);
    }
    for (int k = group; k < RUN_MOST; k += groups) {
        if (!((named >> k) & 1)) continue;
        unsigned long long left = of[k];
        E* out = dE + (int64_t)(v0 + k) * ldde;
        float sum[W];
#pragma unroll
        for (int e = 0; e < W; ++e) sum[e] = 0.f;
        while (left) {
            Piece<E> x[ROWS_AHEAD];
            bool there[ROWS_AHEAD];
#pragma unroll
            for (int u = 0; u < ROWS_AHEAD; ++u) {
                there[u] = left != 0;
                if (there[u]) x[u] = load_piece(dX + (int64_t)(__ffsll(left) - 1) * lddx + c);
                left &= left - 1;
            }
#pragma unroll
            for (int u = 0; u < ROWS_AHEAD; ++u)
                if (there[u])
#pragma unroll
                    for (int e = 0; e < W; ++e) sum[e] += to_f32(x[u].v[e]);
        }
        Piece<E> o;
        if (accumulate) o = load_piece(out + c);
#pragma unroll
        for (int e = 0; e < W; ++e)
            o.v[e] = to_elem(accumulate ? to_f32(o.v[e]) + scale * sum[e] : scale * sum[e], E());
        store_piece(out, c, K, o);
    }
}

// Sorted places of a block: the most that leave 512 workgroups, two a CU.
int run_places(int64_t N, int64_t K, int per_row, int W) {
    const int64_t chunks = (K + (int64_t)per_row * W - 1) / ((int64_t)per_row * W);
    int places = RUN_MOST;
    while (places > 8 && (N + places - 1) / places * per_row / 256 * chunks < 512) places /= 2;
    return places;
}

// Threads of a row: the power of two from 8 to 256 that holds K in 16-byte pieces.
int row_threads(int64_t K, int W) {
    int t = 8;
    while (t < 256 && (int64_t)t * W < K) t *= 2;
    return t;
}

struct GradLayout {
    size_t order, start, part, total;
    int64_t ldpart;
};

GradLayout grad_layout(int64_t N, int64_t K, int64_t V) {
    GradLayout b{};
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    size_t o = 0;
    b.order = o;
    o = up(o + (size_t)N * 4);
    b.start = o;
    o = up(o + (size_t)(V + 1) * 4);
    b.ldpart = (K + 7) / 8 * 8;
    b.part = o;
    // for either type's blocks
    const int64_t places = std::min(run_places(N, K, row_threads(K, 4), 4), run_places(N, K, row_threads(K, 8), 8));
    o = up(o + (size_t)((N + places - 1) / places) * 2 * b.ldpart * 4);
    b.total = o;
    return b;
}

template <typename E>
hipError_t launch_backward(const int64_t* tokens, const E* dX, int64_t lddx, E* dE, int64_t ldde, int64_t N, int64_t K,
                           int64_t V, float scale, bool accumulate, void* workspace, hipStream_t stream) {
    constexpr int W = Piece<E>::W;
    const int per_row = row_threads(K, W), groups = 256 / per_row;
    const unsigned chunks = (unsigned)((K + per_row * W - 1) / (per_row * W));
    // Zero rows go past the caches where dE and dX do not fit the last one.  4096 tokens of
    // a text on 32000 x 4096 73.5 -> 60 us, random ones on 50000 x 4096 100 -> 81; but 34
    // tokens on 25480 x 3584 32 -> 44.
    const bool stream_rows = (V + N) * K * (int64_t)sizeof(E) > INFINITY_CACHE_BYTES;
    // One launch for a few tokens, three -> one, us (of text; all one entry): 64 x 128 on 500
    // 16.3 -> 10.1 (16.7 -> 13.3), 16 x 4096 on 32000 40.9 -> 37.8 (42.7 -> 37.8), 64 x 8192 on
    // 50000 172 -> 168 (173 -> 170); 128 tokens of one entry would take longer (17 -> 25).
    // An accumulated gradient has to look at every entry of the table, so not of large ones.
    if (N <= FEW_TOKENS && V <= (accumulate ? 1 << 17 : 1 << 25)) {
        const dim3 grid((unsigned)((V + RUN_MOST - 1) / RUN_MOST), chunks);
        if (stream_rows)
            hipLaunchKernelGGL((few_tokens_kernel<E, true>), grid, dim3(256), 0, stream, tokens, (int)N, dX, lddx, dE,
                               ldde, K, (int)V, scale, accumulate ? 1 : 0, per_row);
        else
            hipLaunchKernelGGL((few_tokens_kernel<E, false>), grid, dim3(256), 0, stream, tokens, (int)N, dX, lddx, dE,
                               ldde, K, (int)V, scale, accumulate ? 1 : 0, per_row);
        return hipGetLastError();
    }
    const GradLayout b = grad_layout(N, K, V);
    char* ws = static_cast<char*>(workspace);
    int* order = (int*)(ws + b.order);
    int* start = (int*)(ws + b.start);
    float* part = (float*)(ws + b.part);
    // 256 workgroups of equal ranges, or more of SORT_BINS entries
    const int64_t bins = (V + 255) / 256 < SORT_BINS ? (V + 255) / 256 : SORT_BINS;
    int bits = 0;
    while (((int64_t)1 << bits) < bins) ++bits;
    const dim3 ranges((unsigned)((V + bins - 1) / bins)), threads(SORT_WAVES * 64);
    // Shares of up to 8 groups of tokens, or 24, stay in registers between the two passes
    // (read again -> kept: 8192 tokens 12.2 -> 10.5 us, 20011 19.0 -> 17.0); longer ones
    // are read again, 8 groups at a time.
    if (N > SORT_WAVES * 64 * 8 && N <= SORT_WAVES * 64 * 24)
        hipLaunchKernelGGL(sort_tokens_kernel<24>, ranges, threads, 0, stream, tokens, (int)N, (int)V, (int)bins, bits,
                           order, start);
    else
        hipLaunchKernelGGL(sort_tokens_kernel<8>, ranges, threads, 0, stream, tokens, (int)N, (int)V, (int)bins, bits,
                           order, start);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int places = run_places(N, K, per_row, W);
    const int64_t blocks = (N + places - 1) / places, runs = (blocks + groups - 1) / groups;
    // (a launch has less than 2^32 threads)
    const int64_t zeros = accumulate ? 0 : std::min<int64_t>((V + RUN_MOST - 1) / RUN_MOST, ZERO_GROUPS / chunks + 1);
    const dim3 grid((unsigned)(runs + zeros), chunks);
    if (stream_rows)
        hipLaunchKernelGGL((reduce_runs_kernel<E, true>), grid, dim3(256), 0, stream, tokens, dX, lddx, dE, ldde, K,
                           (int)V, scale, accumulate ? 1 : 0, order, start, part, b.ldpart, (int)runs, places, per_row);
    else
        hipLaunchKernelGGL((reduce_runs_kernel<E, false>), grid, dim3(256), 0, stream, tokens, dX, lddx, dE, ldde, K,
                           (int)V, scale, accumulate ? 1 : 0, order, start, part, b.ldpart, (int)runs, places, per_row);
    e = hipGetLastError();
    if (e != hipSuccess || blocks < 2) return e;
    hipLaunchKernelGGL(join_runs_kernel<E>, dim3((unsigned)(blocks - 1), chunks), dim3(JOIN_THREADS), 0, stream, tokens,
                       dE, ldde, K, (int)V, scale, accumulate ? 1 : 0, order, start, part, b.ldpart, places, per_row);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const int64_t* tokens, const void* E, int64_t lde, void* X, int64_t ldx, int64_t N,
                            int64_t K, int64_t V, float scale, bool f32, hipStream_t stream) {
    const int64_t total = N * ((K + (f32 ? 3 : 7)) / (f32 ? 4 : 8));
    const int64_t want = (total + 255) / 256;
    const dim3 grid((unsigned)(want < 65536 ? want : 65536)), block(256);
    const bool past = N * K * (f32 ? 4 : 2) > L2_BYTES;
#define LOOKUP(T, S)                                                                                              \
    hipLaunchKernelGGL((embedding_kernel<T, S>), grid, block, 0, stream, tokens, (const T*)E, lde, (T*)X, ldx, N, K, V, \
                       scale)
    if (f32 && past) LOOKUP(float, true);
    else if (f32) LOOKUP(float, false);
    else if (past) LOOKUP(uint16_t, true);
    else LOOKUP(uint16_t, false);
#undef LOOKUP
    return hipGetLastError();
}

size_t embedding_workspace_bytes(int64_t N, int64_t K, int64_t V) { return grad_layout(N, K, V).total; }

hipError_t launch_embedding_backward(const int64_t* tokens, const void* dX, int64_t lddx, void* dE, int64_t ldde,
                                     int64_t N, int64_t K, int64_t V, float scale, bool accumulate, bool f32,
                                     void* workspace, hipStream_t stream) {
    if (f32)
        return launch_backward<float>(tokens, (const float*)dX, lddx, (float*)dE, ldde, N, K, V, scale, accumulate,
                                      workspace, stream);
    return launch_backward<uint16_t>(tokens, (const uint16_t*)dX, lddx, (uint16_t*)dE, ldde, N, K, V, scale,
                                     accumulate, workspace, stream);
}

}  // namespace espace
