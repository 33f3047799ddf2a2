// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Lookup: bound by the rows it copies.  A thread moves 16 bytes of a row.
//
// Gradient: dE[v] = scale·Σ_{tokens[n] = v} dX[n], in the order of n so that the
// same call gives the same bits: no atomics on sums.
//  * sort: the tokens' numbers n in the order of (token, n), and where each entry's
//    run starts.  A workgroup owns a range of the vocabulary and reads all tokens:
//    first counting (those below its range: where its runs begin; those in it: by
//    entry and by which of its 16 waves' shares of the tokens), then placing them.
//    No workgroup waits for another.  A token's place among equal ones in its wave's
//    64 is found from ballots of the entry's bits.
//  * reduce: a workgroup sums RUN_BLOCK sorted places, and writes the rows of the
//    entries that begin and end there.  An entry that goes on in the next block (a
//    frequent token, half the batch's padding) leaves a float32 partial row per
//    block; further workgroups write the zeros of the entries without a token.
//  * join: the partial rows of each such entry, added in order.
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
template <typename E>
__device__ __forceinline__ void store_piece(E* row, int64_t c, int64_t C, const Piece<E>& v) {
    if (c + Piece<E>::W <= C) {
        *reinterpret_cast<u32x4_t*>(row + c) = __builtin_bit_cast(u32x4_t, v);
    } else {
#pragma unroll
        for (int e = 0; e < Piece<E>::W; ++e)
            if (c + e < C) row[c + e] = v.v[e];
    }
}

template <typename E>
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
        store_piece(X + n * ldx, c, K, v);
    }
}

// ---- gradient ------------------------------------------------------------------

constexpr int SORT_WAVES = 16;
constexpr int SORT_BINS = 1024;           // entries per workgroup, at most
constexpr int RUN_BLOCK = 32;             // sorted places per workgroup

__global__ __launch_bounds__(SORT_WAVES * 64) void sort_tokens_kernel(const int64_t* __restrict__ tokens, int N, int V,
                                                                      int bins, int* __restrict__ order,
                                                                      int* __restrict__ start) {
    __shared__ int count[SORT_WAVES][SORT_BINS];
    __shared__ int sums[SORT_WAVES];
    __shared__ int wave_total[SORT_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lo = blockIdx.x * bins;
    const int nb = V - lo < bins ? V - lo : bins;
    for (int i = threadIdx.x; i < SORT_WAVES * SORT_BINS; i += SORT_WAVES * 64) (&count[0][0])[i] = 0;
    __syncthreads();
    // this wave's share of the tokens, whole groups of 64
    const int groups = (N + 63) / 64, per = (groups + SORT_WAVES - 1) / SORT_WAVES;
    const int g0 = wave * per, g1 = g0 + per < groups ? g0 + per : groups;
    int below = 0;
    for (int g = g0; g < g1; ++g) {
        const int n = g * 64 + lane;
        const int64_t t = n < N ? tokens[n] : -1;
        if (t >= 0 && t < lo) ++below;
        if (t >= lo && t < lo + nb) atomicAdd(&count[wave][(int)t - lo], 1);
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
    for (int g = g0; g < g1; ++g) {
        const int n = g * 64 + lane;
        const int64_t t = n < N ? tokens[n] : -1;
        const bool in = t >= lo && t < lo + nb;
        unsigned long long same = __ballot(in);
        if (same == 0) continue;
        const int bin = in ? (int)t - lo : 0;
        // lanes with the same entry
#pragma unroll
        for (int bit = 0; bit < 10; ++bit) {
            const unsigned long long on = __ballot((bin >> bit) & 1);
            same &= ((bin >> bit) & 1) ? on : ~on;
        }
        if (in) {
            const int rank = __popcll(same & ((1ull << lane) - 1));
            const int place = count[wave][bin] + rank;
            order[place] = n;
            // the last of the equal lanes moves the place on; the wave's lanes have
            // all read it (one wave, in order)
            __builtin_amdgcn_wave_barrier();
            if ((same >> lane) == 1ull) count[wave][bin] = place + 1;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Sum of the runs in places [p0, p1) for the 256 x W columns of blockIdx.y.
template <typename E>
__global__ __launch_bounds__(256) void reduce_runs_kernel(const int64_t* __restrict__ tokens,
                                                          const E* __restrict__ dX, int64_t lddx, E* __restrict__ dE,
                                                          int64_t ldde, int64_t K, int V, float scale, int accumulate,
                                                          const int* __restrict__ order, const int* __restrict__ start,
                                                          float* __restrict__ part, int64_t ldpart, int run_blocks) {
    constexpr int W = Piece<E>::W;
    const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * W;
    if ((int)blockIdx.x >= run_blocks) {
        // zeros for the entries without a token, RUN_BLOCK entries a workgroup
        const int v0 = ((int)blockIdx.x - run_blocks) * RUN_BLOCK;
        const int v1 = v0 + RUN_BLOCK < V ? v0 + RUN_BLOCK : V;
        Piece<E> z;
#pragma unroll
        for (int e = 0; e < W; ++e) z.v[e] = to_elem(0.f, E());
        for (int v = v0; v < v1; ++v)
            if (start[v] == start[v + 1] && c < K) store_piece(dE + (int64_t)v * ldde, c, K, z);
        return;
    }
    __shared__ int row[RUN_BLOCK], entry[RUN_BLOCK];
    const int total = start[V];
    const int p0 = blockIdx.x * RUN_BLOCK;
    if (p0 >= total) return;
    const int np = total - p0 < RUN_BLOCK ? total - p0 : RUN_BLOCK;
    if (threadIdx.x < (unsigned)np) {
        row[threadIdx.x] = order[p0 + threadIdx.x];
        entry[threadIdx.x] = (int)tokens[row[threadIdx.x]];
    }
    __syncthreads();
    if (c >= K) return;
    float sum[W];
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e] = 0.f;
    constexpr int AHEAD = 8;
    for (int q = 0; q < np; q += AHEAD) {
        Piece<E> x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int at = q + u < np ? q + u : np - 1;
            x[u] = load_piece(dX + (int64_t)row[at] * lddx + c);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (q + u >= np) break;
#pragma unroll
            for (int e = 0; e < W; ++e) sum[e] += to_f32(x[u].v[e]);
            const int v = entry[q + u];
            if (q + u + 1 < np && entry[q + u + 1] == v) continue;
            // the run's last place in this block
            const int s = start[v], t = start[v + 1];
            if (s >= p0 && t <= p0 + np) {
                E* out = dE + (int64_t)v * ldde;
                Piece<E> o;
                if (accumulate) o = load_piece(out + c);
#pragma unroll
                for (int e = 0; e < W; ++e)
                    o.v[e] = to_elem(accumulate ? to_f32(o.v[e]) + scale * sum[e] : scale * sum[e], E());
                store_piece(out, c, K, o);
            } else {
                // slot 0: a run that came from the block before, slot 1: one that starts here
                float* o = part + ((int64_t)blockIdx.x * 2 + (s < p0 ? 0 : 1)) * ldpart + c;
#pragma unroll
                for (int e = 0; e < W; e += 4)
                    *reinterpret_cast<f32x4_t*>(o + e) = f32x4_t{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
            }
#pragma unroll
            for (int e = 0; e < W; ++e) sum[e] = 0.f;
        }
    }
}

// The entry whose run starts in block blockIdx.x and goes on in the next ones.
template <typename E>
__global__ __launch_bounds__(256) void join_runs_kernel(const int64_t* __restrict__ tokens, E* __restrict__ dE,
                                                        int64_t ldde, int64_t K, int V, float scale, int accumulate,
                                                        const int* __restrict__ order, const int* __restrict__ start,
                                                        const float* __restrict__ part, int64_t ldpart) {
    constexpr int W = Piece<E>::W;
    const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * W;
    const int total = start[V];
    const int p0 = blockIdx.x * RUN_BLOCK, p1 = p0 + RUN_BLOCK;
    if (p1 >= total || c >= K) return;
    const int v = (int)tokens[order[p1 - 1]];
    const int s = start[v], t = start[v + 1];
    if (s < p0 || t <= p1) return;
    float sum[W];
    auto add = [&](int64_t slot, bool first) {
        const float* p = part + slot * ldpart + c;
#pragma unroll
        for (int e = 0; e < W; e += 4) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(p + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[e + i] = first ? x[i] : sum[e + i] + x[i];
        }
    };
    const int last = (t - 1) / RUN_BLOCK;
    add((int64_t)blockIdx.x * 2 + 1, true);
    for (int k = blockIdx.x + 1; k <= last; ++k) add((int64_t)k * 2, false);
    E* out = dE + (int64_t)v * ldde;
    Piece<E> o;
    if (accumulate) o = load_piece(out + c);
#pragma unroll
    for (int e = 0; e < W; ++e)
        o.v[e] = to_elem(accumulate ? to_f32(o.v[e]) + scale * sum[e] : scale * sum[e], E());
    store_piece(out, c, K, o);
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
    o = up(o + (size_t)((N + RUN_BLOCK - 1) / RUN_BLOCK) * 2 * b.ldpart * 4);
    b.total = o;
    return b;
}

template <typename E>
hipError_t launch_backward(const int64_t* tokens, const E* dX, int64_t lddx, E* dE, int64_t ldde, int64_t N, int64_t K,
                           int64_t V, float scale, bool accumulate, void* workspace, hipStream_t stream) {
    constexpr int W = Piece<E>::W;
    const GradLayout b = grad_layout(N, K, V);
    char* ws = static_cast<char*>(workspace);
    int* order = (int*)(ws + b.order);
    int* start = (int*)(ws + b.start);
    float* part = (float*)(ws + b.part);
    // 256 workgroups of equal ranges, or more of SORT_BINS entries
    const int64_t bins = (V + 255) / 256 < SORT_BINS ? (V + 255) / 256 : SORT_BINS;
    hipLaunchKernelGGL(sort_tokens_kernel, dim3((unsigned)((V + bins - 1) / bins)), dim3(SORT_WAVES * 64), 0, stream,
                       tokens, (int)N, (int)V, (int)bins, order, start);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t runs = (N + RUN_BLOCK - 1) / RUN_BLOCK;
    const int64_t zeros = accumulate ? 0 : (V + RUN_BLOCK - 1) / RUN_BLOCK;
    const unsigned chunks = (unsigned)((K + 256 * W - 1) / (256 * W));
    hipLaunchKernelGGL(reduce_runs_kernel<E>, dim3((unsigned)(runs + zeros), chunks), dim3(256), 0, stream, tokens, dX,
                       lddx, dE, ldde, K, (int)V, scale, accumulate ? 1 : 0, order, start, part, b.ldpart, (int)runs);
    e = hipGetLastError();
    if (e != hipSuccess || runs < 2) return e;
    hipLaunchKernelGGL(join_runs_kernel<E>, dim3((unsigned)(runs - 1), chunks), dim3(256), 0, stream, tokens, dE, ldde,
                       K, (int)V, scale, accumulate ? 1 : 0, order, start, part, b.ldpart);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const int64_t* tokens, const void* E, int64_t lde, void* X, int64_t ldx, int64_t N,
                            int64_t K, int64_t V, float scale, bool f32, hipStream_t stream) {
    const int64_t total = N * ((K + (f32 ? 3 : 7)) / (f32 ? 4 : 8));
    const int64_t want = (total + 255) / 256;
    const dim3 grid((unsigned)(want < 65536 ? want : 65536)), block(256);
    if (f32)
        hipLaunchKernelGGL(embedding_kernel<float>, grid, block, 0, stream, tokens, (const float*)E, lde, (float*)X, ldx,
                           N, K, V, scale);
    else
        hipLaunchKernelGGL(embedding_kernel<uint16_t>, grid, block, 0, stream, tokens, (const uint16_t*)E, lde,
                           (uint16_t*)X, ldx, N, K, V, scale);
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
