// Losses on the logits of a linear head, and the gradient of those logits, in pieces
// of the vocabulary.
//
// With s_v = x·w_v / t, a token's log-sum-exp over the vocabulary is that of its
// pieces: each gives its largest s and Σ exp(s - it), and lse = m + log Σ_pieces
// l·exp(m_piece - m) is exact however the vocabulary is cut.  Pieces are joined in
// their order, so that the same call gives the same bits.  The gradient of the logits
// needs lse alone, G = coef·(exp(s - lse) - p), so a piece of it is made from a piece
// of the logits, used in both gradients' products, and dropped.
//
// Everything is float32 up to G, which is rounded to bfloat16 for the matrix cores
// once, relative to the largest coefficient c (most training steps weigh all tokens
// alike: r = coef / c is then 1, and an entry -r of a label with a small probability
// is exact); c multiplies the float32 sums.  What that rounding costs, as the norm of dX's
// or dW's error (4096 tokens on 32000 x 4096; the results' own rounding alone: 1.66e-3):
// all tokens alike 1.67e-3, weights of 0.1 to 1.1 2.2e-3, a mean over each sequence 2.0e-3
// (601 tokens on 50257 x 1024: 2.5e-3), a teacher's 64 entries 2.3e-3 to 2.6e-3.  A
// second term (train_api.hip: kTwoTerms) takes it away, and makes dX's and dW's products
// twice as long.
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"
#include "train.hpp"

namespace espace {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float exp_f(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ __forceinline__ float nan_f() { return __builtin_nanf(""); }

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// Σ exp(s - m) of a set, given that of its parts: l·exp(m_part - m), 0 for a part whose
// logits are all -infinity
__device__ __forceinline__ float rescale(float l, float from, float to) {
    return from == -INFINITY ? 0.f : l * exp_f(from - to);
}

// ---- targets -------------------------------------------------------------------

// One wave per token, entry 64 u + lane in register u.  An entry's rank among the
// columns, and the sum of equal ones, come from T broadcasts of an entry to all: T
// squared comparisons, 64 at a time.  4096 tokens of 64 entries 11 us, 128 35, 256 135,
// 512 535, 1024 1970.
template <int U>
__global__ __launch_bounds__(256) void teacher_kernel(const int64_t* __restrict__ index, int64_t ldi,
                                                      const float* __restrict__ logits, int64_t ldl, int N, int T,
                                                      int V, float inv_t, TeacherOut out) {
    __shared__ int lds_col[4][64 * U];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int n = blockIdx.x * 4 + wave;
    if (n >= N) return;
    int c[U];
    float z[U];
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = 64 * u + lane;
        c[u] = -1;
        z[u] = -INFINITY;
        if (j < T) {
            const int64_t i = index[(int64_t)n * ldi + j];
            if (i >= 0) {
                z[u] = i < V ? logits[(int64_t)n * ldl + j] * inv_t : nan_f();
                c[u] = i < V ? (int)i : V - 1;
            }
        }
        m = fmaxf(m, z[u]);
    }
    m = wave_max(m);
    float l = 0.f, p[U], lp[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        p[u] = z[u] == -INFINITY ? 0.f : exp_f(z[u] - m);
        l += p[u];
    }
    l = wave_sum(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float lg = logf(l);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        p[u] *= inv;
        lp[u] = z[u] == -INFINITY ? 0.f : (z[u] - m) - lg;
    }
    if (out.sorted || out.mass) {
        float sum[U];
        int rank[U];
        bool again[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            sum[u] = 0.f;
            rank[u] = 0;
            again[u] = false;
        }
#pragma unroll
        for (int v = 0; v < U; ++v)
            for (int k = 0; k < 64 && 64 * v + k < T; ++k) {
                const int ck = __builtin_amdgcn_readlane(c[v], k);
                const float pk = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p[v]), k));
                const int j = 64 * v + k;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool before = j < 64 * u + lane;
                    if (c[u] == ck) {
                        sum[u] += pk;
                        again[u] |= before;
                    }
                    rank[u] += ck >= 0 && (ck < c[u] || (ck == c[u] && before));
                }
            }
        if (out.sorted) {
            int there = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (c[u] >= 0) {
                    lds_col[wave][rank[u]] = c[u];
                    out.sorted[(int64_t)n * T + rank[u]] = c[u];
                    out.place[(int64_t)n * T + rank[u]] = (uint16_t)(64 * u + lane);
                }
                there += __popcll(__ballot(c[u] >= 0));
            }
            __builtin_amdgcn_wave_barrier();      // the wave's own LDS, in order
            const int slabs = (V + LOSS_SLAB - 1) / LOSS_SLAB;
            for (int s = lane; s <= slabs + 1; s += 64) {     // (a tile may end a slab later)
                // entries before the slab
                const int64_t edge = (int64_t)s * LOSS_SLAB;
                int lo = 0, hi = there;
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (lds_col[wave][mid] < edge) lo = mid + 1;
                    else hi = mid;
                }
                out.first[(int64_t)n * out.ldfirst + s] = (uint16_t)lo;
            }
        }
        if (out.mass) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                p[u] = sum[u];
                if (again[u]) c[u] = -1;
            }
            // l is 0 without a target, NaN where an entry is
            if (lane == 0) out.mass[n] = l == 0.f ? 0.f : 1.f;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = 64 * u + lane;
        if (j < T) {
            out.col[(int64_t)n * T + j] = c[u];
            out.p[(int64_t)n * T + j] = p[u];
            if (out.logp) out.logp[(int64_t)n * T + j] = lp[u];
        }
    }
}

// ---- forward -------------------------------------------------------------------

// Q times four sums, from the first slab's address: the slabs are added in order, AHEAD
// loads of each in flight (past the last: it again).
template <int Q, int AHEAD>
__device__ __forceinline__ void add_slabs(f32x4_t (&x)[Q], const float* p, int slabs, int64_t stride) {
#pragma unroll
    for (int q = 0; q < Q; ++q) x[q] = *reinterpret_cast<const f32x4_t*>(p + 4 * q);
    for (int s = 1; s < slabs; s += AHEAD) {
        f32x4_t y[AHEAD][Q];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int q = 0; q < Q; ++q)
                y[u][q] = *reinterpret_cast<const f32x4_t*>(p + min(s + u, slabs - 1) * stride + 4 * q);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (s + u < slabs)
#pragma unroll
                for (int q = 0; q < Q; ++q) x[q] += y[u][q];
    }
}

// four logits
__device__ __forceinline__ f32x4_t logits4(const float* p, const Logits& S) {
    f32x4_t x[1];
    add_slabs<1, 4>(x, p, S.slabs, S.stride);
    return x[0];
}

// A token's loss from its targets' logits; all lanes of a wave, for an entry each.
__device__ __forceinline__ float entries_loss(const LossTargets& t, int64_t row, int lane, float ls,
                                              float* __restrict__ picked, float tt) {
    float v = 0.f;
    for (int j = lane; j < t.T; j += 64) {
        const int64_t at = row * t.T + j;
        if (t.col[at] < 0) picked[j] = 0.f;
        else if (t.p[at] != 0.f) v += t.p[at] * ((t.logp[at] + ls) - picked[j]);
    }
    return wave_sum(v) * tt;
}
__device__ __forceinline__ float label_loss(int64_t label, int V, float ls, float logit) {
    return label >= V ? nan_f() : (label >= 0 ? ls - logit : 0.f);
}

// STAT_COLS columns of one token: 256 threads of 4 x 4 columns each, kept in
// registers between the maximum and the sum.  WHOLE: they are all of the vocabulary,
// and the token's loss follows at once.
template <bool WHOLE>
__global__ __launch_bounds__(256) void stats_kernel(Logits S, int c0, int cols,
                                                    float inv_t, LossTargets t, float2* __restrict__ part, int N,
                                                    int part0, int n0, float* __restrict__ picked, int64_t ldpk,
                                                    float tt, float* __restrict__ loss, float* __restrict__ lse) {
    __shared__ float red[8];
    const int n = n0 + blockIdx.y;
    const int b0 = blockIdx.x * STAT_COLS;
    const int left = cols - b0 < STAT_COLS ? cols - b0 : STAT_COLS;
    const float* row = S.S + (int64_t)n * S.lds + b0;
    float* pick = picked + (int64_t)n * ldpk;
    float v[4][4];
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 1024 + threadIdx.x * 4;
        // rows are padded to a multiple of 8 columns
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
        if (c < left) x = logits4(row + c, S);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[i][e] = c + e < left ? x[e] * inv_t : -INFINITY;
            m = fmaxf(m, v[i][e]);
        }
    }
    for (int j = threadIdx.x; j < t.T; j += 256) {
        const int64_t c = (t.labels ? t.labels[n] : (int64_t)t.col[(int64_t)n * t.T + j]) - c0 - b0;
        if (c >= 0 && c < left) {
            float x = row[c];
            for (int s = 1; s < S.slabs; ++s) x += row[c + s * S.stride];
            pick[j] = x * inv_t;
        }
    }
    m = wave_max(m);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane == 0) red[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float l = 0.f;
    // all -infinity: the sum stays 0, and NaN (which a maximum passes over) stays NaN
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) l += exp_f(v[i][e] - base);
    l = wave_sum(l);
    if (lane == 0) red[4 + wave] = l;
    __syncthreads();                              // and the logits at `pick` are written
    if (wave != 0) return;
    l = (red[4] + red[5]) + (red[6] + red[7]);
    if constexpr (!WHOLE) {
        if (lane == 0) part[(int64_t)(part0 + blockIdx.x) * N + n] = make_float2(l == 0.f ? -INFINITY : base, l);
        return;
    }
    const float ls = m == -INFINITY && l == 0.f ? -INFINITY : base + logf(l);
    const float x = t.labels ? (lane == 0 ? label_loss(t.labels[n], cols, ls, pick[0]) : 0.f)
                             : entries_loss(t, n, lane, ls, pick, tt);
    if (lane == 0) {
        loss[n] = x;
        lse[n] = ls;
    }
}

// (m, l) of two sets together
__device__ __forceinline__ void join(float& m, float& l, float m2, float l2) {
    const float to = fmaxf(m, m2);
    l = rescale(l, m, to) + rescale(l2, m2, to);
    m = to;
}

// 16 tokens: 64 threads each join every 64th part of a token, in order, then each
// other's; every wave takes a token's entries.
__global__ __launch_bounds__(1024) void finish_kernel(const float2* __restrict__ part, int nparts, int N, int V,
                                                      float tt, LossTargets t, float* __restrict__ picked,
                                                      int64_t ldpk, float* __restrict__ loss, float* __restrict__ lse) {
    __shared__ float red_m[16][17], red_l[16][17], lse_of[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int n = blockIdx.x * 16 + x;
    float m = -INFINITY, l = 0.f;
    if (n < N)
        for (int i = y; i < nparts; i += 64) {
            const float2 q = part[(int64_t)i * N + n];
            join(m, l, q.x, q.y);
        }
    join(m, l, __shfl_xor(m, 16), __shfl_xor(l, 16));
    join(m, l, __shfl_xor(m, 32), __shfl_xor(l, 32));
    if (lane < 16) {
        red_m[wave][x] = m;
        red_l[wave][x] = l;
    }
    __syncthreads();
    if (threadIdx.x < 16) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, red_m[i][x]);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += rescale(red_l[i][x], red_m[i][x], top);
        const float ls = top + logf(sum);
        lse_of[x] = ls;
        if (n < N) {
            lse[n] = ls;
            if (t.labels) loss[n] = label_loss(t.labels[n], V, ls, picked[(int64_t)n * ldpk]);
        }
    }
    if (t.labels) return;
    __syncthreads();
    const int64_t row = (int64_t)blockIdx.x * 16 + wave;
    if (row >= N) return;
    const float v = entries_loss(t, row, lane, lse_of[wave], picked + row * ldpk, tt);
    if (lane == 0) loss[row] = v;
}

// ---- backward ------------------------------------------------------------------

__device__ __forceinline__ float coef_of(int n, const float* dloss, const int64_t* labels, const float* mass, float t,
                                         int V) {
    if (labels) return labels[n] < 0 ? 0.f : (labels[n] >= V ? nan_f() : dloss[n]);
    return mass[n] == 0.f ? 0.f : dloss[n] * t;
}
// the largest of finite |a| that coefficients are taken relative to
__device__ __forceinline__ float scale_of(float m) {
    return m < 1.17549435e-38f ? 1.f : m;         // all 0, or too small to divide by
}

// One workgroup: two passes over the tokens, COEF_OWN a thread kept in registers.  8192
// tokens 6.4 us (with the list of the live ones 15), 65536 85, 2^21 - 1 3.4 ms.
constexpr int COEF_OWN = 8;

__global__ __launch_bounds__(1024) void coef_kernel(const float* __restrict__ dloss,
                                                    const int64_t* __restrict__ labels,
                                                    const float* __restrict__ mass, float t, int N, int V,
                                                    float* __restrict__ r, float* __restrict__ scale,
                                                    const float* __restrict__ lse, LiveTokens live) {
    __shared__ float red[16];
    __shared__ int found[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto coef = [&](int n) { return coef_of(n, dloss, labels, mass, t, V); };
    float own[COEF_OWN];
    float m = 0.f;
#pragma unroll
    for (int u = 0; u < COEF_OWN; ++u) {
        const int n = u * 1024 + threadIdx.x;
        own[u] = n < N ? coef(n) : 0.f;
        const float a = fabsf(own[u]);
        if (a < INFINITY) m = fmaxf(m, a);
    }
    for (int n = COEF_OWN * 1024 + threadIdx.x; n < N; n += 1024) {
        const float a = fabsf(coef(n));
        if (a < INFINITY) m = fmaxf(m, a);
    }
    m = wave_max(m);
    if (lane == 0) red[wave] = m;
    __syncthreads();
    m = red[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) m = fmaxf(m, red[i]);
    m = scale_of(m);
    if (threadIdx.x == 0) scale[0] = m;
    int before = 0;                               // live tokens of the rounds before
    auto round = [&](int n, float c) {
        const float x = c / m;
        if (n < N) r[n] = x;
        if (!live.count) return;
        const bool in = n < N && x != 0.f;
        const unsigned long long mask = __ballot(in);
        if (lane == 0) found[wave] = __popcll(mask);
        __syncthreads();
        int at = before + __popcll(mask & ((1ull << lane) - 1));
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i < wave) at += found[i];
            before += found[i];
        }
        if (n < N) live.where[n] = in ? at : -1;
        if (in) {
            live.token[at] = n;
            live.r[at] = x;
            live.lse[at] = lse[n];
            if (labels) live.labels[at] = labels[n];
        }
        __syncthreads();
    };
#pragma unroll
    for (int u = 0; u < COEF_OWN; ++u)
        if (u * 1024 < N) round(u * 1024 + threadIdx.x, own[u]);
    for (int n0 = COEF_OWN * 1024; n0 < N; n0 += 1024) {
        const int n = n0 + threadIdx.x;
        round(n, n < N ? coef(n) : 0.f);
    }
    if (live.count && threadIdx.x == 0) {
        live.count[0] = before > 0 ? before : 1;
        if (before == 0) {
            live.token[0] = 0;
            live.r[0] = 0.f;
            live.lse[0] = 0.f;
            if (labels) live.labels[0] = -1;
        }
    }
}

__device__ __forceinline__ uint16_t to_elem(float v, uint16_t) { return (uint16_t)bf16_rne(v); }
__device__ __forceinline__ float to_elem(float v, float) { return v; }

__device__ __forceinline__ float from_elem(uint16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ float from_elem(float v) { return v; }
__device__ __forceinline__ uint16_t zero_of(uint16_t) { return 0; }
__device__ __forceinline__ float zero_of(float) { return 0.f; }

// 64 x 64 of G, its transpose through LDS.  Term 1 is what term 0's rounding left.
template <typename E>
__global__ __launch_bounds__(256) void grad_kernel(Logits S, int N, int c0, int cols,
                                                   float inv_t, const float* __restrict__ lse,
                                                   const float* __restrict__ r, LossTargets t, int entries,
                                                   GradOut out) {
    __shared__ float less[64][65];                // Σ p of the tile's entries
    __shared__ E tile[64][64 + 4 / sizeof(E)];
    const int n0 = blockIdx.y * 64, b0 = blockIdx.x * 64;
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;    // 4 columns, 16 rows a pass
    float g[4][4];
    if (entries) {
        for (int i = threadIdx.x; i < 64 * 64; i += 256) less[i >> 6][i & 63] = 0.f;
        __syncthreads();
        // (an entry has one place after its equals were added to it)
        const int64_t end = min((int64_t)N, (int64_t)n0 + 64) * t.T;
        for (int64_t at = (int64_t)n0 * t.T + threadIdx.x; at < end; at += 256) {
            const int c = t.col[at] - c0 - b0;
            if (t.col[at] >= 0 && c >= 0 && c < 64) less[at / t.T - n0][c] = t.p[at];
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = n0 + i * 16 + y, c = b0 + 4 * x;
#pragma unroll
        for (int e = 0; e < 4; ++e) g[i][e] = 0.f;
        if (n >= N || c >= cols) continue;
        const float rn = r[n];
        const f32x4_t s = logits4(S.S + (int64_t)n * S.lds + c, S);
        const float ls = lse[n];
        const int64_t at = t.labels ? t.labels[n] - c0 - c : -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v = exp_f(s[e] * inv_t - ls);
            if (at == e) v -= 1.f;
            if (entries) v -= less[i * 16 + y][4 * x + e];
            // a token without a target: 0 whatever its logits are
            g[i][e] = rn == 0.f ? 0.f : rn * v;
        }
    }
    for (int term = 0; term < out.terms; ++term) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = n0 + i * 16 + y, c = b0 + 4 * x;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const E q = to_elem(g[i][e], E());
                g[i][e] -= from_elem(q);
                tile[i * 16 + y][4 * x + e] = q;
                if (out.G && n < (out.terms > 1 ? out.ldx : N) && c + e < cols)
                    ((E*)out.G)[((int64_t)term * out.ldx + n) * out.ldg + c + e] = q;
            }
        }
        if (!out.GT) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = b0 + i * 16 + y, n = n0 + 4 * x;
            if (c >= cols) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < out.ldx) ((E*)out.GT)[c * out.ldgt + term * out.ldx + n + e] = tile[4 * x + e][i * 16 + y];
        }
        __syncthreads();
    }
}

template <typename E>
__global__ __launch_bounds__(256) void fix_kernel(LossTargets t, const float* __restrict__ picked, int64_t ldpk,
                                                  const float* __restrict__ lse, const float* __restrict__ r, int N,
                                                  int c0, int cols, GradOut out) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (int64_t)N * t.T) return;
    const int c = t.col[at] - c0;
    if (t.col[at] < 0 || c < 0 || c >= cols) return;
    const int n = (int)(at / t.T), j = (int)(at - (int64_t)n * t.T);
    const float rn = r[n];
    if (rn == 0.f) return;
    const int row = out.where ? out.where[n] : n;
    float g = rn * (exp_f(picked[(int64_t)n * ldpk + j] - lse[n]) - t.p[at]);
    for (int term = 0; term < out.terms; ++term) {
        const E q = to_elem(g, E());
        g -= from_elem(q);
        if (out.G) ((E*)out.G)[((int64_t)term * out.ldx + row) * out.ldg + c] = q;
        if (out.GT) ((E*)out.GT)[c * out.ldgt + term * out.ldx + row] = q;
    }
}

// 64 x 64 through LDS, 16 bytes a load and a store; from(n): the row of X that row n is,
// -1 for zeros.
template <typename E> using TransposeTile = E[64][64 + 4 / sizeof(E)];

template <typename E, class From>
__device__ __forceinline__ void transpose_tile(TransposeTile<E>& tile, const E* __restrict__ X, int64_t ldx_, int N,
                                               int K, int n0, int k0, E* __restrict__ dst, int64_t ldd, int64_t ldx,
                                               int terms, From from) {
    constexpr int W = 16 / sizeof(E), PER = 64 / W;          // elements of a piece, pieces of 64
#pragma unroll
    for (int q = threadIdx.x; q < 64 * PER; q += 256) {
        const int n = n0 + q / PER, k = k0 + q % PER * W;
        struct { E v[W]; } x;
        u32x4_t raw = {0u, 0u, 0u, 0u};
        // rows of X are padded to 16 bytes
        const int row = n < N && k < K ? from(n) : -1;
        if (row >= 0) raw = *reinterpret_cast<const u32x4_t*>(X + (int64_t)row * ldx_ + k);
        __builtin_memcpy(&x, &raw, 16);
#pragma unroll
        for (int e = 0; e < W; ++e) tile[q / PER][q % PER * W + e] = x.v[e];
    }
    __syncthreads();
#pragma unroll
    for (int q = threadIdx.x; q < 64 * PER; q += 256) {
        const int k = k0 + q / PER, n = n0 + q % PER * W;
        // ldx is a multiple of 8: a piece that starts before it ends there
        if (k >= K || n >= ldx) continue;
        struct { E v[W]; } x;
#pragma unroll
        for (int e = 0; e < W; ++e) x.v[e] = tile[q % PER * W + e][q / PER];
        u32x4_t raw;
        __builtin_memcpy(&raw, &x, 16);
        for (int term = 0; term < terms; ++term)
            *reinterpret_cast<u32x4_t*>(dst + (int64_t)k * ldd + term * ldx + n) = raw;
    }
}

template <typename E>
__global__ __launch_bounds__(256) void transpose_live_kernel(const E* __restrict__ X, int64_t ldx_,
                                                             const float* __restrict__ r, int N, int K,
                                                             E* __restrict__ dst, int64_t ldd, int64_t ldx, int terms,
                                                             LiveTokens live) {
    __shared__ TransposeTile<E> tile;
    const int n0 = blockIdx.x * 64;
    if (live.count) {
        N = live.count[0];
        r = live.r;
        if (n0 >= N) return;
    }
    transpose_tile<E>(tile, X, ldx_, N, K, n0, blockIdx.y * 64, dst, ldd, ldx, terms,
                      [&](int n) { return r[n] == 0.f ? -1 : (live.count ? live.token[n] : n); });
}

// Few tokens: coef_kernel (workgroup 0) and the transposes of X and W in one launch; a
// token is left out of X's where its coefficient is 0.
constexpr int PREPARE_TOKENS = 2048;

template <typename E>
__global__ __launch_bounds__(256) void prepare_kernel(const float* __restrict__ dloss,
                                                      const int64_t* __restrict__ labels,
                                                      const float* __restrict__ mass, float t, int N, int V, int K,
                                                      float* __restrict__ r, float* __restrict__ scale,
                                                      const E* __restrict__ X, int64_t ldx_, E* __restrict__ XT,
                                                      int64_t ldxt, int64_t ldn, int terms, int x_tiles,
                                                      const E* __restrict__ W, int64_t ldw, E* __restrict__ WT,
                                                      int64_t ldwt) {
    auto coef = [&](int n) { return coef_of(n, dloss, labels, mass, t, V); };
    if (blockIdx.x == 0) {
        constexpr int OWN = PREPARE_TOKENS / 256;
        __shared__ float red[4];
        float own[OWN], m = 0.f;
#pragma unroll
        for (int u = 0; u < OWN; ++u) {
            const int n = u * 256 + threadIdx.x;
            own[u] = n < N ? coef(n) : 0.f;
            const float a = fabsf(own[u]);
            if (a < INFINITY) m = fmaxf(m, a);
        }
        m = wave_max(m);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
        m = scale_of(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        if (threadIdx.x == 0) scale[0] = m;
#pragma unroll
        for (int u = 0; u < OWN; ++u) {
            const int n = u * 256 + threadIdx.x;
            if (n < N) r[n] = own[u] / m;
        }
        return;
    }
    __shared__ TransposeTile<E> tile;
    const int b = blockIdx.x - 1, across = (K + 63) / 64;
    if (b < x_tiles)
        transpose_tile<E>(tile, X, ldx_, N, K, b / across * 64, b % across * 64, XT, ldxt, ldn, terms,
                          [&](int n) { return coef(n) == 0.f ? -1 : n; });
    else
        transpose_tile<E>(tile, W, ldw, V, K, (b - x_tiles) / across * 64, (b - x_tiles) % across * 64, WT, ldwt, ldwt,
                          1, [](int v) { return v; });
}

__global__ __launch_bounds__(256) void add_f32_kernel(f32x4_t* __restrict__ acc, const f32x4_t* __restrict__ src,
                                                      int64_t quads) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quads; i += (int64_t)gridDim.x * 256)
        acc[i] += src[i];
}

// 8 columns a thread
template <typename E>
__global__ __launch_bounds__(256) void sum_out_kernel(const float* __restrict__ src, int64_t lds, int slabs,
                                                      int64_t stride, const float* __restrict__ scale,
                                                      E* __restrict__ out, int64_t ldo, int64_t R, int64_t C, const int* __restrict__ count,
                                                      const int* __restrict__ rows) {
    const float a = scale[0];
    if (count) R = count[0];
    const int64_t pieces = (C + 7) / 8, total = R * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces, c = (i - row * pieces) * 8;
        // rows of src are padded to a multiple of 8 columns
        const float* p = src + row * lds + c;
        f32x4_t x[2];
        add_slabs<2, 8>(x, p, slabs, stride);
        struct { E v[8]; } q;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            q.v[e] = to_elem(a * x[0][e], E());
            q.v[4 + e] = to_elem(a * x[1][e], E());
        }
        E* o = out + (count ? rows[row] : row) * ldo + c;
        if (c + 8 <= C) {
            u32x4_t raw[sizeof(E) / 2];
            __builtin_memcpy(raw, &q, 8 * sizeof(E));
#pragma unroll
            for (int e = 0; e < (int)sizeof(E) / 2; ++e) reinterpret_cast<u32x4_t*>(o)[e] = raw[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < C) o[e] = q.v[e];
        }
    }
}

// One wave per token.
__global__ __launch_bounds__(256) void zero_dead_kernel(const float* __restrict__ r, uint16_t* __restrict__ out,
                                                        int64_t ldo, int N, int64_t C) {
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (n >= N || r[n] != 0.f) return;
    uint16_t* row = out + (int64_t)n * ldo;
    for (int64_t c = (threadIdx.x & 63) * 8; c < C; c += 512) {
        if (c + 8 <= C) {
            *reinterpret_cast<u32x4_t*>(row + c) = u32x4_t{0u, 0u, 0u, 0u};
        } else {
            for (int e = 0; c + e < C; ++e) row[c + e] = 0;
        }
    }
}

template <typename E>
__global__ __launch_bounds__(256) void zero_kernel(E* __restrict__ out, int64_t ldo, int64_t R, int64_t C) {
    const int64_t total = R * C;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256)
        out[i / C * ldo + i % C] = zero_of(E());
}

unsigned blocks_of(int64_t items, int64_t most = 16384) {
    const int64_t b = (items + 255) / 256;
    return (unsigned)(b < 1 ? 1 : (b < most ? b : most));
}

}  // namespace

hipError_t launch_teacher(const int64_t* index, int64_t ldi, const float* logits, int64_t ldl, int N, int T, int V,
                          float inv_t, const TeacherOut& out, hipStream_t stream) {
    const dim3 grid((N + 3) / 4), block(256);
#define TEACHER(U) \
    hipLaunchKernelGGL(teacher_kernel<U>, grid, block, 0, stream, index, ldi, logits, ldl, N, T, V, inv_t, out)
    if (T <= 64) TEACHER(1);
    else if (T <= 128) TEACHER(2);
    else if (T <= 256) TEACHER(4);
    else if (T <= 512) TEACHER(8);
    else TEACHER(16);
#undef TEACHER
    return hipGetLastError();
}

hipError_t launch_loss_stats(const Logits& S, int N, int c0, int cols, float inv_t,
                             const LossTargets& t, float2* part, int part0, float* picked, int64_t ldpk,
                             hipStream_t stream) {
    // a launch has at most 65535 workgroups in y
    const int chunks = (cols + STAT_COLS - 1) / STAT_COLS;
    for (int n0 = 0; n0 < N; n0 += 65535) {
        const int rows = N - n0 < 65535 ? N - n0 : 65535;
        hipLaunchKernelGGL(stats_kernel<false>, dim3(chunks, rows), dim3(256), 0, stream, S, c0, cols, inv_t, t, part, N,
                           part0, n0, picked, ldpk, 0.f, nullptr, nullptr);
    }
    return hipGetLastError();
}

hipError_t launch_loss_whole(const Logits& S, int N, int V, float temperature, const LossTargets& t, float* picked,
                             int64_t ldpk, float* loss, float* lse, hipStream_t stream) {
    for (int n0 = 0; n0 < N; n0 += 65535) {
        const int rows = N - n0 < 65535 ? N - n0 : 65535;
        hipLaunchKernelGGL(stats_kernel<true>, dim3(1, rows), dim3(256), 0, stream, S, 0, V, 1.f / temperature, t, nullptr,
                           N, 0, n0, picked, ldpk, temperature * temperature, loss, lse);
    }
    return hipGetLastError();
}

hipError_t launch_loss_finish(const float2* part, int nparts, int N, int V, float temperature, const LossTargets& t,
                              float* picked, int64_t ldpk, float* loss, float* lse, hipStream_t stream) {
    hipLaunchKernelGGL(finish_kernel, dim3((N + 15) / 16), dim3(1024), 0, stream, part, nparts, N, V,
                       temperature * temperature, t, picked, ldpk, loss, lse);
    return hipGetLastError();
}

hipError_t launch_loss_coef(const float* dloss, const int64_t* labels, const float* mass, float t, int N, int V,
                            float* r, float* scale, const float* lse, const LiveTokens& live, hipStream_t stream) {
    hipLaunchKernelGGL(coef_kernel, dim3(1), dim3(1024), 0, stream, dloss, labels, mass, t, N, V, r, scale, lse, live);
    return hipGetLastError();
}

bool loss_prepare_supported(int64_t N, int64_t V, int64_t K) {
    const int64_t across = (K + 63) / 64;
    return N <= PREPARE_TOKENS && ((N + 63) / 64 + (V + 63) / 64) * across < (int64_t)1 << 23;
}

hipError_t launch_loss_prepare(const float* dloss, const int64_t* labels, const float* mass, float t, int N, int V, int K,
                               float* r, float* scale, const void* X, int64_t ldx_, void* XT, int64_t ldxt, int64_t ldn,
                               int terms, const void* W, int64_t ldw, void* WT, int64_t ldwt, bool f32,
                               hipStream_t stream) {
    const int across = (K + 63) / 64, x_tiles = XT ? (N + 63) / 64 * across : 0, w_tiles = WT ? (V + 63) / 64 * across : 0;
    const dim3 grid(1 + x_tiles + w_tiles), block(256);
    if (f32)
        hipLaunchKernelGGL(prepare_kernel<float>, grid, block, 0, stream, dloss, labels, mass, t, N, V, K, r, scale,
                           (const float*)X, ldx_, (float*)XT, ldxt, ldn, terms, x_tiles, (const float*)W, ldw,
                           (float*)WT, ldwt);
    else
        hipLaunchKernelGGL(prepare_kernel<uint16_t>, grid, block, 0, stream, dloss, labels, mass, t, N, V, K, r, scale,
                           (const uint16_t*)X, ldx_, (uint16_t*)XT, ldxt, ldn, terms, x_tiles, (const uint16_t*)W, ldw,
                           (uint16_t*)WT, ldwt);
    return hipGetLastError();
}

// N < 2^21 tokens, K <= 2^21 features: at most 32768 workgroups of 64 rows in y
static_assert((1 << 21) / 64 <= 65535, "launch limit");

hipError_t launch_loss_grad(const Logits& S, int N, int c0, int cols, float inv_t, const float* lse,
                            const float* r, const LossTargets& t, bool entries, const GradOut& out,
                            hipStream_t stream) {
    const dim3 grid((cols + 63) / 64, (N + 63) / 64), block(256);
    if (out.f32)
        hipLaunchKernelGGL(grad_kernel<float>, grid, block, 0, stream, S, N, c0, cols, inv_t, lse, r, t,
                           entries ? 1 : 0, out);
    else
        hipLaunchKernelGGL(grad_kernel<uint16_t>, grid, block, 0, stream, S, N, c0, cols, inv_t, lse, r, t,
                           entries ? 1 : 0, out);
    return hipGetLastError();
}

hipError_t launch_loss_fix(const LossTargets& t, const float* picked, int64_t ldpk, const float* lse, const float* r,
                           int N, int c0, int cols, const GradOut& out, hipStream_t stream) {
    const dim3 grid((unsigned)(((int64_t)N * t.T + 255) / 256)), block(256);
    if (out.f32)
        hipLaunchKernelGGL(fix_kernel<float>, grid, block, 0, stream, t, picked, ldpk, lse, r, N, c0, cols, out);
    else
        hipLaunchKernelGGL(fix_kernel<uint16_t>, grid, block, 0, stream, t, picked, ldpk, lse, r, N, c0, cols, out);
    return hipGetLastError();
}

hipError_t launch_transpose_live(const void* X, int64_t ldx_, const float* r, int N, int K, void* dst, int64_t ldd,
                                 int64_t ldx, int terms, bool f32, const LiveTokens* live, hipStream_t stream) {
    const LiveTokens l = live ? *live : LiveTokens{};
    const dim3 grid((N + 63) / 64, (K + 63) / 64), block(256);
    if (f32)
        hipLaunchKernelGGL(transpose_live_kernel<float>, grid, block, 0, stream, (const float*)X, ldx_, r, N, K,
                           (float*)dst, ldd, ldx, terms, l);
    else
        hipLaunchKernelGGL(transpose_live_kernel<uint16_t>, grid, block, 0, stream, (const uint16_t*)X, ldx_, r, N, K,
                           (uint16_t*)dst, ldd, ldx, terms, l);
    return hipGetLastError();
}

hipError_t launch_add_f32(float* acc, const float* src, int64_t elems, hipStream_t stream) {
    hipLaunchKernelGGL(add_f32_kernel, dim3(blocks_of(elems / 4)), dim3(256), 0, stream, (f32x4_t*)acc,
                       (const f32x4_t*)src, elems / 4);
    return hipGetLastError();
}

hipError_t launch_sum_out(const float* src, int64_t lds, int slabs, int64_t stride, const float* scale, void* out,
                          int64_t ldo, int64_t R, int64_t C, bool f32, const LiveTokens* live, hipStream_t stream) {
    const dim3 grid(blocks_of(R * ((C + 7) / 8))), block(256);
    const int *count = live ? live->count : nullptr, *rows = live ? live->token : nullptr;
    if (f32)
        hipLaunchKernelGGL(sum_out_kernel<float>, grid, block, 0, stream, src, lds, slabs, stride, scale, (float*)out,
                           ldo, R, C, count, rows);
    else
        hipLaunchKernelGGL(sum_out_kernel<uint16_t>, grid, block, 0, stream, src, lds, slabs, stride, scale,
                           (uint16_t*)out, ldo, R, C, count, rows);
    return hipGetLastError();
}

hipError_t launch_zero_dead(const float* r, void* out, int64_t ldo, int N, int64_t C, hipStream_t stream) {
    hipLaunchKernelGGL(zero_dead_kernel, dim3((N + 3) / 4), dim3(256), 0, stream, r, (uint16_t*)out, ldo, N, C);
    return hipGetLastError();
}

hipError_t launch_zero(void* out, int64_t ldo, int64_t R, int64_t C, bool f32, hipStream_t stream) {
    const dim3 grid(blocks_of(R * C)), block(256);
    if (f32) hipLaunchKernelGGL(zero_kernel<float>, grid, block, 0, stream, (float*)out, ldo, R, C);
    else hipLaunchKernelGGL(zero_kernel<uint16_t>, grid, block, 0, stream, (uint16_t*)out, ldo, R, C);
    return hipGetLastError();
}

}  // namespace espace
