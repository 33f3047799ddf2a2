// Host-side launchers of the losses' and the embedding's kernels (internal to the
// library).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace espace {

// The targets of N tokens: one label each (labels), or T entries each (col, p; col
// < 0: none) that launch_teacher made.
struct LossTargets {
    const int64_t* labels = nullptr;
    const int* col = nullptr;
    const float* p = nullptr;
    const float* logp = nullptr;
    int T = 1;
};

// Columns of S that one workgroup of launch_loss_stats reduces.
constexpr int STAT_COLS = 4096;

// The teacher's distributions: col[n][j] its entry (-1: empty), p[n][j] and, if
// wanted, logp[n][j].
struct TeacherOut {
    int* col = nullptr;
    float* p = nullptr;
    float* logp = nullptr;
    // wanted for the backward pass: an entry that occurs again is added to its first
    // place, whose other places become empty, and mass[n] is 1, or 0 for a token
    // without a target
    float* mass = nullptr;
    // wanted for LossEpi: the entries in the order of their columns, their places, and
    // how many lie before each LOSS_SLAB columns, up to the second past the last (rows
    // ldfirst apart)
    int* sorted = nullptr;
    uint16_t* place = nullptr;
    uint16_t* first = nullptr;
    int64_t ldfirst = 0;
};
hipError_t launch_teacher(const int64_t* index, int64_t ldi, const float* logits, int64_t ldl, int N, int T, int V,
                          float inv_t, const TeacherOut& out, hipStream_t stream);

// Logits as float32 sums: `slabs` of them, `stride` apart, to be added in order.
struct Logits {
    const float* S = nullptr;
    int64_t lds = 0;
    int slabs = 1;
    int64_t stride = 0;
};
// Columns [c0, c0 + cols) of the logits of N tokens: the largest s / t and Σ
// exp(s / t - it) of every STAT_COLS of them at part[k][n] (k from part0 on), and s / t
// of the targets among them at picked[n][j].
hipError_t launch_loss_stats(const Logits& S, int N, int c0, int cols, float inv_t,
                             const LossTargets& t, float2* part, int part0, float* picked, int64_t ldpk,
                             hipStream_t stream);
// The whole vocabulary's (V <= STAT_COLS): loss and lse, and picked with its empty
// places.
hipError_t launch_loss_whole(const Logits& S, int N, int V, float temperature, const LossTargets& t, float* picked,
                             int64_t ldpk, float* loss, float* lse, hipStream_t stream);
// loss and lse from the nparts parts of each token; picked of empty places.
hipError_t launch_loss_finish(const float2* part, int nparts, int N, int V, float temperature, const LossTargets& t,
                              float* picked, int64_t ldpk, float* loss, float* lse, hipStream_t stream);

// The tokens with a gradient (r is not 0), in their order: count[0] of them (one with r
// 0 where there is none), their numbers, and their r, lse and labels; where[n] the place
// of token n among them, -1 of the others.
struct LiveTokens {
    int* count = nullptr;
    int* token = nullptr;
    int* where = nullptr;
    float* r = nullptr;
    float* lse = nullptr;
    int64_t* labels = nullptr;
};
// r[n] = coef[n] / c and scale[0] = c, with coef the factor of token n's row of G (0
// without a target) and c the largest of their magnitudes.  live.count NULL: not wanted.
// Coefficients, X transposed (XT null: not) and all of W (WT null: not) in one launch,
// where supported and no list of live tokens is wanted.
bool loss_prepare_supported(int64_t N, int64_t V, int64_t K);
hipError_t launch_loss_prepare(const float* dloss, const int64_t* labels, const float* mass, float t, int N, int V, int K,
                               float* r, float* scale, const void* X, int64_t ldx_, void* XT, int64_t ldxt, int64_t ldn,
                               int terms, const void* W, int64_t ldw, void* WT, int64_t ldwt, bool f32,
                               hipStream_t stream);
hipError_t launch_loss_coef(const float* dloss, const int64_t* labels, const float* mass, float t, int N, int V,
                            float* r, float* scale, const float* lse, const LiveTokens& live, hipStream_t stream);
// A piece of G, N rows and `cols` columns, and its transpose (either NULL: not wanted).
// terms 2: bfloat16 entries as a sum of two, the second ldx rows on in G and ldx columns
// on in GT; rows and columns [N, ldx) of either are then zeros.
struct GradOut {
    void* G = nullptr;
    int64_t ldg = 0;
    void* GT = nullptr;
    int64_t ldgt = 0;
    int64_t ldx = 0;
    int terms = 1;
    bool f32 = false;
    const int* where = nullptr;     // rows of live tokens alone
};
// G of columns [c0, c0 + cols) from their logits; entries: with those of a teacher,
// else they are launch_loss_fix's.
hipError_t launch_loss_grad(const Logits& S, int N, int c0, int cols, float inv_t, const float* lse,
                            const float* r, const LossTargets& t, bool entries, const GradOut& out,
                            hipStream_t stream);
// The teacher's entries among these columns, from their logits `picked`.
hipError_t launch_loss_fix(const LossTargets& t, const float* picked, int64_t ldpk, const float* lse, const float* r,
                           int N, int c0, int cols, const GradOut& out, hipStream_t stream);
// dst[k][n] = X[n][k], 0 where r[n] is 0 and in the columns [N, ldx); terms 2: once
// more ldx columns on.
// live: dst[k][i] = X[token[i]][k] of the live tokens (terms 1; columns past them are
// not all written).
hipError_t launch_transpose_live(const void* X, int64_t ldx_, const float* r, int N, int K, void* dst, int64_t ldd,
                                 int64_t ldx, int terms, bool f32, const LiveTokens* live, hipStream_t stream);
// acc += src (rows of ld elements, a multiple of 4)
hipError_t launch_add_f32(float* acc, const float* src, int64_t elems, hipStream_t stream);
// out[r][c] = scale[0]·Σ of `slabs` of src, `stride` apart, in their order; live: of the
// live tokens' rows, to their rows of out
hipError_t launch_sum_out(const float* src, int64_t lds, int slabs, int64_t stride, const float* scale, void* out,
                          int64_t ldo, int64_t R, int64_t C, bool f32, const LiveTokens* live, hipStream_t stream);
// zeros in the rows of the tokens without a gradient (r 0; bfloat16)
hipError_t launch_zero_dead(const float* r, void* out, int64_t ldo, int N, int64_t C, hipStream_t stream);
// zeros in the columns [0, C) of R rows
hipError_t launch_zero(void* out, int64_t ldo, int64_t R, int64_t C, bool f32, hipStream_t stream);

// ---- embedding -----------------------------------------------------------------
hipError_t launch_embedding(const int64_t* tokens, const void* E, int64_t lde, void* X, int64_t ldx, int64_t N,
                            int64_t K, int64_t V, float scale, bool f32, hipStream_t stream);
size_t embedding_workspace_bytes(int64_t N, int64_t K, int64_t V);
hipError_t launch_embedding_backward(const int64_t* tokens, const void* dX, int64_t lddx, void* dE, int64_t ldde,
                                     int64_t N, int64_t K, int64_t V, float scale, bool accumulate, bool f32,
                                     void* workspace, hipStream_t stream);

}  // namespace espace
