// C entry points of the losses on a linear head's logits and of the embedding: the
// checks of their arguments, the pieces of the vocabulary, and the launches.
#include "espace_train.h"

#include <cmath>
#include <algorithm>

#include "api.hpp"
#include "kernels.hpp"
#include "train.hpp"

using namespace espace::api;

namespace {

using espace::LossTargets;

constexpr int64_t kMaxTokens = (int64_t)1 << 22;

int64_t ld8(int64_t c) { return (c + 7) / 8 * 8; }

// Columns of a piece of the logits: about 2^25 of them (128 MB of float32, half the
// Infinity Cache), in pieces of equal width, a multiple of 256.
int64_t piece_cols(int64_t N, int64_t V) {
    const int64_t most = std::max<int64_t>(((int64_t)1 << 25) / std::max<int64_t>(N, 1) / 256, 1) * 256;
    const int64_t pieces = (V + most - 1) / most;
    return std::min(((V + pieces - 1) / pieces + 255) / 256 * 256, V);
}

struct Layout {
    size_t S, part, picked, col, p, logp, total;             // forward
    size_t mass, r, scale, XT, G, GT, WT, acc, slab, out;    // backward
    int64_t P, lds, nparts;
    int64_t ldn, ldp, ldk;
};

Layout loss_layout(bool backward, int64_t N, int64_t K, int64_t V, int64_t T, espace_dtype dt) {
    Layout b{};
    const size_t es = elem_size(dt);
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o = align_ws(o + bytes);
        return at;
    };
    b.P = piece_cols(N, V);
    b.lds = espace::splitk_ld((int)b.P);
    const int64_t pieces = (V + b.P - 1) / b.P;
    b.nparts = pieces * ((b.P + espace::STAT_COLS - 1) / espace::STAT_COLS);
    b.S = take((size_t)N * b.lds * 4);
    if (T > 0) {
        b.col = take((size_t)N * T * 4);
        b.p = take((size_t)N * T * 4);
    }
    if (!backward) {
        b.part = take((size_t)N * b.nparts * 8);
        if (T > 0) b.logp = take((size_t)N * T * 4);
        else b.picked = take((size_t)N * 4);
        b.total = o;
        return b;
    }
    b.ldn = ld8(N);
    b.ldp = ld8(b.P);
    b.ldk = espace::splitk_ld((int)K);
    if (T > 0) b.mass = take((size_t)N * 4);
    b.r = take((size_t)N * 4);
    b.scale = take(4);
    b.XT = take((size_t)K * b.ldn * es);
    b.G = take((size_t)N * b.ldp * es);
    b.GT = take((size_t)b.P * b.ldn * es);
    b.WT = take((size_t)K * b.ldp * es);
    b.acc = take((size_t)N * b.ldk * 4);
    if (pieces > 1) b.slab = take((size_t)N * b.ldk * 4);
    b.out = take((size_t)b.P * b.ldk * 4);
    b.total = o;
    return b;
}

espace_status check_sizes(int64_t N, int64_t K, int64_t V) {
    if (N < 0 || N >= kMaxTokens) return fail(ESPACE_ERR_SHAPE, "need 0 <= N < 2^22 tokens (N=%lld)", (long long)N);
    if (K < 1 || K > kMaxDim || V < 1 || V > kMaxDim)
        return fail(ESPACE_ERR_SHAPE, "need 1 <= K, V <= 2^30 (K=%lld, V=%lld)", (long long)K, (long long)V);
    return ESPACE_OK;
}

espace_status check_array(const char* name, const void* p, size_t align) {
    if (!p) return fail(ESPACE_ERR_NULL, "%s is NULL", name);
    if ((uintptr_t)p % align) return fail(ESPACE_ERR_ALIGN, "%s: pointer not %zu-byte aligned", name, align);
    return ESPACE_OK;
}

// [rows][cols] of elements of `size` bytes, rows ld apart
espace_status check_rows(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, size_t size) {
    ESPACE_TRY(check_array(name, p, size));
    if (ld < cols || ld > kMaxDim * 4 || rows * ld > ((int64_t)1 << 40))
        return fail(ESPACE_ERR_SHAPE, "%s: leading dimension %lld for %lld columns", name, (long long)ld,
                    (long long)cols);
    return ESPACE_OK;
}

Range bytes(const char* name, const void* p, size_t n) {
    return Range{name, (uintptr_t)p, (uintptr_t)p + (p ? n : 0)};
}
// the elements that a [rows][cols] array has: the last row ends at its last column
Range rows_range(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, size_t size) {
    return bytes(name, p, (size_t)((rows - 1) * ld + cols) * size);
}

espace_status check_outputs(const Range* outs, int nout, const Range* ins, int nin) {
    for (int i = 0; i < nout; ++i) {
        if (outs[i].lo == outs[i].hi) continue;
        ESPACE_TRY(check_alias(outs[i], ins, nin));
        ESPACE_TRY(check_alias(outs[i], outs, i));
    }
    return ESPACE_OK;
}

espace_status check_teacher(const int64_t* index, int64_t ldi, const float* logits, int64_t ldl, const float* picked,
                            int64_t ldpk, int64_t N, int64_t T) {
    ESPACE_TRY(check_rows("index", index, N, T, ldi, 8));
    ESPACE_TRY(check_rows("logits", logits, N, T, ldl, 4));
    return check_rows("picked", picked, N, T, ldpk, 4);
}

espace_status check_temperature(int64_t T, float t) {
    if (T < 1 || T > ESPACE_MAX_TEACHER_ENTRIES)
        return fail(ESPACE_ERR_SHAPE, "need 1 <= T <= %d (T=%lld)", ESPACE_MAX_TEACHER_ENTRIES, (long long)T);
    if (!(t > 0.f) || !std::isfinite(t) || !std::isfinite(1.f / t) || !std::isfinite(t * t))
        return fail(ESPACE_ERR_SHAPE, "temperature must be positive and finite, its square and inverse too (%g)", (double)t);
    return ESPACE_OK;
}

#define ESPACE_LAUNCH(what, x)                                                              \
    do {                                                                                    \
        const hipError_t _e = (x);                                                          \
        if (_e != hipSuccess) return fail(ESPACE_ERR_HIP, what ": %s", hipGetErrorString(_e)); \
    } while (0)

// columns [c0, c0 + cols) of the logits, float32
espace_status logits_piece(const void* X, int64_t ldx, const void* W, int64_t ldw, float* S, int64_t N, int64_t K,
                           int64_t c0, int64_t cols, espace_dtype dt, hipStream_t stream) {
    return run_tn_f32(X, ldx, (const char*)W + (size_t)c0 * ldw * elem_size(dt), ldw, S,
                      espace::splitk_ld((int)cols), N, cols, K, dt, stream);
}

espace_status loss_forward(const void* X, int64_t ldx, const void* W, int64_t ldw, LossTargets t, float* loss,
                           float* lse, float* picked, int64_t ldpk, int64_t N, int64_t K, int64_t V,
                           float temperature, espace_dtype dt, const Layout& b, char* ws, hipStream_t stream) {
    float* S = (float*)(ws + b.S);
    float2* part = (float2*)(ws + b.part);
    int part0 = 0;
    for (int64_t c0 = 0; c0 < V; c0 += b.P) {
        const int64_t cols = std::min(b.P, V - c0);
        ESPACE_TRY(logits_piece(X, ldx, W, ldw, S, N, K, c0, cols, dt, stream));
        ESPACE_LAUNCH("loss statistics",
                      espace::launch_loss_stats(S, espace::splitk_ld((int)cols), (int)N, (int)c0, (int)cols,
                                                1.f / temperature, t, part, (int)b.nparts, part0, picked, ldpk, stream));
        part0 += (int)((cols + espace::STAT_COLS - 1) / espace::STAT_COLS);
    }
    // the last piece may have had fewer parts than the others
    ESPACE_LAUNCH("loss", espace::launch_loss_finish(part, (int)b.nparts, part0, (int)N, (int)V, temperature, t, picked,
                                                     ldpk, loss, lse, stream));
    return ESPACE_OK;
}

espace_status loss_backward(const void* X, int64_t ldx, const void* W, int64_t ldw, const LossTargets& t,
                            const float* dloss, const float* mass, const float* lse, const float* picked, int64_t ldpk,
                            void* dX, int64_t lddx, void* dW, int64_t lddw, int64_t N, int64_t K, int64_t V,
                            float temperature, espace_dtype dt, const Layout& b, char* ws, hipStream_t stream) {
    const bool f32 = dt == ESPACE_F32;
    const size_t es = elem_size(dt);
    float* S = (float*)(ws + b.S);
    float* r = (float*)(ws + b.r);
    float* scale = (float*)(ws + b.scale);
    float* acc = (float*)(ws + b.acc);
    float* slab = (float*)(ws + b.slab);
    float* out = (float*)(ws + b.out);
    void *XT = ws + b.XT, *G = ws + b.G, *GT = ws + b.GT, *WT = ws + b.WT;
    ESPACE_LAUNCH("loss coefficients", espace::launch_loss_coef(dloss, t.labels, mass, temperature, (int)N, (int)V, r,
                                                                scale, stream));
    if (dW) ESPACE_LAUNCH("transpose", espace::launch_transpose_live(X, ldx, r, (int)N, (int)K, XT, b.ldn, f32, stream));
    for (int64_t c0 = 0; c0 < V; c0 += b.P) {
        const int64_t cols = std::min(b.P, V - c0);
        const int64_t lds = espace::splitk_ld((int)cols);
        const char* Wp = (const char*)W + (size_t)c0 * ldw * es;
        ESPACE_TRY(logits_piece(X, ldx, W, ldw, S, N, K, c0, cols, dt, stream));
        ESPACE_LAUNCH("logits' gradient", espace::launch_loss_grad(S, lds, (int)N, (int)c0, (int)cols,
                                                                   1.f / temperature, lse, r, t.labels, G, b.ldp, GT,
                                                                   b.ldn, f32, stream));
        if (!t.labels)
            ESPACE_LAUNCH("teacher's entries", espace::launch_loss_fix(t, picked, ldpk, lse, r, (int)N, (int)c0,
                                                                       (int)cols, G, b.ldp, GT, b.ldn, f32, stream));
        if (dX) {
            ESPACE_LAUNCH("transpose", espace::launch_transpose(Wp, ldw, (int)cols, (int)K, WT, b.ldp, f32, stream));
            ESPACE_TRY(run_tn_f32(G, b.ldp, WT, b.ldp, c0 ? slab : acc, b.ldk, N, K, cols, dt, stream));
            if (c0) ESPACE_LAUNCH("sum", espace::launch_add_f32(acc, slab, N * b.ldk, stream));
        }
        if (dW) {
            ESPACE_TRY(run_tn_f32(GT, b.ldn, XT, b.ldn, out, b.ldk, cols, K, N, dt, stream));
            ESPACE_LAUNCH("gradient", espace::launch_scale_out(out, b.ldk, scale, (char*)dW + (size_t)c0 * lddw * es,
                                                               lddw, cols, K, f32, stream));
        }
    }
    if (dX) ESPACE_LAUNCH("gradient", espace::launch_scale_out(acc, b.ldk, scale, dX, lddx, N, K, f32, stream));
    return ESPACE_OK;
}

// Both forward calls; T = 0: labels.
espace_status forward(const void* X, int64_t ldx, const void* W, int64_t ldw, const int64_t* labels,
                      const int64_t* index, int64_t ldi, const float* logits, int64_t ldl, float* loss, float* lse,
                      float* picked, int64_t ldpk, int64_t N, int64_t K, int64_t V, int64_t T, float temperature,
                      espace_dtype dt, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    ESPACE_TRY(check_mat("X", X, N, K, ldx, dt));
    ESPACE_TRY(check_mat("W", W, V, K, ldw, dt));
    if (T) ESPACE_TRY(check_teacher(index, ldi, logits, ldl, picked, ldpk, N, T));
    else ESPACE_TRY(check_array("labels", labels, 8));
    ESPACE_TRY(check_array("loss", loss, 4));
    ESPACE_TRY(check_array("lse", lse, 4));
    const Layout b = loss_layout(false, N, K, V, T, dt);
    ESPACE_TRY(check_workspace(workspace, workspace_bytes, b.total));
    const Range ins[] = {mat_range("X", X, N, ldx, dt), mat_range("W", W, V, ldw, dt),
                         T ? rows_range("index", index, N, T, ldi, 8) : bytes("labels", labels, N * 8),
                         T ? rows_range("logits", logits, N, T, ldl, 4) : Range{"logits", 0, 0}};
    const Range outs[] = {bytes("workspace", workspace, workspace_bytes), bytes("loss", loss, N * 4),
                          bytes("lse", lse, N * 4),
                          T ? rows_range("picked", picked, N, T, ldpk, 4) : Range{"picked", 0, 0}};
    ESPACE_TRY(check_outputs(outs, 4, ins, 4));
    ESPACE_TRY(check_device());
    char* ws = (char*)workspace;
    LossTargets t;
    t.labels = labels;
    if (T) {
        t.col = (int*)(ws + b.col);
        t.p = (float*)(ws + b.p);
        t.logp = (float*)(ws + b.logp);
        t.T = (int)T;
        ESPACE_LAUNCH("teacher", espace::launch_teacher(index, ldi, logits, ldl, (int)N, (int)T, (int)V,
                                                        1.f / temperature, false, (int*)(ws + b.col),
                                                        (float*)(ws + b.p), (float*)(ws + b.logp), nullptr, stream));
    } else {
        picked = (float*)(ws + b.picked);
        ldpk = 1;
    }
    return loss_forward(X, ldx, W, ldw, t, loss, lse, picked, ldpk, N, K, V, temperature, dt, b, ws, stream);
}

// Both backward calls; T = 0: labels.
espace_status backward(const float* dloss, const void* X, int64_t ldx, const void* W, int64_t ldw,
                       const int64_t* labels, const int64_t* index, int64_t ldi, const float* logits, int64_t ldl,
                       const float* lse, const float* picked, int64_t ldpk, void* dX, int64_t lddx, void* dW,
                       int64_t lddw, int64_t N, int64_t K, int64_t V, int64_t T, float temperature, espace_dtype dt,
                       void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (dW) ESPACE_TRY(check_mat("dW", dW, V, K, lddw, dt));
    if (N == 0) {
        // the gradient of no tokens
        if (!dW) return ESPACE_OK;
        ESPACE_TRY(check_device());
        ESPACE_LAUNCH("gradient", espace::launch_zero(dW, lddw, V, K, dt == ESPACE_F32, stream));
        return ESPACE_OK;
    }
    if (!dX && !dW) return ESPACE_OK;
    ESPACE_TRY(check_mat("X", X, N, K, ldx, dt));
    ESPACE_TRY(check_mat("W", W, V, K, ldw, dt));
    ESPACE_TRY(check_array("dloss", dloss, 4));
    if (T) ESPACE_TRY(check_teacher(index, ldi, logits, ldl, picked, ldpk, N, T));
    else ESPACE_TRY(check_array("labels", labels, 8));
    ESPACE_TRY(check_array("lse", lse, 4));
    if (dX) ESPACE_TRY(check_mat("dX", dX, N, K, lddx, dt));
    const Layout b = loss_layout(true, N, K, V, T, dt);
    ESPACE_TRY(check_workspace(workspace, workspace_bytes, b.total));
    const Range ins[] = {mat_range("X", X, N, ldx, dt), mat_range("W", W, V, ldw, dt),
                         T ? rows_range("index", index, N, T, ldi, 8) : bytes("labels", labels, N * 8),
                         T ? rows_range("logits", logits, N, T, ldl, 4) : Range{"logits", 0, 0},
                         T ? rows_range("picked", picked, N, T, ldpk, 4) : Range{"picked", 0, 0},
                         bytes("dloss", dloss, N * 4), bytes("lse", lse, N * 4)};
    const Range outs[] = {bytes("workspace", workspace, workspace_bytes),
                          dX ? mat_range("dX", dX, N, lddx, dt) : Range{"dX", 0, 0},
                          dW ? mat_range("dW", dW, V, lddw, dt) : Range{"dW", 0, 0}};
    ESPACE_TRY(check_outputs(outs, 3, ins, 7));
    ESPACE_TRY(check_device());
    char* ws = (char*)workspace;
    LossTargets t;
    t.labels = labels;
    float* mass = (float*)(ws + b.mass);
    if (T) {
        t.col = (int*)(ws + b.col);
        t.p = (float*)(ws + b.p);
        t.T = (int)T;
        ESPACE_LAUNCH("teacher", espace::launch_teacher(index, ldi, logits, ldl, (int)N, (int)T, (int)V,
                                                        1.f / temperature, true, (int*)(ws + b.col),
                                                        (float*)(ws + b.p), nullptr, mass, stream));
    }
    return loss_backward(X, ldx, W, ldw, t, dloss, mass, lse, picked, ldpk, dX, lddx, dW, lddw, N, K, V, temperature,
                         dt, b, ws, stream);
}

}  // namespace

extern "C" {

size_t espace_linear_loss_workspace_bytes(int backward, int64_t N, int64_t K, int64_t V, int64_t T,
                                          espace_dtype dt) {
    if (dt != ESPACE_F32 && dt != ESPACE_BF16) return SIZE_MAX;
    if (N < 0 || N >= kMaxTokens || K < 1 || K > kMaxDim || V < 1 || V > kMaxDim) return SIZE_MAX;
    if (T < 0 || T > ESPACE_MAX_TEACHER_ENTRIES) return SIZE_MAX;
    return N ? loss_layout(backward != 0, N, K, V, T, dt).total : 0;
}

espace_status espace_linear_cross_entropy(const void* X, int64_t ldx, const void* W, int64_t ldw,
                                          const int64_t* labels, float* loss, float* lse, int64_t N, int64_t K,
                                          int64_t V, espace_dtype dt, void* workspace, size_t workspace_bytes,
                                          hipStream_t stream) {
    ESPACE_TRY(check_dtype(dt));
    ESPACE_TRY(check_sizes(N, K, V));
    if (N == 0) return ok();
    ESPACE_TRY(forward(X, ldx, W, ldw, labels, nullptr, 0, nullptr, 0, loss, lse, nullptr, 0, N, K, V, 0, 1.f, dt,
                       workspace, workspace_bytes, stream));
    return ok();
}

espace_status espace_linear_cross_entropy_backward(const float* dloss, const void* X, int64_t ldx, const void* W,
                                                   int64_t ldw, const int64_t* labels, const float* lse, void* dX,
                                                   int64_t lddx, void* dW, int64_t lddw, int64_t N, int64_t K,
                                                   int64_t V, espace_dtype dt, void* workspace,
                                                   size_t workspace_bytes, hipStream_t stream) {
    ESPACE_TRY(check_dtype(dt));
    ESPACE_TRY(check_sizes(N, K, V));
    ESPACE_TRY(backward(dloss, X, ldx, W, ldw, labels, nullptr, 0, nullptr, 0, lse, nullptr, 0, dX, lddx, dW, lddw, N,
                        K, V, 0, 1.f, dt, workspace, workspace_bytes, stream));
    return ok();
}

espace_status espace_linear_distillation(const void* X, int64_t ldx, const void* W, int64_t ldw, const int64_t* index,
                                         int64_t ldi, const float* logits, int64_t ldl, float* loss, float* lse,
                                         float* picked, int64_t ldpk, int64_t N, int64_t K, int64_t V, int64_t T,
                                         float temperature, espace_dtype dt, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream) {
    ESPACE_TRY(check_dtype(dt));
    ESPACE_TRY(check_sizes(N, K, V));
    ESPACE_TRY(check_temperature(T, temperature));
    if (N == 0) return ok();
    ESPACE_TRY(forward(X, ldx, W, ldw, nullptr, index, ldi, logits, ldl, loss, lse, picked, ldpk, N, K, V, T,
                       temperature, dt, workspace, workspace_bytes, stream));
    return ok();
}

espace_status espace_linear_distillation_backward(const float* dloss, const void* X, int64_t ldx, const void* W,
                                                  int64_t ldw, const int64_t* index, int64_t ldi, const float* logits,
                                                  int64_t ldl, const float* lse, const float* picked, int64_t ldpk,
                                                  void* dX, int64_t lddx, void* dW, int64_t lddw, int64_t N,
                                                  int64_t K, int64_t V, int64_t T, float temperature,
                                                  espace_dtype dt, void* workspace, size_t workspace_bytes,
                                                  hipStream_t stream) {
    ESPACE_TRY(check_dtype(dt));
    ESPACE_TRY(check_sizes(N, K, V));
    ESPACE_TRY(check_temperature(T, temperature));
    ESPACE_TRY(backward(dloss, X, ldx, W, ldw, nullptr, index, ldi, logits, ldl, lse, picked, ldpk, dX, lddx, dW, lddw,
                        N, K, V, T, temperature, dt, workspace, workspace_bytes, stream));
    return ok();
}

espace_status espace_embedding(const int64_t* tokens, const void* E, int64_t lde, void* X, int64_t ldx, int64_t N,
                               int64_t K, int64_t V, float scale, espace_dtype dt, hipStream_t stream) {
    ESPACE_TRY(check_dtype(dt));
    ESPACE_TRY(check_sizes(N, K, V));
    if (N == 0) return ok();
    ESPACE_TRY(check_array("tokens", tokens, 8));
    ESPACE_TRY(check_mat("E", E, V, K, lde, dt));
    ESPACE_TRY(check_mat("X", X, N, K, ldx, dt));
    const Range ins[] = {bytes("tokens", tokens, N * 8), mat_range("E", E, V, lde, dt)};
    ESPACE_TRY(check_alias(mat_range("X", X, N, ldx, dt), ins, 2));
    ESPACE_TRY(check_device());
    ESPACE_LAUNCH("embedding", espace::launch_embedding(tokens, E, lde, X, ldx, N, K, V, scale, dt == ESPACE_F32,
                                                        stream));
    return ok();
}

size_t espace_embedding_workspace_bytes(int64_t N, int64_t K, int64_t V) {
    if (N < 0 || N >= kMaxTokens || K < 1 || K > kMaxDim || V < 1 || V > kMaxDim) return SIZE_MAX;
    return N ? align_ws(espace::embedding_workspace_bytes(N, K, V)) : 0;
}

espace_status espace_embedding_backward(const int64_t* tokens, const void* dX, int64_t lddx, void* dE, int64_t ldde,
                                        int64_t N, int64_t K, int64_t V, float scale, int accumulate,
                                        espace_dtype dt, void* workspace, size_t workspace_bytes,
                                        hipStream_t stream) {
    ESPACE_TRY(check_dtype(dt));
    ESPACE_TRY(check_sizes(N, K, V));
    ESPACE_TRY(check_mat("dE", dE, V, K, ldde, dt));
    if (N == 0) {
        if (accumulate) return ok();
        ESPACE_TRY(check_device());
        ESPACE_LAUNCH("embedding gradient", espace::launch_zero(dE, ldde, V, K, dt == ESPACE_F32, stream));
        return ok();
    }
    ESPACE_TRY(check_array("tokens", tokens, 8));
    ESPACE_TRY(check_mat("dX", dX, N, K, lddx, dt));
    const size_t need = align_ws(espace::embedding_workspace_bytes(N, K, V));
    ESPACE_TRY(check_workspace(workspace, workspace_bytes, need));
    const Range ins[] = {bytes("tokens", tokens, N * 8), mat_range("dX", dX, N, lddx, dt)};
    const Range outs[] = {bytes("workspace", workspace, workspace_bytes), mat_range("dE", dE, V, ldde, dt)};
    ESPACE_TRY(check_outputs(outs, 2, ins, 2));
    ESPACE_TRY(check_device());
    ESPACE_LAUNCH("embedding gradient",
                  espace::launch_embedding_backward(tokens, dX, lddx, dE, ldde, N, K, V, scale, accumulate != 0,
                                                    dt == ESPACE_F32, workspace, stream));
    return ok();
}

}  // extern "C"
