// C entry points of the losses on a linear head's logits and of the embedding: the
// checks of their arguments, the pieces of the vocabulary, and the launches.
#include "espace_train.h"

#include <cmath>
#include <cstdio>
#include <algorithm>

#include "api.hpp"
#include "kernels.hpp"
#include "train.hpp"

using namespace espace::api;

namespace {

using espace::LossTargets;

constexpr int64_t kMaxTokens = (int64_t)1 << 21, kMaxWidth = (int64_t)1 << 21;

int64_t ld8(int64_t c) { return (c + 7) / 8 * 8; }

// Columns of a piece of the vocabulary, a multiple of 256: the most that keep N·columns
// within `elems`, in whole rounds of 256 x 256 tiles on all CUs where those fit, else in
// pieces of equal width.
int64_t piece_cols(int64_t N, int64_t V, int64_t elems) {
    const int64_t most = std::max<int64_t>(elems / N / 256, 1) * 256;
    if (V <= most) return V;
    const int64_t tr = (N + 255) / 256;
    int64_t round = 256;                           // tile columns of whole rounds
    for (int64_t t = tr; t % 2 == 0 && round > 1; t /= 2) round /= 2;
    if (round * 256 <= most) return most / (round * 256) * (round * 256);
    const int64_t pieces = (V + most - 1) / most;
    return ((V + pieces - 1) / pieces + 255) / 256 * 256;
}

// Pieces that are kept as float32 logits: 128 MB, half the Infinity Cache.  Those of G
// where the logits stay in registers: as much, and as much again its transpose (twice
// that of half as wide pieces: 8192 tokens on 50257 x 6144 16.7 -> 15.9 ms, with fewer
// passes over dX's sums; 4096 on 32000 x 4096 3.46 -> 3.50).
constexpr int64_t kLogits = (int64_t)1 << 25, kGrads = (int64_t)1 << 26;
// Where the epilogues cannot take a call's leading dimensions: narrow pieces, which fit
// any layout.
constexpr int64_t kNarrow = 256;
// Tokens up to which a bfloat16 entry of G is kept as the sum of two: the products of so
// few are bound by reading W, so a second term costs little (65 tokens of 8 teacher's
// entries: dX and dW 2.4e-3 off, 1.7e-3 with two, the rounding of the results).
constexpr int64_t kTwoTerms = 128;
// Depth ranges of the logits' and dX's products whose sums the next pass adds, and the
// floats of them.
constexpr int64_t kRanges = 32, kRangeFloats = (int64_t)1 << 24;

int most_ranges(int64_t R, int64_t ld) { return (int)std::max<int64_t>(1, std::min(kRanges, kRangeFloats / (R * ld))); }

// How a gradient's product runs: on the tiles that take W, or G, as it lies, ending in
// the tiles' epilogue or in float32 sums of depth ranges; on the small tiles, ending
// there too; or as float32 sums of transposed operands that a pass of their own rounds.
struct Way {
    enum { SUMS, SMALL, EPILOGUE, RANGES } how = SUMS;
    int tile = -1;                // or the small tiles' configuration
    int ranges = 1;
    bool tiled() const { return how == EPILOGUE || how == RANGES; }
};
Way way_of(const F32Plan& p) {
    Way w;
    if (p.kind == F32Plan::TILED) w.how = p.ranges == 1 ? Way::EPILOGUE : Way::RANGES;
    else if (p.kind == F32Plan::MID && p.ranges == 1) w.how = Way::SMALL;
    w.tile = p.tile;
    w.ranges = p.ranges;
    return w;
}

struct Layout {
    size_t S, part, picked, col, p, logp, sorted, place, first;    // forward (S, col, p: both)
    size_t mass, r, scale, XT, G, GT, WT, acc, out, live, total;   // backward
    int tile;                    // >= 0: the logits' epilogues on this tile
    int64_t P;                   // columns of a piece
    int terms;
    Way x, w;                    // dX's and dW's products
    bool f32_x, f32_w;           // those of float32 read W, and G, as they lie
    int ranges_s, ranges_x;      // of the logits' (tile < 0) and dX's (sums) products, at most
    int64_t rows;                // of G, and of dX's sums: a second term's from ldn on
    int64_t ldn, ldp, ldk, ldfirst;
};

Layout loss_layout(bool backward, int64_t N, int64_t K, int64_t V, int64_t T, espace_dtype dt) {
    Layout b{};
    const size_t es = elem_size(dt);
    const bool bf16 = dt == ESPACE_BF16;
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o = align_ws(o + bytes);
        return at;
    };
    b.terms = bf16 && N <= kTwoTerms ? 2 : 1;
    b.P = backward ? piece_cols(N, V, kGrads) : V;
    b.tile = -1;
    if (bf16 && b.terms == 1) {
        const F32Plan p = f32_plan(b.P, N, K, ld8(K), ld8(K), 1, true);
        if (p.kind == F32Plan::TILED) b.tile = p.tile;
    }
    b.ranges_s = 1;
    if (b.tile < 0) {
        b.P = piece_cols(N, V, kLogits);
        b.ranges_s = most_ranges(N, espace::splitk_ld((int)b.P));
    }
    b.S = take((size_t)N * espace::splitk_ld((int)(b.tile < 0 ? b.P : std::min(V, kNarrow))) * 4 * b.ranges_s);
    if (T > 0) {
        b.col = take((size_t)N * T * 4);
        b.p = take((size_t)N * T * 4);
    }
    b.ldn = ld8(N);
    if (!backward) {
        if (b.tile >= 0) b.XT = take((size_t)K * b.ldn * es);
        const int64_t pieces = (V + b.P - 1) / b.P, stats = (b.P + espace::STAT_COLS - 1) / espace::STAT_COLS;
        const int64_t slabs = (V + espace::LOSS_SLAB - 1) / espace::LOSS_SLAB;
        b.part = take((size_t)N * (b.tile < 0 ? pieces * stats : std::max(slabs + 1, (V + kNarrow - 1) / kNarrow)) * 8);
        if (T > 0) {
            b.logp = take((size_t)N * T * 4);
            if (b.tile >= 0) {
                b.ldfirst = slabs + 2;
                b.sorted = take((size_t)N * T * 4);
                b.place = take((size_t)N * T * 2);
                b.first = take((size_t)N * b.ldfirst * 2);
            }
        } else {
            b.picked = take((size_t)N * 4);
        }
        b.total = o;
        return b;
    }
    const int64_t pieces = (V + b.P - 1) / b.P;
    b.ldp = ld8(b.P);
    b.ldk = espace::splitk_ld((int)K);
    if (T > 0) b.mass = take((size_t)N * 4);
    b.r = take((size_t)N * 4);
    b.scale = take(4);
    b.live = take((size_t)N * 24 + 8);           // count, then LiveTokens' arrays
    const int64_t ldgt = b.ldn * b.terms, depth = b.terms == 1 ? N : ldgt;
    b.rows = depth;
    b.ranges_x = pieces <= 4 ? most_ranges(b.rows, b.ldk) : 1;
    if (bf16) {
        // (either operand order of dW's product has this price)
        const F32Plan w = f32_plan(K, b.P, depth, ldgt, ldgt, 1, true), small = f32_plan(b.P, K, depth, ldgt, ldgt, 1);
        b.w = w.kind == F32Plan::TILED ? way_of(w) : (small.kind == F32Plan::MID ? way_of(small) : Way{});
        // (the small tiles take W transposed: read and written at 4.5 TB/s)
        const double turned = 3.0 + 4e-6 * K * b.P / 4.5;
        b.x = way_of(f32_plan(b.rows, K, b.P, b.ldp, b.ldp, b.ranges_x, true, turned));
        // two terms are added by the pass that rounds
        if (b.terms > 1 && b.x.how == Way::EPILOGUE) b.x.how = Way::RANGES;
        // the small tiles do not add to what is there, and the ranges of many pieces
        // find no room
        if ((b.x.how == Way::SMALL && (pieces > 1 || b.terms > 1)) || (b.x.how == Way::RANGES && pieces > 4)) b.x = Way{};
    }
    b.f32_x = !bf16 && espace::gemm_tn_f32_terms_supported(N, K, b.P, b.ldp, K, false, true);
    b.f32_w = !bf16 && espace::gemm_tn_f32_terms_supported(b.P, K, N, b.ldp, ldgt, true, false);
    // Narrow pieces, which take transposed operands and float32 sums, may be needed
    // where the tiles are planned.
    const bool tiles = b.tile >= 0 || b.x.tiled() || b.f32_x;
    const int64_t narrow = ld8(std::min(V, kNarrow));
    b.XT = take((size_t)K * ldgt * es);
    b.G = take((size_t)b.rows * b.ldp * es);
    b.GT = take((size_t)(b.w.tiled() || b.f32_w ? narrow : b.P) * ldgt * es);
    b.WT = take((size_t)K * (b.x.tiled() || b.f32_x ? narrow : b.ldp) * es);
    // sums of dX: of more than one piece to be added to, or ranges, or two pieces'
    int64_t sums = std::min<int64_t>(pieces, 2);
    if (b.x.how == Way::EPILOGUE || b.x.how == Way::SMALL) sums = pieces > 1 ? 1 : 0;
    else if (pieces <= 4) sums = b.ranges_x * pieces;
    if (tiles) sums = std::max<int64_t>(sums, 2);
    b.acc = take((size_t)b.rows * b.ldk * 4 * sums);
    b.out = take((size_t)(b.w.how != Way::SUMS || b.f32_w ? narrow : b.P) * b.ldk * 4);
    b.total = o;
    return b;
}

espace_status check_sizes(int64_t N, int64_t K, int64_t V) {
    if (N < 0 || N >= kMaxTokens) return fail(ESPACE_ERR_SHAPE, "need 0 <= N < 2^21 tokens (N=%lld)", (long long)N);
    if (K < 1 || K > kMaxWidth || V < 1 || V > kMaxDim)
        return fail(ESPACE_ERR_SHAPE, "need 1 <= K <= 2^21 and 1 <= V <= 2^30 (K=%lld, V=%lld)", (long long)K, (long long)V);
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

const int64_t kLim = (int64_t)1 << 31;

// columns [c0, c0 + cols) of the logits, float32
espace_status logits_piece(const void* X, int64_t ldx, const void* W, int64_t ldw, float* S, int64_t N, int64_t K,
                           int64_t c0, int64_t cols, espace_dtype dt, int ranges, espace::Logits* out,
                           hipStream_t stream) {
    out->S = S;
    out->lds = espace::splitk_ld((int)cols);
    out->stride = N * out->lds;
    return run_tn_f32(X, ldx, (const char*)W + (size_t)c0 * ldw * elem_size(dt), ldw, S, out->lds, N, cols, K, dt,
                      stream, ranges, &out->slabs);
}

void log_plan(const Layout& b, bool backward, bool fused, int64_t N, int64_t K, int64_t V, int64_t T, int64_t P) {
    if (!plan_log()) return;
    std::fprintf(stderr,
                 "espace loss plan N=%lld K=%lld V=%lld T=%lld: backward=%d fused=%d tile=%d columns=%lld terms=%d "
                 "x=%d w=%d ranges_s=%d ranges_x=%d\n",
                 (long long)N, (long long)K, (long long)V, (long long)T, backward, fused, b.tile, (long long)P, b.terms,
                 (int)b.x.how, (int)b.w.how, b.ranges_s, b.ranges_x);
}

espace_status loss_forward(const void* X, int64_t ldx, const void* W, int64_t ldw, LossTargets t, float* loss,
                           float* lse, float* picked, int64_t ldpk, int64_t N, int64_t K, int64_t V,
                           float temperature, espace_dtype dt, const Layout& b, char* ws, hipStream_t stream) {
    float* S = (float*)(ws + b.S);
    float2* part = (float2*)(ws + b.part);
    const float inv_t = 1.f / temperature;
    int parts = 0;
    // the epilogue's launches: rows of W below 2^31 elements, in whole slabs
    const int64_t step = 256;
    const bool fused = b.tile >= 0 && K * b.ldn < kLim && std::min(V, step) * ldw < kLim;
    log_plan(b, false, fused, N, K, V, t.labels ? 0 : t.T, fused ? V : (b.tile >= 0 ? std::min(V, kNarrow) : b.P));
    if (fused) {
        const int64_t most = V * ldw < kLim ? V : (kLim - 1) / ldw / step * step;
        void* XT = ws + b.XT;
        ESPACE_LAUNCH("transpose", espace::launch_transpose(X, ldx, (int)N, (int)K, XT, b.ldn, false, stream));
        for (int64_t c0 = 0; c0 < V; c0 += most) {
            const int64_t cols = std::min(most, V - c0);
            espace::LossEpi e;
            e.inv_t = inv_t;
            e.col0 = (int)c0;
            e.labels = t.labels;
            e.part = part + (size_t)(c0 / espace::LOSS_SLAB) * N;
            e.picked = picked;
            e.ldpk = ldpk;
            if (!t.labels) {
                e.col = (int*)(ws + b.sorted);
                e.place = (uint16_t*)(ws + b.place);
                e.first = (uint16_t*)(ws + b.first);
                e.ldfirst = b.ldfirst;
                e.T = t.T;
            }
            ESPACE_TRY(run_tn_loss((const uint16_t*)W + c0 * ldw, ldw, XT, b.ldn, nullptr, 0, cols, N, K, b.tile,
                                   espace::LOSS_STATS, e, stream));
        }
        parts = (int)((V + espace::LOSS_SLAB - 1) / espace::LOSS_SLAB);
    } else {
        const int64_t P = b.tile >= 0 ? std::min(V, kNarrow) : b.P;
        for (int64_t c0 = 0; c0 < V; c0 += P) {
            const int64_t cols = std::min(P, V - c0);
            espace::Logits s;
            ESPACE_TRY(logits_piece(X, ldx, W, ldw, S, N, K, c0, cols, dt, b.ranges_s, &s, stream));
            if (cols == V && V <= espace::STAT_COLS) {
                ESPACE_LAUNCH("loss", espace::launch_loss_whole(s, (int)N, (int)V, temperature, t, picked, ldpk, loss,
                                                                lse, stream));
                return ESPACE_OK;
            }
            ESPACE_LAUNCH("loss statistics", espace::launch_loss_stats(s, (int)N, (int)c0, (int)cols, inv_t, t, part,
                                                                       parts, picked, ldpk, stream));
            parts += (int)((cols + espace::STAT_COLS - 1) / espace::STAT_COLS);
        }
    }
    ESPACE_LAUNCH("loss", espace::launch_loss_finish(part, parts, (int)N, (int)V, temperature, t, picked, ldpk, loss,
                                                     lse, stream));
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
    float* out = (float*)(ws + b.out);
    void *XT = ws + b.XT, *G = ws + b.G, *GT = ws + b.GT, *WT = ws + b.WT;
    const float inv_t = 1.f / temperature;
    // leading dimensions past the tiles' offsets: narrow pieces and float32 sums
    const bool narrow = ((b.tile >= 0 || b.x.tiled()) && (b.P * ldw >= kLim || K * b.ldn * b.terms >= kLim)) ||
                        (b.f32_x && !espace::gemm_tn_f32_terms_supported(N, K, b.P, b.ldp, ldw, false, true));
    const bool fused = b.tile >= 0 && !narrow;
    const int64_t P = narrow ? std::min(V, kNarrow) : b.P;
    const int64_t pieces = (V + P - 1) / P;
    const Way wx = narrow ? Way{} : b.x, ww = narrow ? Way{} : b.w;
    // the products of the tokens with a gradient alone, where all of them can (also where
    // one is not wanted: the other has the same bits then)
    const bool compact = fused && wx.tiled() && ww.tiled();
    espace::LiveTokens live;
    if (compact) {
        live.labels = (int64_t*)(ws + b.live);
        live.token = (int*)(live.labels + N);
        live.where = live.token + N;
        live.r = (float*)(live.where + N);
        live.lse = live.r + N;
        live.count = (int*)(live.lse + N);
    }
    const int64_t slab = b.rows * b.ldk;                        // of dX's sums
    const bool many = pieces <= 4 && !narrow;                   // their ranges stay apart
    const int64_t ldgt = b.ldn * b.terms, ldwt = ld8(P);
    // up to as many entries as a tile of G has columns: with the tile (its 64 tokens'
    // entries are looked through for each), else by a pass over the entries
    const bool few = !t.labels && !fused && t.T <= 64;
    int sums = 0;                                               // slabs in acc
    log_plan(b, true, fused, N, K, V, t.labels ? 0 : t.T, P);
    const bool turn_x = dW || fused, turn_w = dX && !wx.tiled() && !(f32 && b.f32_x && !narrow);
    const bool together = !compact && espace::loss_prepare_supported(N, V, K);
    const bool turned_w = together && turn_w && pieces == 1;
    if (together)
        ESPACE_LAUNCH("loss coefficients",
                      espace::launch_loss_prepare(dloss, t.labels, mass, temperature, (int)N, (int)V, (int)K, r, scale,
                                                  X, ldx, turn_x ? XT : nullptr, ldgt, b.ldn, b.terms, W, ldw,
                                                  turned_w ? WT : nullptr, ldwt, f32, stream));
    else
        ESPACE_LAUNCH("loss coefficients", espace::launch_loss_coef(dloss, t.labels, mass, temperature, (int)N, (int)V,
                                                                    r, scale, lse, live, stream));
    if (turn_x && !together)
        ESPACE_LAUNCH("transpose", espace::launch_transpose_live(X, ldx, r, (int)N, (int)K, XT, ldgt, b.ldn, b.terms,
                                                                 f32, compact ? &live : nullptr, stream));
    for (int64_t c0 = 0; c0 < V; c0 += P) {
        const int64_t cols = std::min(P, V - c0);
        const char* Wp = (const char*)W + (size_t)c0 * ldw * es;
        const bool last = c0 + cols == V;
        const bool fx = f32 && b.f32_x && !narrow;
        const bool fw = f32 && espace::gemm_tn_f32_terms_supported(cols, K, N, b.ldp, ldgt, true, false);
        espace::GradOut go;
        go.G = dX || fused || ww.tiled() || fw ? G : nullptr;
        go.ldg = b.ldp;
        go.GT = dW && !ww.tiled() && !fw ? GT : nullptr;
        go.ldgt = ldgt;
        go.ldx = b.ldn;
        go.terms = b.terms;
        go.f32 = f32;
        go.where = live.where;
        if (fused) {
            espace::LossEpi e;
            e.inv_t = inv_t;
            e.col0 = (int)c0;
            e.labels = t.labels ? (compact ? live.labels : t.labels) : nullptr;
            e.lse = compact ? live.lse : lse;
            e.r = compact ? live.r : r;
            e.count = live.count;
            e.GT = (uint16_t*)go.GT;
            e.ldgt = ldgt;
            ESPACE_TRY(run_tn_loss(Wp, ldw, XT, ldgt, G, b.ldp, cols, N, K, b.tile, espace::LOSS_GRAD, e, stream));
        } else {
            espace::Logits s;
            ESPACE_TRY(logits_piece(X, ldx, W, ldw, S, N, K, c0, cols, dt, b.ranges_s, &s, stream));
            ESPACE_LAUNCH("logits' gradient", espace::launch_loss_grad(s, (int)N, (int)c0, (int)cols, inv_t, lse, r, t,
                                                                       few, go, stream));
        }
        if (!t.labels && !few)
            ESPACE_LAUNCH("teacher's entries", espace::launch_loss_fix(t, picked, ldpk, lse, r, (int)N, (int)c0,
                                                                       (int)cols, go, stream));
        if (dX) {
            if (turn_w && !turned_w)
                ESPACE_LAUNCH("transpose", espace::launch_transpose(Wp, ldw, (int)cols, (int)K, WT, ldwt, f32, stream));
            if (wx.how == Way::EPILOGUE) {
                espace::LossEpi e;
                e.acc = acc;
                e.ldacc = b.ldk;
                e.scale = scale;
                e.add = c0 > 0;
                e.last = last;
                e.count = live.count;
                e.rows = live.token;
                ESPACE_TRY(run_tn_loss(G, b.ldp, Wp, ldw, dX, lddx, N, K, cols, wx.tile, espace::LOSS_GRAD_OUT, e,
                                       stream));
            } else if (wx.how == Way::RANGES) {
                int made = 1;
                ESPACE_TRY(run_tiled_ranges(G, b.ldp, Wp, ldw, acc + sums * slab, b.rows, K, cols, wx.tile, wx.ranges,
                                            live.count, &made, stream));
                sums += made;
            } else if (wx.how == Way::SMALL) {
                ESPACE_TRY(run_tn_scaled_mid(G, b.ldp, WT, ldwt, dX, lddx, N, K, cols, wx.tile, scale, stream));
            } else {
                int made = 1;
                float* to = acc + sums * slab;
                const int most = many ? b.ranges_x : 1;
                if (fx)
                    ESPACE_TRY(run_tn_f32_depth((const float*)G, b.ldp, false, (const float*)Wp, ldw, true, to, b.ldk, N,
                                                K, cols, nullptr, most, &made, stream));
                else
                    ESPACE_TRY(run_tn_f32(G, b.ldp, WT, ldwt, to, b.ldk, b.rows, K, cols, dt, stream, most, &made));
                if (many || !sums) sums += made;
                else ESPACE_LAUNCH("sum", espace::launch_add_f32(acc, acc + slab, slab, stream));
            }
        }
        if (dW) {
            void* o = (char*)dW + (size_t)c0 * lddw * es;
            const int64_t depth = b.rows;
            if (ww.how == Way::EPILOGUE) {
                espace::LossEpi e;
                e.scale = scale;
                e.last = 1;
                e.count = live.count;
                ESPACE_TRY(run_tn_loss(XT, ldgt, G, b.ldp, o, lddw, K, cols, depth, ww.tile, espace::LOSS_GRAD_OUT_T, e,
                                       stream));
            } else if (ww.how == Way::SMALL) {
                ESPACE_TRY(run_tn_scaled_mid(GT, ldgt, XT, ldgt, o, lddw, cols, K, depth, ww.tile, scale, stream));
            } else if (fw) {
                int made = 1;
                ESPACE_TRY(run_tn_f32_depth((const float*)G, b.ldp, true, (const float*)XT, ldgt, false, (float*)o, lddw,
                                            cols, K, N, scale, 1, &made, stream));
            } else {
                ESPACE_TRY(run_tn_f32(GT, ldgt, XT, ldgt, out, b.ldk, cols, K, depth, dt, stream));
                ESPACE_LAUNCH("gradient", espace::launch_sum_out(out, b.ldk, 1, 0, scale, o, lddw, cols, K, f32, nullptr,
                                                                 stream));
            }
        }
    }
    if (dX && (wx.how == Way::SUMS || wx.how == Way::RANGES))
        // a second term's rows are a slab of their own
        ESPACE_LAUNCH("gradient", espace::launch_sum_out(acc, b.ldk, sums * b.terms, slab / b.terms, scale, dX, lddx, N,
                                                         K, f32, compact ? &live : nullptr, stream));
    if (dX && compact) ESPACE_LAUNCH("gradient", espace::launch_zero_dead(r, dX, lddx, (int)N, K, stream));
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
        espace::TeacherOut to;
        to.col = (int*)(ws + b.col);
        to.p = (float*)(ws + b.p);
        to.logp = (float*)(ws + b.logp);
        if (b.tile >= 0) {
            to.sorted = (int*)(ws + b.sorted);
            to.place = (uint16_t*)(ws + b.place);
            to.first = (uint16_t*)(ws + b.first);
            to.ldfirst = b.ldfirst;
        }
        ESPACE_LAUNCH("teacher", espace::launch_teacher(index, ldi, logits, ldl, (int)N, (int)T, (int)V,
                                                        1.f / temperature, to, stream));
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
        espace::TeacherOut to;
        to.col = (int*)(ws + b.col);
        to.p = (float*)(ws + b.p);
        to.mass = mass;
        ESPACE_LAUNCH("teacher", espace::launch_teacher(index, ldi, logits, ldl, (int)N, (int)T, (int)V,
                                                        1.f / temperature, to, stream));
    }
    return loss_backward(X, ldx, W, ldw, t, dloss, mass, lse, picked, ldpk, dX, lddx, dW, lddw, N, K, V, temperature,
                         dt, b, ws, stream);
}

}  // namespace

extern "C" {

size_t espace_linear_loss_workspace_bytes(int backward, int64_t N, int64_t K, int64_t V, int64_t T,
                                          espace_dtype dt) {
    if (dt != ESPACE_F32 && dt != ESPACE_BF16) return SIZE_MAX;
    if (N < 0 || N >= kMaxTokens || K < 1 || K > kMaxWidth || V < 1 || V > kMaxDim) return SIZE_MAX;
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
    if (N < 0 || N >= kMaxTokens || K < 1 || K > kMaxWidth || V < 1 || V > kMaxDim) return SIZE_MAX;
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
