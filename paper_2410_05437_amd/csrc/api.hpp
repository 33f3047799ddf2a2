// What the C entry points share (espace_api.hip defines it): statuses, the checks
// of arguments, and products of two matrices under the library's plans.
#pragma once

#include "espace.h"

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kernels.hpp"

namespace espace {
namespace api {

constexpr int64_t kMaxDim = (int64_t)1 << 30;
constexpr size_t kWsAlign = 256;

// Sets the thread's last error and returns the status; ok() clears it.
espace_status fail(espace_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
espace_status ok();

size_t elem_size(espace_dtype dt);
size_t align_ws(size_t x);

// Compute units of the current device.
int device_cus();

// ESPACE_PLAN_LOG=1 prints each product's plan to stderr (read once per process).
bool plan_log();

// An operand's addresses, for the check that no output overlaps it.
struct Range { const char* name; uintptr_t lo, hi; };
Range mat_range(const char* name, const void* p, int64_t rows, int64_t ld, espace_dtype dt);

espace_status check_dtype(espace_dtype dt);
espace_status check_mat(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, espace_dtype dt);
espace_status check_alias(const Range& out, const Range* ins, int n);
espace_status check_workspace(void* ws, size_t have, size_t need);
espace_status check_device();

// C[r][c] = Σ_k A[r][k]·B[c][k] under the library's plan for the sizes, with C in float32
// whatever the operands' type, ldc = splitk_ld(Cc) and C
// the library's own scratch: columns up to ldc may be written.  Needs no partial
// sums.  ranges > 1: the sums of up to so many depth ranges, *made of them, R·ldc apart
// in C, not combined.
espace_status run_tn_f32(const void* A, int64_t lda, const void* B, int64_t ldb, float* C, int64_t ldc, int64_t R,
                         int64_t Cc, int64_t D, espace_dtype dt, hipStream_t stream, int ranges = 1,
                         int* made = nullptr);
// float32 with an operand depth-major and the result scaled, where
// gemm_tn_f32_terms_supported().
espace_status run_tn_f32_depth(const float* A, int64_t lda, bool a_depth, const float* B, int64_t ldb, bool b_depth,
                               float* C, int64_t ldc, int64_t R, int64_t Cc, int64_t D, const float* scale, int ranges,
                               int* made, hipStream_t stream);
// Its plan for bfloat16: the cheapest of 256 x 256 and 256 x 192 tiles, priced as the
// other tiled products, and the small tiles; one or two rows may take the streaming
// kernel, matrices past the kernels' offsets one with 64-bit ones.
struct F32Plan {
    enum Kind { WIDE, GEMV, MID, TILED } kind = WIDE;
    int tile = -1;            // of kind TILED; the small tiles' configuration of kind MID
    int ranges = 1;
};
// depth: with B as [D][Cc] on the tiles, which are then faster (16384 deep, 4096 x 4096
// 390 us where the others' price is 419).  extra: us that the small tiles cost besides.
F32Plan f32_plan(int64_t R, int64_t Cc, int64_t D, int64_t lda, int64_t ldb, int ranges, bool depth = false,
                 double extra = 0);
// The float32 sums of plan.ranges depth ranges on the tiles of a plan of kind TILED, with
// B as [D][Cc]; *made of them, R·splitk_ld(Cc) apart.  count: the rows that there are
// of R (a device int; NULL: all).
espace_status run_tiled_ranges(const void* A, int64_t lda, const void* B, int64_t ldb, float* C, int64_t R, int64_t Cc,
                               int64_t D, int tile, int ranges, const int* count, int* made, hipStream_t stream);
// C = scale[0]·A·Bᵀ rounded to bfloat16, on the small tiles of such a plan in one range.
espace_status run_tn_scaled_mid(const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc,
                                int64_t R, int64_t Cc, int64_t D, int config, const float* scale, hipStream_t stream);
// A product of a loss (LossEpi) on a tile of kind TILED.
espace_status run_tn_loss(const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc, int64_t R,
                          int64_t Cc, int64_t D, int tile, LossMode mode, const LossEpi& epi, hipStream_t stream);

#define ESPACE_TRY(x)                       \
    do {                                    \
        espace_status _s = (x);             \
        if (_s != ESPACE_OK) return _s;     \
    } while (0)

}  // namespace api
}  // namespace espace
