// float32 "TN" product C[r][c] = sum_k A[r][k] * B[c][k] on the fp32 MFMA
// (the float32 layers and gradients, the calibration products), and the losses'
// products on the bfloat16 one (gemm_tn_f32_terms_kernel).
//
// fp32 MFMA issue 256 flops per clock and CU, twice the vector ALU's rate
// without packed instructions.  In both kernels on them the MFMA takes the B rows as
// its first operand, so a lane ends with runs of 4 consecutive output columns
// of one row, and the depth index of an operand is permuted the same way for
// both: a lane's 16-byte chunk holds 4 consecutive k, chunk q of a row goes
// to lane group q, and MFMA e of a slab takes element e of every chunk.  The
// sums of 32 (tiled) or 8 to 16 terms are formed apart and then added, so that
// a long sum rounds at its full size that many times less often.
#include <type_traits>

#include "common.hpp"
#include "kernels.hpp"

namespace espace {

namespace {

__device__ __forceinline__ f32x4_t load4_masked(const float* row, int k, int depth) {
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    const int nvalid = depth - k;
    if (nvalid >= 4) {
        v = *reinterpret_cast<const f32x4_t*>(row + k);
    } else if (nvalid > 0) {
        const f32x4_t t = *reinterpret_cast<const f32x4_t*>(row + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < nvalid ? t[e] : 0.f;
    }
    return v;
}

template <int MI> struct AccF;
template <> struct AccF<32> { typedef f32x16_t type; };
template <> struct AccF<16> { typedef f32x4_t type; };

__device__ __forceinline__ f32x16_t mfma_f32(float b, float a, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(b, a, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mfma_f32(float b, float a, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(b, a, c, 0, 0, 0);
}

// Four consecutive columns c .. c + 3 of output row `row`.
__device__ __forceinline__ void store4(float* row, int c, int Cc, f32x4_t v) {
    if (c + 4 <= Cc) {
        *reinterpret_cast<f32x4_t*>(row + c) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < Cc) row[c + e] = v[e];
    }
}

// Tiles of BM x BN outputs, four waves as 2 x 2, each a grid of 32 x 32 blocks
// of v_mfma_f32_32x32x2_f32.  Bound by the matrix cores: a 32-deep step of a
// 128 x 128 tile is 4096 cycles of MFMA per SIMD against 32 KB of operands, so
// two LDS stages of 128-byte rows, two workgroups per CU and one barrier per
// step suffice: 4096^3 in 1030 us, 133 TFLOP/s of the 157 the matrix cores
// issue (the vector-ALU kernel before it, 64 x 64 tiles: 1760 us; 1100 x 2048
// x 2048: 172 -> 103 us; 1024^3: 65 -> 24 us).  Chunk c of row r sits at chunk c ^ ((r >> 1) & 7): the 16 rows
// that 16 neighbouring lanes read fall on all 64 banks.
constexpr int TK = 32;                            // depth step: 128-byte rows

template <int BM, int BN>
__global__ __launch_bounds__(256, 2)
void gemm_tn_f32_mfma_kernel(const float* __restrict__ A, int64_t lda, const float* __restrict__ B, int64_t ldb,
                             float* __restrict__ C, int64_t ldc, int R, int Cc, int D, int tiles_c) {
    constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32;
    constexpr int STAGE = (BM + BN) * TK * 4;
    constexpr int LPW = (BM + BN) / 8 / 4;        // 1 KB loads (8 rows) per wave and stage
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE];
    int tile_r, tile_c;
    tile_coords<4>(blockIdx.x, gridDim.x, tiles_c, 0, tile_r, tile_c);
    const int row0 = tile_r * BM, col0 = tile_c * BN;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr0 = (wave >> 1) * WM, wc0 = (wave & 1) * WN;

    // descriptors over the tile's own rows (the launcher checks that these
    // span less than 2^32 bytes); rows past the matrix repeat its last row
    const int nr = min(BM, R - row0), nc = min(BN, Cc - col0);
    const auto ra = __builtin_amdgcn_make_buffer_rsrc((void*)(A + (int64_t)row0 * lda), (short)0,
                                                      (int)(uint32_t)((uint64_t)nr * lda * 4u), 0x00020000);
    const auto rb = __builtin_amdgcn_make_buffer_rsrc((void*)(B + (int64_t)col0 * ldb), (short)0,
                                                      (int)(uint32_t)((uint64_t)nc * ldb * 4u), 0x00020000);
    unsigned off[LPW];
    int kc[LPW];
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
        const int q = wave + 4 * j;
        const int rl = 8 * q + (lane >> 3);
        const bool isA = 8 * q < BM;
        const int rr = isA ? rl : rl - BM;
        kc[j] = ((lane & 7) ^ ((rr >> 1) & 7)) * 4;
        const int g = isA ? min(rr, nr - 1) : min(rr, nc - 1);
        off[j] = (unsigned)(((uint64_t)g * (isA ? lda : ldb) + kc[j]) * 4u);
    }
    auto issue = [&](int t) {
        unsigned char* stage = smem + (t & 1) * STAGE;
        const int k0 = t * TK;
#pragma unroll
        for (int j = 0; j < LPW; ++j) {
            const int q = wave + 4 * j;
            // chunks at or past the depth are read past the descriptor: zeros
            const unsigned o = k0 + kc[j] < D ? off[j] + (unsigned)k0 * 4u : 0xFFFFFFF0u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(8 * q < BM ? ra : rb,
                                                     (__attribute__((address_space(3))) void*)(stage + q * 1024), 16,
                                                     (int)o, 0, 0, 0);
        }
    };

    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const int lr = lane & 31, lh = lane >> 5, sw = (lr >> 1) & 7;
    const int steps = (D + TK - 1) / TK;
    issue(0);
    for (int t = 0; t < steps; ++t) {
        // this wave's loads of step t have landed, and after the barrier
        // every wave's; every wave is done reading the other stage
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (t + 1 < steps) issue(t + 1);
        const unsigned char* stage = smem + (t & 1) * STAGE;
        const unsigned char* pa = stage + (wr0 + lr) * (TK * 4);
        const unsigned char* pb = stage + (BM + wc0 + lr) * (TK * 4);
        const int left = D - t * TK;              // only the last step has fewer than TK
        f32x16_t part[TM][TN];
#pragma unroll
        for (int s = 0; s < TK / 8; ++s) {
            const int c = ((2 * s + lh) ^ sw) * 16;
            f32x4_t fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = *reinterpret_cast<const f32x4_t*>(pa + i * 32 * TK * 4 + c);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = *reinterpret_cast<const f32x4_t*>(pb + j * 32 * TK * 4 + c);
            if (left < TK) {
                // the chunk that straddles the depth: its padding is not used
                const int nv = left - 8 * s - 4 * lh;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
#pragma unroll
                    for (int i = 0; i < TM; ++i) fa[i][e] = e < nv ? fa[i][e] : 0.f;
#pragma unroll
                    for (int j = 0; j < TN; ++j) fb[j][e] = e < nv ? fb[j][e] : 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        part[i][j] = mfma_f32(fb[j][e], fa[i][e], s == 0 && e == 0 ? f32x16_t{} : part[i][j]);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] += part[i][j];
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int r = row0 + wr0 + 32 * i + lr;
        if (r >= R) continue;
        float* row = C + (int64_t)r * ldc;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                store4(row, col0 + wc0 + 32 * j + 8 * q + 4 * lh, Cc,
                       f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]});
    }
}

// x as the sum of three bfloat16 (Henry, Tang and Heinecke, "Leveraging the bfloat16
// artificial intelligence datatype for higher-precision computations", ARITH 2019): each
// rounds what the ones before it leave, whose differences float32 holds exactly.  8 values
// to three 16-byte chunks.
__device__ __forceinline__ void split3(f32x4_t lo, f32x4_t hi, u32x4_t (&t)[3]) {
    float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
    for (int s = 0; s < 3; ++s)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            t[s][q] = pack_bf16x2(x[2 * q], x[2 * q + 1]);
            x[2 * q] -= __uint_as_float(t[s][q] << 16);
            x[2 * q + 1] -= __uint_as_float(t[s][q] & 0xffff0000u);
        }
}

// The same product on the bfloat16 matrix cores (the losses' products): with a = a0 + a1 +
// a2 and b likewise, a0 b0 + a0 b1 + a1 b0 + a1 b1 + a0 b2 + a2 b0 leaves out a1 b2 + a2 b1
// + a2 b2, at most 2^-23 of |a b| (each term at most 2^-8 of the one before it), as two
// roundings of float32; the sums are float32.  601 x 1000 x 5003 tokens, features and
// vocabulary: error of the losses and gradients 4.9e-7, with the fp32 MFMA 1.7e-6, of
// which a sum takes 8 times as many.  (An infinity is not the sum of its terms: NaN.)
//
// Six products of 16 times the fp32 MFMA's rate: 2.7 times its peak; a step of a 128 x 128
// tile is 1536 cycles of MFMA per SIMD.  Each element is split once, by the thread that
// loads it (some 110 vector instructions a step and wave), and lies in LDS as three planes
// of 64-byte rows.  The splits stand between the MFMA (mix()), the loads run two steps
// ahead, and 8 waves give each SIMD two: 601 x 1000 x 5003 on 128 x 128 tiles with 4 waves
// and the loads one step ahead 66 us, scheduled 56, 8 waves 51, all of the split between
// the MFMA 44 (fp32 MFMA: 65); 1024 x 1024 x 8192 108 -> 91.  Bound by the issue of vector
// instructions and MFMA, 44% of the matrix cores' cycles; a third LDS stage, which takes
// the wait after the barrier away, 45 us.
//
// AD, BD: the operand lies depth-major, [D][rows]: a thread's 8 elements are of as many
// lines, which the lanes of a wave read along.  dX = G W and dW = G' X take W and G so,
// without a pass that transposes either, and the result times `scale`: a step of 601 x
// 1000 x 5003 228 -> 207 us, 100 x 2000 x 16000 357 -> 260.
template <int BM, int BN, int WR, int WC, bool AD, bool BD>
__global__ __launch_bounds__(64 * WR * WC, 2)
void gemm_tn_f32_terms_kernel(const float* __restrict__ A, int64_t lda, const float* __restrict__ B, int64_t ldb,
                              float* __restrict__ C, int64_t ldc, int R, int Cc, int D, int tiles_c, int per_range,
                              int64_t stride, const float* __restrict__ scale) {
    constexpr int WM = BM / WR, WN = BN / WC, TM = WM / 32, TN = WN / 32;
    constexpr int PLANE = (BM + BN) * TK * 2, STAGE = 3 * PLANE;
    constexpr int ROWS = 16 * WR * WC;            // rows that the threads' pieces of 8 elements are of
    constexpr int NP = (BM + BN) / ROWS;          // pieces a thread and step
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE];
    // depth range blockIdx.y: per_range elements, a multiple of 2 TK; its sums `stride` on
    const int first = blockIdx.y * per_range;
    A += first * (AD ? lda : 1);
    B += first * (BD ? ldb : 1);
    C += blockIdx.y * stride;
    D = min(D - first, per_range);
    int tile_r, tile_c;
    tile_coords<4>(blockIdx.x, gridDim.x, tiles_c, 0, tile_r, tile_c);
    const int row0 = tile_r * BM, col0 = tile_c * BN;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr0 = wave / WC * WM, wc0 = wave % WC * WN;

    // descriptors over the tile's own rows, from this range's first element on (the
    // launcher checks that these span less than 2^32 bytes); rows past the matrix repeat
    // its last row
    const int nr = min(BM, R - row0), nc = min(BN, Cc - col0);
    auto rsrc = [&](bool depth, const float* M, int64_t ld, int r0, int n) {
        const uint64_t elems = depth ? (uint64_t)(D - 1) * ld + n : (uint64_t)n * ld - first;
        return __builtin_amdgcn_make_buffer_rsrc((void*)(M + (depth ? r0 : r0 * ld)), (short)0,
                                                 (int)(uint32_t)(elems * 4u), 0x00020000);
    };
    const auto ra = rsrc(AD, A, lda, row0, nr), rb = rsrc(BD, B, ldb, col0, nc);
    // piece j: 8 elements of row ROWS j + threadIdx.x / 4, or threadIdx.x % ROWS where the
    // operand is depth-major; chunk c of row r sits at chunk c ^ ((r >> 2) & 3): the 16 rows
    // of 64 bytes that neighbouring lanes read fall on all banks
    auto row_of = [&](bool depth) { return depth ? (int)threadIdx.x % ROWS : (int)threadIdx.x >> 2; };
    auto chunk_of = [&](bool depth) { return depth ? wave * 64 / ROWS : (int)threadIdx.x & 3; };
    unsigned off[NP];
    int put[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const bool isA = ROWS * j < BM, dm = isA ? AD : BD;
        const int64_t ld = isA ? lda : ldb;
        const int rr = ROWS * j + row_of(dm), k = chunk_of(dm) * 8;
        const int g = isA ? min(rr, nr - 1) : min(rr - BM, nc - 1);
        off[j] = (unsigned)((uint64_t)(dm ? k * ld + g : g * ld + k) * 4u);
        put[j] = rr * (TK * 2) + ((chunk_of(dm) ^ ((rr >> 2) & 3)) * 16);
    }
    // the elements of two steps in flight
    f32x4_t x[2][NP][2];
    auto load = [&](int t, int j) {
        const bool isA = ROWS * j < BM;
        if (isA ? AD : BD) {
            // lines past the depth are past the descriptor: zeros (the launcher checks that
            // those that are read ahead span less than 2^32 bytes, too)
            const unsigned line = (unsigned)(isA ? lda : ldb) * 4u;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[t & 1][j][e / 4][e % 4] = __builtin_bit_cast(
                    float, __builtin_amdgcn_raw_buffer_load_b32(isA ? ra : rb, (int)(off[j] + (t * TK + e) * line), 0, 0));
            return;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // chunks at or past the depth are read past the descriptor: zeros
            const int k = t * TK + chunk_of(false) * 8 + 4 * h;
            const unsigned o = k < D ? off[j] + (unsigned)(t * TK + 4 * h) * 4u : 0xFFFFFFF0u;
            x[t & 1][j][h] =
                __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(isA ? ra : rb, (int)o, 0, 0));
        }
    };
    // the chunk that straddles the depth: its padding is not used
    auto mask = [&](int t) {
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            if (ROWS * j < BM ? AD : BD) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[t & 1][j][h][e] = t * TK + chunk_of(false) * 8 + 4 * h + e < D ? x[t & 1][j][h][e] : 0.f;
        }
    };
    auto stage_in = [&](int t, int j) {
        u32x4_t v[3];
        split3(x[t & 1][j][0], x[t & 1][j][1], v);
#pragma unroll
        for (int p = 0; p < 3; ++p)
            *reinterpret_cast<u32x4_t*>(smem + (t & 1) * STAGE + p * PLANE + put[j]) = v[p];
    };

    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const int lr = lane & 31, lh = lane >> 5, sw = (lr >> 2) & 3;
    const int steps = (D + TK - 1) / TK;
    bf16x8_t fa[2][TM][3], fb[2][TN][3];
    auto read = [&](int t, int u) {
        const unsigned char* pa = smem + (t & 1) * STAGE + (wr0 + lr) * (TK * 2);
        const unsigned char* pb = smem + (t & 1) * STAGE + (BM + wc0 + lr) * (TK * 2);
        const int c = ((2 * u + lh) ^ sw) * 16;
#pragma unroll
        for (const int p : {1, 0, 2}) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
                fa[u][i][p] = *reinterpret_cast<const bf16x8_t*>(pa + p * PLANE + i * 32 * TK * 2 + c);
#pragma unroll
            for (int j = 0; j < TN; ++j)
                fb[u][j][p] = *reinterpret_cast<const bf16x8_t*>(pb + p * PLANE + j * 32 * TK * 2 + c);
        }
    };
    auto multiply = [&](int u) {
        // in the order in which the terms are read
        constexpr int ta[6] = {1, 1, 0, 0, 2, 0}, tb[6] = {1, 0, 1, 0, 0, 2};
#pragma unroll
        for (int q = 0; q < 6; ++q)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[u][j][tb[q]], fa[u][i][ta[q]], acc[i][j], 0,
                                                                        0, 0);
    };
#pragma unroll
    for (int j = 0; j < NP; ++j) load(0, j);
#pragma unroll
    for (int j = 0; j < NP; ++j) load(1, j);
    if (TK > D) mask(0);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        stage_in(0, j);
        load(2, j);
    }
    constexpr int HALF = NP / 2;
    // a slab's MFMA between the split of the half of a later step, and its reads
    auto mix = [&]() {
#pragma unroll
        for (int q = 0; q < 6 * TM * TN; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                    // MFMA
            __builtin_amdgcn_sched_group_barrier(0x002, 54 * (NP - HALF) / (6 * TM * TN) + 1, 0);    // VALU
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                    // LDS reads
            __builtin_amdgcn_sched_group_barrier(0x220, 1, 0);                    // LDS writes, loads
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // step t, whose parity the caller knows
    auto step = [&](int t) {
        if ((t + 2) * TK > D) mask(t + 1);
        // every wave has written its part of step t and is done reading the other stage
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        read(t, 0);
        __builtin_amdgcn_sched_barrier(0);
        multiply(0);
        read(t, 1);
#pragma unroll
        for (int j = 0; j < HALF; ++j) {
            stage_in(t + 1, j);
            load(t + 3, j);
        }
        mix();
        multiply(1);
#pragma unroll
        for (int j = HALF; j < NP; ++j) {
            stage_in(t + 1, j);
            load(t + 3, j);
        }
        mix();
        // (the loads stay where they are)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // pairs of steps: past the depth they add zeros
    for (int t = 0; t < steps; t += 2) {
        step(t);
        step(t + 1);
    }
    const float a = scale ? scale[0] : 1.f;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int r = row0 + wr0 + 32 * i + lr;
        if (r >= R) continue;
        float* row = C + (int64_t)r * ldc;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                store4(row, col0 + wc0 + 32 * j + 8 * q + 4 * lh, Cc,
                       f32x4_t{a * acc[i][j][4 * q], a * acc[i][j][4 * q + 1], a * acc[i][j][4 * q + 2],
                               a * acc[i][j][4 * q + 3]});
    }
}

// Products too small to fill the chip with tiles: one MI x MI block of the
// output per workgroup, its W waves taking turns at the depth (UD consecutive
// slabs of 256 / MI each, loaded straight to registers), the partial sums
// added in wave order through LDS.  Bound by latency, or by the stream of the
// many-row operand for a few tokens: with the depth one serial chain per tile
// the 128 x 64 x 256 projection took 17 us and 16 x 4096 x 2048 130 us, now
// below 10 us with the launch.
template <int MI, int W, int UD>
__global__ __launch_bounds__(W * 64)
void gemm_tn_f32_split_kernel(const float* __restrict__ A, int64_t lda, const float* __restrict__ B, int64_t ldb,
                              float* __restrict__ C, int64_t ldc, int R, int Cc, int D, int tiles_c) {
    using Acc = typename AccF<MI>::type;
    constexpr int SD = 256 / MI;                  // depth of a slab: one 16-byte chunk per lane
    constexpr int NQ = MI * MI / 256;             // 4-column runs per lane
    __shared__ f32x4_t red[W][NQ][64];
    int tile_r, tile_c;
    tile_coords<4>(blockIdx.x, gridDim.x, tiles_c, 0, tile_r, tile_c);
    const int row0 = tile_r * MI, col0 = tile_c * MI;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane % MI, lk = lane / MI * 4;
    const float* arow = A + (int64_t)min(row0 + lr, R - 1) * lda;
    const float* brow = B + (int64_t)min(col0 + lr, Cc - 1) * ldb;
    Acc acc;
#pragma unroll
    for (int e = 0; e < 4 * NQ; ++e) acc[e] = 0.f;
    for (int k0 = wave * UD * SD; k0 < D; k0 += W * UD * SD) {
        f32x4_t fa[UD], fb[UD];
        if (k0 + UD * SD <= D) {
#pragma unroll
            for (int u = 0; u < UD; ++u) {
                fb[u] = *reinterpret_cast<const f32x4_t*>(brow + k0 + u * SD + lk);
                fa[u] = *reinterpret_cast<const f32x4_t*>(arow + k0 + u * SD + lk);
            }
        } else {
#pragma unroll
            for (int u = 0; u < UD; ++u) {
                fb[u] = load4_masked(brow, k0 + u * SD + lk, D);
                fa[u] = load4_masked(arow, k0 + u * SD + lk, D);
            }
        }
#pragma unroll
        for (int u = 0; u < UD; ++u) {
            Acc part = {};
#pragma unroll
            for (int e = 0; e < 4; ++e) part = mfma_f32(fb[u][e], fa[u][e], part);
            acc += part;
        }
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) red[wave][q][lane] = f32x4_t{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    if (wave >= NQ) return;
    f32x4_t v = red[0][wave][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) v += red[w][wave][lane];
    const int r = row0 + lr;
    if (r < R) store4(C + (int64_t)r * ldc, col0 + 8 * wave + lk, Cc, v);
}

}  // namespace


hipError_t launch_gemm_tn_f32(const float* A, int64_t lda, const float* B, int64_t ldb,
                              float* C, int64_t ldc, int R, int Cc, int D, int cus, hipStream_t stream) {
    auto tiles = [&](int t) { return (int64_t)((R + t - 1) / t) * ((Cc + t - 1) / t); };
    // the tiled kernels' 32-bit offsets inside a tile
    const bool fits = (lda > ldb ? lda : ldb) * 128 * 4 < ((int64_t)1 << 32);
    const int few = R < Cc ? R : Cc;
    auto tiled = [&](auto kernel, int t) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)tiles(t)), dim3(256), 0, stream, A, lda, B, ldb, C, ldc, R, Cc, D,
                           (Cc + t - 1) / t);
        return hipGetLastError();
    };
    // one launch unless its 512-thread workgroups were 2^32 threads, a launch's limit
    auto split = [&](auto kernel, int t) {
        const int64_t most = 1 << 22;
        const int64_t tc = (Cc + t - 1) / t < most ? (Cc + t - 1) / t : most;
        const int64_t cols = tc * t, rows = most / tc * t;
        for (int64_t r = 0; r < R; r += rows)
            for (int64_t c = 0; c < Cc; c += cols) {
                const int nr = (int)(R - r < rows ? R - r : rows), nc = (int)(Cc - c < cols ? Cc - c : cols);
                hipLaunchKernelGGL(kernel, dim3((unsigned)(((nr + t - 1) / t) * ((nc + t - 1) / t))), dim3(512), 0,
                                   stream, A + r * lda, lda, B + c * ldb, ldb, C + r * ldc + c, ldc, nr, nc, D,
                                   (nc + t - 1) / t);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
        return hipSuccess;
    };
    // Few rows or columns first: a tile's unused half or more costs as much as the
    // used one.  Up to 16 of them, 16 x 16 blocks whose waves split the depth (1 x 32768
    // x 1024 28 us, 64 x 64 tiles 41, 128 x 128 ones 74; 100000 x 8 x 512 45, 66 and 140); up
    // to 32, 32 x 32 ones (17 x 65536 x 1024 68, 75 and 135), but at shallow depths 64 x
    // 64 tiles once they are enough (24 x 65536 x 256 22 against 26, 30000 x 32 x 64 5.8
    // against 7.0; 32 x 16384 x 256 9.2 against 8.4).
    if (few <= 16) return split(gemm_tn_f32_split_kernel<16, 8, 4>, 16);
    const bool shallow = D <= 256 && tiles(64) * 128 >= (int64_t)cus * D;
    if (few <= 32 && tiles(32) >= 5 * (int64_t)cus / 8 && !(fits && shallow))
        return split(gemm_tn_f32_split_kernel<32, 8, 4>, 32);
    // 128 x 128 tiles once there is one for every CU (4096^3, 1024 tiles:
    // 1030 against 1079 us with 64 x 64 tiles; 2048 x 2048 x 8192, 256: 542
    // against 549; 1100 x 2048 x 2048, 153: 132 against 103); 64 x 64 tiles
    // from half as many as CUs (1000 x 600 x 1500, 160 tiles: 33 against 36
    // us with 32 x 32 blocks; 200 x 1024 x 1024, 64: 23 against 11).  Below
    // that the depth is split over a workgroup's waves: 32 x 32 blocks from
    // 5/8 as many as CUs (200 x 1024 x 1024, 224 blocks: 11 against 17 us
    // with 16 x 16 ones; 200 x 300 x 2000, 70: 16 against 9.5), 16 x 16
    // blocks below.
    if (fits && few > 64 && tiles(128) >= cus) return tiled(gemm_tn_f32_mfma_kernel<128, 128>, 128);
    if (fits && tiles(64) >= cus / 2) return tiled(gemm_tn_f32_mfma_kernel<64, 64>, 64);
    if (tiles(32) >= 5 * (int64_t)cus / 8) return split(gemm_tn_f32_split_kernel<32, 8, 4>, 32);
    return split(gemm_tn_f32_split_kernel<16, 8, 4>, 16);
}

// Tiles of 128 or 64 on the bfloat16 matrix cores, and depth ranges, by their estimated
// time: the tiles of the fullest CU at the rates that the two reach (215 and 150
// TFLOP/s), a launch and its ramp 8 us, and the sums written and read again.  dX of N x K
// x V on one range -> on the cheapest, us: 601 x 1000 x 5003 104 -> 47 (with the sums' pass
// 52), 275 x 256 x 15712 291 -> 32, 100 x 2000 x 16000 298 -> 52.
bool gemm_tn_f32_terms_supported(int64_t R, int64_t Cc, int64_t D, int64_t lda, int64_t ldb, bool a_depth,
                                 bool b_depth) {
    // 32-bit byte offsets inside a tile, of the steps that are read ahead of the depth too.
    // Few rows leave most of a tile empty, but a depth-major B would have to be transposed
    // first (dX of 16 x 2000 x 16000: the step 240 -> 167 us, 32 x 700 x 9000 87 -> 69, 28 x
    // 432 x 3200 level).
    auto fits = [&](int64_t ld, bool depth) { return (depth ? D + 8 * TK : 128) * ld * 4 < ((int64_t)1 << 32); };
    return (R > 32 || b_depth) && Cc > 32 && fits(lda, a_depth) && fits(ldb, b_depth);
}

hipError_t launch_gemm_tn_f32_ranges(const float* A, int64_t lda, const float* B, int64_t ldb, float* C, int64_t ldc,
                                     int R, int Cc, int D, int cus, int ranges, int* made, bool a_depth, bool b_depth,
                                     const float* scale, hipStream_t stream) {
    *made = 1;
    if (!gemm_tn_f32_terms_supported(R, Cc, D, lda, ldb, a_depth, b_depth)) {
        if (a_depth || b_depth || scale) return hipErrorInvalidValue;
        return launch_gemm_tn_f32(A, lda, B, ldb, C, ldc, R, Cc, D, cus, stream);
    }
    double best = 1e300;
    int tile = 64;
    for (const int t : {64, 128}) {
        const int64_t tiles = (int64_t)((R + t - 1) / t) * ((Cc + t - 1) / t);
        for (int s = 1; s <= ranges && (s == 1 || D / s >= 128); ++s) {
            const int64_t rounds = (tiles * s + cus - 1) / cus;
            const double us = rounds * (2.0 * t * t * D / s) / ((t == 64 ? 150e6 : 215e6) / 256) + 8.0 +
                              (s > 1 ? 2.0 * s * R * (double)Cc * 4 / 4e6 : 0.0);
            if (us < best) {
                best = us;
                tile = t;
                *made = s;
            }
        }
    }
    const int per = ((D + *made - 1) / *made + 2 * TK - 1) / (2 * TK) * (2 * TK);
    *made = (D + per - 1) / per;
    const int64_t tr = (R + tile - 1) / tile, tc = (Cc + tile - 1) / tile;
    const dim3 grid((unsigned)(tr * tc), (unsigned)*made);
    auto run = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, A, lda, B, ldb, C, ldc, R, Cc, D, (int)tc, per,
                           (int64_t)R * ldc, scale);
        return hipGetLastError();
    };
    auto order = [&](auto ad, auto bd) {
        constexpr bool AD = decltype(ad)::value, BD = decltype(bd)::value;
        return tile == 128 ? run(gemm_tn_f32_terms_kernel<128, 128, 2, 4, AD, BD>, 512)
                           : run(gemm_tn_f32_terms_kernel<64, 64, 2, 2, AD, BD>, 256);
    };
    using No = std::false_type;
    using Yes = std::true_type;
    if (a_depth) return b_depth ? hipErrorInvalidValue : order(Yes{}, No{});
    return b_depth ? order(No{}, Yes{}) : order(No{}, No{});
}

}  // namespace espace
