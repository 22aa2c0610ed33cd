// Matrices with a side of at most 64, orthogonalised by one block each, all steps in one launch.  Part of scalecom.hip's single
// translation unit; the mathematics, the number formats and the scaling are those of orthogonalize_kernels.h.
//
// X lives in registers, in two halves, from the first to the last step: every wave holds blocks of 16 columns in the layout in which the
// matrix units leave a product (four consecutive rows of one column per lane).  That layout is at the same time an operand of B X
// whose inner dimension is permuted, and B's columns can be read in the same order, so X enters the product from where it
// is.  For S = X X^T every wave turns its own columns round through LDS, 32 at a time, and multiplies them with themselves: one
// set of fragments is both operands, and only the tiles on and above the diagonal are computed.  The waves' sums are then added up in order.
// Bound by one block's chain of steps (LDS, barriers, products in turn), whatever the number of matrices up to the number of CUs: the 22
// of a small residual network (up to 64 x 576, f32) take 53 us, 10 us a step; in tiles of 128 x 128, fifteen launches, they took 247.
#pragma once

#include <hip/hip_runtime.h>

#include "orthogonalize_kernels.h"

namespace {

constexpr int kSmallSide = 64, kSmallLong = 640;            // sides of the matrices that this path takes
constexpr int kSmallWaves = 8, kSmallThreads = kSmallWaves * kLanes;
constexpr int kSmallColumns = 16 * kSmallWaves;             // of a stage: one block of columns per wave
constexpr int kSmallBlocks = kSmallLong / kSmallColumns;    // of columns, per wave
constexpr int kSmallTiles = 10;                             // 16 x 16 tiles of S on and above the diagonal
constexpr int kSmallSlice = kSmallTiles * 1024;             // bytes per wave: 32 columns of X, both planes (8 KB), then its sums
constexpr int kSmallPlane = kSmallSide * kSmallSide * 2;    // of S or B

struct SmallMatrix {
    int64_t src, stride;
    int32_t rows, cols;
};
constexpr int kSmallMatrices = 150;                         // per launch: 3600 bytes of arguments
struct SmallTable {
    SmallMatrix m[kSmallMatrices];
};
struct SmallSteps {
    int n;
    int growth[SCALECOM_ORTHO_STEPS_MAX];
    float coeffs[3 * SCALECOM_ORTHO_STEPS_MAX];
};

__device__ __forceinline__ void split_four(float a, float b, float c, float d, half4_t& hi, half4_t& lo)
{
    const float v[4] = {a, b, c, d};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        _Float16 h, l;
        split_half(v[r], h, l);
        hi[r] = h;
        lo[r] = l;
    }
}

// Byte offset of element (row, col) in a plane of 64 columns: pieces as in orthogonalize_kernels.h.
__device__ __forceinline__ uint32_t small_offset(uint32_t row, uint32_t col) { return static_cast<uint32_t>(plane_offset(row, col, kSmallSide / kPieceCols)); }

// A slice's plane: 32 rows (columns of X) of 64: two pieces' upper halves.
__device__ __forceinline__ uint32_t slice_offset(uint32_t row, uint32_t col)
{
    return col / kPieceCols * (kPieceBytes / 2) + piece_chunk(row, col % kPieceCols / 8) + col % 8 * 2;
}

struct SmallShared {
    char slice[kSmallWaves][kSmallSlice];
    char s_plane[2][kSmallPlane];                           // E, the part of S off the diagonal
    char b_plane[2][kSmallPlane];                           // and B's
    float ds[kSmallSide], db[kSmallSide];
    double norms[kSmallWaves];
};

// RF: blocks of 16 rows that hold something (1, 2, or 4 for three as well).  (A block has read all of its matrix before it writes: `out`
// may be `update`.)
template <typename U, bool SPLIT, int RF>
__device__ __forceinline__ void small_matrix(const U* update, typename std::conditional<SPLIT, float, uint16_t>::type* out, const SmallMatrix t,
                                             const SmallSteps& steps, float eps, SmallShared& lds)
{
    constexpr int SIDE = RF > 2 ? 64 : 32, KF = SIDE / 32;  // of S, with zeros in the lower half for RF = 1
    constexpr int TILES = RF * (RF + 1) / 2;
    const bool tall = t.rows > t.cols;
    const int m = tall ? t.cols : t.rows, n = tall ? t.rows : t.cols;
    const int64_t row_step = tall ? 1 : t.stride, col_step = tall ? t.stride : 1;
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int g = lane / 16, c16 = lane % 16;
    const int turns = (n + kSmallColumns - 1) / kSmallColumns;
    // rows rf * 16 + g * 4 + r of column (turn * 8 + wave) * 16 + c16
    half4_t xh[kSmallBlocks][RF], xl[kSmallBlocks][RF];
    const int64_t first = t.src + (g * 4) * row_step + (wave * 16 + c16) * col_step;
    const auto inside = [&](int c, int rf, int r) { return rf * 16 + g * 4 + r < m && (c * kSmallWaves + wave) * 16 + c16 < n; };
    int lift;
    {
        float u[kSmallBlocks][RF][4];
        double sum = 0.0;
#pragma unroll
        for (int c = 0; c < kSmallBlocks; ++c)
#pragma unroll
            for (int rf = 0; rf < RF; ++rf)
#pragma unroll
                for (int r = 0; r < 4; ++r) {               // (what lies outside reads the matrix's first element and counts as zero)
                    const bool in = inside(c, rf, r);
                    const float v = widen(update[in ? first + (rf * 16 + r) * row_step + c * kSmallColumns * col_step : t.src]);
                    u[c][rf][r] = in ? v : 0.0f;
                }
#pragma unroll
        for (int c = 0; c < kSmallBlocks; ++c)
#pragma unroll
            for (int rf = 0; rf < RF; ++rf)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += static_cast<double>(u[c][rf][r]) * u[c][rf][r];
        for (int w = kLanes / 2; w > 0; w /= 2) sum += __shfl_xor(sum, w);
        if (lane == 0) lds.norms[wave] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < kSmallWaves; ++w) sum += lds.norms[w];
        const OrthoScale scale(sum, eps);
        lift = scale.lift;
#pragma unroll
        for (int c = 0; c < kSmallBlocks; ++c)
#pragma unroll
            for (int rf = 0; rf < RF; ++rf) split_four(static_cast<float>(u[c][rf][0] * scale.factor), static_cast<float>(u[c][rf][1] * scale.factor),
                                                       static_cast<float>(u[c][rf][2] * scale.factor), static_cast<float>(u[c][rf][3] * scale.factor),
                                                       xh[c][rf], xl[c][rf]);
    }
    char* slice = lds.slice[wave];
    const LanePlaces columns(0, lane);
    if (RF == 1)                                            // (what no tile covers)
        for (int e = threadIdx.x; e < 2 * kSmallPlane / 16; e += kSmallThreads) {
            reinterpret_cast<vf4_t*>(lds.s_plane[0])[e] = vf4_t{0.0f, 0.0f, 0.0f, 0.0f};
            reinterpret_cast<vf4_t*>(lds.b_plane[0])[e] = vf4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
#pragma unroll 1
    for (int step = 0; step < steps.n; ++step) {
        const float ca = steps.coeffs[3 * step], cb = steps.coeffs[3 * step + 1], cc = steps.coeffs[3 * step + 2];
        const int growth = steps.growth[step];
        // S = X X^T
        acc4_t s[TILES];
#pragma unroll
        for (int i = 0; i < TILES; ++i) s[i] = acc4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < kSmallBlocks; c += 2) {
            if (c >= turns) continue;                       // (uniform)
            // a row of the slice's planes is a column of X: 16 of one block of columns, 16 of the next
            const half4_t zero = {0, 0, 0, 0};
#pragma unroll
            for (int rf = 0; rf < RF; ++rf)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const bool there = c + half < kSmallBlocks;
                    const uint32_t at = slice_offset(half * 16 + c16, rf * 16 + g * 4);
                    *reinterpret_cast<half4_t*>(slice + at) = there ? xh[there ? c + half : 0][rf] : zero;
                    if (SPLIT) *reinterpret_cast<half4_t*>(slice + 4096 + at) = there ? xl[there ? c + half : 0][rf] : zero;
                }
            wave_lds_fence();
            half8_t h[RF], l[RF];
#pragma unroll
            for (int rf = 0; rf < RF; ++rf) {
                h[rf] = read_fragment<true>(slice, rf, columns);
                if (SPLIT) l[rf] = read_fragment<true>(slice + 4096, rf, columns);
            }
            const auto term = [&](const half8_t (&u)[RF], const half8_t (&v)[RF]) {
#pragma unroll
                for (int j = 0; j < RF; ++j)
#pragma unroll
                    for (int i = 0; i <= j; ++i) s[j * (j + 1) / 2 + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(u[i], v[j], s[j * (j + 1) / 2 + i], 0, 0, 0);
            };
            if (SPLIT) {
                term(l, h);
                term(h, l);
            }
            term(h, h);
            wave_lds_fence();
        }
        // the waves' sums put together, one lane's four of a tile per thread
#pragma unroll
        for (int i = 0; i < TILES; ++i) *reinterpret_cast<acc4_t*>(slice + (i * kLanes + lane) * sizeof(acc4_t)) = s[i];
        __syncthreads();
        for (int e = threadIdx.x; e < TILES * kLanes; e += kSmallThreads) {
            acc4_t v = *reinterpret_cast<const acc4_t*>(lds.slice[0] + e * sizeof(acc4_t));
#pragma unroll
            for (int w = 1; w < kSmallWaves; ++w) v += *reinterpret_cast<const acc4_t*>(lds.slice[w] + e * sizeof(acc4_t));
            const int tile = e / kLanes, tj = tile >= 6 ? 3 : tile >= 3 ? 2 : tile >= 1 ? 1 : 0, ti = tile - tj * (tj + 1) / 2;
            const int i = ti * 16 + g * 4, j = tj * 16 + c16;    // (e and the thread have the same lane)
            half4_t h, l;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float d = ldexpf(v[r] * (1.0f / (kXScale * kXScale)), -2 * lift);
                if (i + r == j) lds.ds[j] = d;
                _Float16 a, b;
                split_half(i + r == j ? 0.0f : d * kSScale, a, b);
                h[r] = a;
                l[r] = b;
            }
            *reinterpret_cast<half4_t*>(lds.s_plane[0] + small_offset(j, i)) = h;
            if (SPLIT) *reinterpret_cast<half4_t*>(lds.s_plane[1] + small_offset(j, i)) = l;
            if (ti == tj) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) {                   // the other side of the diagonal
                *reinterpret_cast<_Float16*>(lds.s_plane[0] + small_offset(i + r, j)) = h[r];
                if (SPLIT) *reinterpret_cast<_Float16*>(lds.s_plane[1] + small_offset(i + r, j)) = l[r];
            }
        }
        __syncthreads();
        // B = b S + c S S, one product of 16 x 16 per wave and turn
        constexpr int blocks = RF;
#pragma unroll
        for (int turn = 0; turn < (blocks * blocks + kSmallWaves - 1) / kSmallWaves; ++turn) {
            const int tile = turn * kSmallWaves + wave;
            if (tile >= blocks * blocks) continue;          // (uniform)
            const int i0 = tile / blocks * 16, j0 = tile % blocks * 16;
            acc4_t q = acc4_t{0.0f, 0.0f, 0.0f, 0.0f}, ql = q;
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                const uint32_t ai = small_offset(i0 + c16, k * 32 + g * 8), aj = small_offset(j0 + c16, k * 32 + g * 8);
                const half8_t a = *reinterpret_cast<const half8_t*>(lds.s_plane[0] + ai), b = *reinterpret_cast<const half8_t*>(lds.s_plane[0] + aj);
                if (SPLIT) {
                    const half8_t al = *reinterpret_cast<const half8_t*>(lds.s_plane[1] + ai), bl = *reinterpret_cast<const half8_t*>(lds.s_plane[1] + aj);
                    ql = __builtin_amdgcn_mfma_f32_16x16x32_f16(al, b, ql, 0, 0, 0);
                    ql = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, bl, ql, 0, 0, 0);
                }
                q = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, q, 0, 0, 0);
            }
            if (SPLIT) q += ql;
            const int i = i0 + g * 4, j = j0 + c16;
            const uint32_t at = small_offset(j, i);
            const half4_t eh = *reinterpret_cast<const half4_t*>(lds.s_plane[0] + at);
            half4_t el = {0, 0, 0, 0}, h, l;
            if (SPLIT) el = *reinterpret_cast<const half4_t*>(lds.s_plane[1] + at);
            const float dj = lds.ds[j];
            const acc4_t di = *reinterpret_cast<const acc4_t*>(lds.ds + i);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float e = (static_cast<float>(eh[r]) + static_cast<float>(el[r])) * (1.0f / kSScale), v = q[r] * (1.0f / (kSScale * kSScale));
                if (i + r == j) lds.db[j] = fmaf(cb, dj, cc * fmaf(dj, dj, v));
                const float off = fmaf(cb, e, cc * fmaf(di[r] + dj, e, v)) * kBScale;
                _Float16 a, b;
                split_half(i + r == j ? 0.0f : off, a, b);
                h[r] = a;
                l[r] = b;
            }
            *reinterpret_cast<half4_t*>(lds.b_plane[0] + at) = h;
            if (SPLIT) *reinterpret_cast<half4_t*>(lds.b_plane[1] + at) = l;
        }
        __syncthreads();
        const int less = max(lift - growth, 0) - lift;
        const float p_scale = ldexpf(1.0f / kBScale, less);
        // X <- a X + B X.  Of 32 rows of X a lane holds four of the upper 16 and four of the lower: B's columns in that order.
        half8_t bh[RF][KF], bl[RF][KF];
        acc4_t d[RF];
#pragma unroll
        for (int rf = 0; rf < RF; ++rf) {
            d[rf] = (*reinterpret_cast<const acc4_t*>(lds.db + rf * 16 + g * 4) + ca) * kBScale;
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                const uint32_t upper = small_offset(rf * 16 + c16, k * 32 + g * 4), lower = small_offset(rf * 16 + c16, k * 32 + 16 + g * 4);
                const auto both = [&](const char* plane) {
                    return __builtin_shufflevector(*reinterpret_cast<const half4_t*>(plane + upper), *reinterpret_cast<const half4_t*>(plane + lower), 0, 1, 2,
                                                   3, 4, 5, 6, 7);
                };
                bh[rf][k] = both(lds.b_plane[0]);
                if (SPLIT) bl[rf][k] = both(lds.b_plane[1]);
            }
        }
#pragma unroll
        for (int c = 0; c < kSmallBlocks; ++c) {
            if (c >= turns) continue;
            acc4_t p[RF];                                   // the product is added to a X
#pragma unroll
            for (int rf = 0; rf < RF; ++rf)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    p[rf][r] = fmaf(d[rf][r], static_cast<float>(xh[c][rf][r]), d[rf][r] * static_cast<float>(xl[c][rf][r]));
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                const half4_t zero = {0, 0, 0, 0};
                const bool two = 2 * k + 1 < RF;
                const half8_t h = __builtin_shufflevector(xh[c][2 * k], two ? xh[c][two ? 2 * k + 1 : 0] : zero, 0, 1, 2, 3, 4, 5, 6, 7);
                const half8_t l = __builtin_shufflevector(xl[c][2 * k], two ? xl[c][two ? 2 * k + 1 : 0] : zero, 0, 1, 2, 3, 4, 5, 6, 7);
                const auto term = [&](const half8_t (&u)[RF][KF], const half8_t& v) {
#pragma unroll
                    for (int rf = 0; rf < RF; ++rf) p[rf] = __builtin_amdgcn_mfma_f32_16x16x32_f16(u[rf][k], v, p[rf], 0, 0, 0);
                };
                if (SPLIT) {
                    term(bl, h);
                    term(bh, l);
                }
                term(bh, h);
            }
#pragma unroll
            for (int rf = 0; rf < RF; ++rf)
#pragma unroll
                for (int r = 0; r < 4; ++r) {               // (split_half of p * p_scale, without rounding that product)
                    xh[c][rf][r] = static_cast<_Float16>(p[rf][r] * p_scale);
                    xl[c][rf][r] = static_cast<_Float16>(fmaf(p[rf][r], p_scale, -static_cast<float>(xh[c][rf][r])));
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        lift += less;
    }
    const float back = ldexpf(1.0f / kXScale, -lift);
#pragma unroll
    for (int c = 0; c < kSmallBlocks; ++c) {
        if (c >= turns) continue;
#pragma unroll
        for (int rf = 0; rf < RF; ++rf)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (inside(c, rf, r))
                    put(out + first + (rf * 16 + r) * row_step + c * kSmallColumns * col_step,
                        (static_cast<float>(xh[c][rf][r]) + static_cast<float>(xl[c][rf][r])) * back);
    }
}

template <typename U, bool SPLIT>
__global__ void __launch_bounds__(kSmallThreads)
k_ortho_small(const U* update, typename std::conditional<SPLIT, float, uint16_t>::type* out, const SmallTable table, const SmallSteps steps, float eps)
{
    __shared__ __attribute__((aligned(1024))) SmallShared lds;
    const SmallMatrix t = table.m[blockIdx.x];
    const int m = min(t.rows, t.cols);
    if (m <= 16)
        small_matrix<U, SPLIT, 1>(update, out, t, steps, eps, lds);
    else if (m <= 32)
        small_matrix<U, SPLIT, 2>(update, out, t, steps, eps, lds);
    else
        small_matrix<U, SPLIT, 4>(update, out, t, steps, eps, lds);
}

}  // namespace
