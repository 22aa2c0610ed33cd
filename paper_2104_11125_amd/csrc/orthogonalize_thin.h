// Long matrices with a side of at most 16, orthogonalised by way of their Gram matrix in binary64.  Part of scalecom.hip's single
// translation unit.
//
// Every step multiplies X by a polynomial in G = X X^T from the left, so O = Q U with a product Q of polynomials in the first
// G, of 16 x 16 at most: one pass over U for G (whose trace is |U|^2), the steps on G and Q alone, one pass for O.  Q's
// elements reach the product of the steps' a (485 for the usual five) where X has hardly any extent, and an error in them meets X's
// largest values: binary64 has bits to spare for that, 16-bit halves have not, which is why larger matrices do not go this way.
// G is carried on as P G P, and what its roundings leave where X has no extent, 2^-53 of its largest value and of either sign, grows by the
// square of what X may grow by.  Where an eigenvalue came to be clearly negative in this way, a + b g + c g^2 would grow with it without
// bound (16 steps of 4.0848, -6.8946, 2.9270 on a 16 x 1000 of rank 3: a singular value of 52 087, 1.2 in truth).  So before X may have grown by
// more than 2^kThinGrowthBits since G was formed, G is formed anew from X = Q U, one pass over U, and has no negative eigenvalues beyond 2^-53 again.
// Bound by three launches and the steps' chain: 1 x 1000, 7 x 1000 and 1 x 70001, f32 to bfloat16, take 10 + 13 + 10 us (a call of
// eight steps, f32, 33; of nine, with a second G, 53); 1 x 70001 as a matrix padded to 128 rows took 55 us a step.
#pragma once

#include <hip/hip_runtime.h>

#include "orthogonalize_small.h"

namespace {

constexpr int kThinSide = 16;
constexpr int kThinColumns = 512;                           // of X, per block of the two passes
constexpr int kThinGram = kThinSide * kThinSide;            // doubles
static_assert(kThinGram == kBlock, "one element per thread");
constexpr int kThinGrowthBits = 16;                         // 2^-53 of G becomes 2^-19 at most (a step's bits are rounded); eight steps with the usual coefficients
static_assert(kThinGrowthBits >= 6, "a step's growth is 32 at most, which with the rounding is six bits: every run has a step at least");

struct ThinMatrix {
    int64_t src, stride;
    int32_t rows, cols;
    uint32_t block_first, blocks;                           // of the two passes
};
constexpr int kThinMatrices = 90;                           // per launch: 3240 bytes of arguments
struct ThinTable {
    uint32_t first[kThinMatrices];                          // block
    ThinMatrix m[kThinMatrices];
};

struct ThinPlace {                                          // rows of X: the short side
    int m, n;
    int64_t row_step, col_step;
    __device__ __forceinline__ explicit ThinPlace(const ThinMatrix& t)
    {
        const bool tall = t.rows > t.cols;
        m = tall ? t.cols : t.rows;
        n = tall ? t.rows : t.cols;
        row_step = tall ? 1 : t.stride;
        col_step = tall ? t.stride : 1;
    }
};

// A thread's column of a thin matrix, in binary64.
template <typename U>
__device__ __forceinline__ void thin_column(const U* update, const ThinMatrix& t, const ThinPlace& o, int64_t col, double (&u)[kThinSide])
{
#pragma unroll
    for (int k = 0; k < kThinSide; ++k) u[k] = k < o.m ? widen(update[t.src + k * o.row_step + col * o.col_step]) : 0.0;
}

// Row i of Q times that column.
__device__ __forceinline__ double thin_row(const double (&q)[kThinSide][kThinSide], int i, int m, const double (&u)[kThinSide])
{
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kThinSide; ++k)
        if (k < m) sum = fma(q[i][k], u[k], sum);
    return sum;
}

// A block's share of X X^T, of 512 columns: of X = U or, AGAIN, of X = Q U, whose values are binary64 and go through LDS 256 columns at a time.
template <typename U, bool AGAIN>
__global__ void __launch_bounds__(kBlock)
k_thin_gram(const U* __restrict__ update, int n_matrices, int first, const ThinTable table, const double* __restrict__ q, double* __restrict__ partial)
{
    constexpr int kColumns = AGAIN ? kBlock : kThinColumns;
    __shared__ typename std::conditional<AGAIN, double, float>::type lds[kThinSide][kColumns + 1];
    __shared__ double of_q[kThinSide][kThinSide];
    const int at = find_block(table.first, n_matrices, blockIdx.x);
    const ThinMatrix t = table.m[at];
    const uint32_t part = blockIdx.x - table.first[at], block = t.block_first + part;
    const ThinPlace o(t);
    if (AGAIN) of_q[threadIdx.x / kThinSide][threadIdx.x % kThinSide] = q[static_cast<size_t>(first + at) * kThinGram + threadIdx.x];
    // a thread takes one element (i, j) over its group's share of the columns
    __shared__ double sums[kBlock];
    const int pairs = o.m * o.m, groups = kBlock / pairs, pair = threadIdx.x % pairs, group = threadIdx.x / pairs;
    const int i = pair / o.m, j = pair % o.m;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
    for (int turn = 0; turn < kThinColumns / kColumns; ++turn) {
        const int64_t c0 = static_cast<int64_t>(part) * kThinColumns + turn * kColumns;
        const int columns = static_cast<int>(min(static_cast<int64_t>(kColumns), o.n - c0));   // (of the last part's second half: less than none)
        if (AGAIN) {
            __syncthreads();                                // Q is there, the columns before are done with
            if (static_cast<int>(threadIdx.x) < columns) {
                double u[kThinSide];
                thin_column(update, t, o, c0 + threadIdx.x, u);
                for (int row = 0; row < o.m; ++row) lds[row][threadIdx.x] = thin_row(of_q, row, o.m, u);
            }
        } else {
            for (int e = threadIdx.x; e < o.m * kColumns; e += kBlock) {
                // consecutive threads along the caller's rows
                const int row = o.col_step == 1 ? e / kColumns : e % o.m, col = o.col_step == 1 ? e % kColumns : e / o.m;
                lds[row][col] = col < columns ? widen(update[t.src + row * o.row_step + (c0 + col) * o.col_step]) : 0.0f;
            }
        }
        __syncthreads();
        if (group < groups) {
            int c = group;
            for (; c + 3 * groups < columns; c += 4 * groups)
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] = fma(static_cast<double>(lds[i][c + k * groups]), static_cast<double>(lds[j][c + k * groups]), s[k]);
            for (; c < columns; c += groups) s[0] = fma(static_cast<double>(lds[i][c]), static_cast<double>(lds[j][c]), s[0]);
        }
    }
    sums[threadIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    double sum = 0.0;
    const int row = threadIdx.x / kThinSide, col = threadIdx.x % kThinSide;
    if (row < o.m && col < o.m)
        for (int k = 0; k < groups; ++k) sum += sums[k * pairs + row * o.m + col];
    partial[static_cast<size_t>(block) * kThinGram + threadIdx.x] = sum;
}

// G from its shares, and Q through the steps [begin, end): one block per matrix, four threads per element for the sum.  q[matrix]:
// Q / (|U| + eps), row by row; read where these are not the first steps (G is that of X already then).
constexpr int kThinSums = 4;
__global__ void __launch_bounds__(kThinSums * kThinGram)
k_thin_steps(const double* __restrict__ partial, int first, const ThinTable table, const SmallSteps steps, int begin, int end, float eps, double* __restrict__ q)
{
    __shared__ double g[kThinSide][kThinSide + 1], p[kThinSide][kThinSide + 1], w[kThinSide][kThinSide + 1], sums[kThinSums][kThinGram];
    const ThinMatrix t = table.m[blockIdx.x];
    const int m = min(t.rows, t.cols);
    const int element = threadIdx.x % kThinGram, turn = threadIdx.x / kThinGram;
    const int i = element / kThinSide, j = element % kThinSide;
    const double* from = partial + static_cast<size_t>(t.block_first) * kThinGram + element;
    double s[8] = {};
    uint32_t b = turn;
    for (; b + 7 * kThinSums < t.blocks; b += 8 * kThinSums)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += from[static_cast<size_t>(b + k * kThinSums) * kThinGram];
    for (; b < t.blocks; b += kThinSums) s[0] += from[static_cast<size_t>(b) * kThinGram];
    sums[turn][element] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    __syncthreads();
    // the first 256 threads go on; the others only come to the barriers
    const bool mine_too = turn == 0;                        // (whole waves)
    if (mine_too) g[i][j] = (sums[0][element] + sums[1][element]) + (sums[2][element] + sums[3][element]);
    __syncthreads();
    double mine = 0.0;                                      // Q
    double* const to = q + static_cast<size_t>(first + blockIdx.x) * kThinGram + element;
    if (begin == 0) {
        double trace = 0.0;
        for (int k = 0; k < m; ++k) trace += g[k][k];
        const double inv = 1.0 / (sqrt(trace) + static_cast<double>(eps));
        __syncthreads();
        if (mine_too) g[i][j] *= inv * inv;
        mine = i == j ? inv : 0.0;
    } else if (mine_too) {
        mine = *to;
    }
    __syncthreads();
    const auto product = [&](const double (&u)[kThinSide][kThinSide + 1], const double (&v)[kThinSide][kThinSide + 1]) {
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < kThinSide; ++k) sum = fma(u[i][k], v[k][j], sum);
        return sum;
    };
    for (int step = begin; step < end; ++step) {
        const double a = steps.coeffs[3 * step], c1 = steps.coeffs[3 * step + 1], c2 = steps.coeffs[3 * step + 2];
        if (mine_too) {
            const double square = product(g, g);
            p[i][j] = (i == j ? a : 0.0) + c1 * g[i][j] + c2 * square;   // a I + b G + c G G
            w[i][j] = mine;
        }
        __syncthreads();
        double pg = 0.0;
        if (mine_too) {
            mine = product(p, w);                           // Q <- P Q
            pg = product(p, g);
        }
        __syncthreads();
        if (mine_too) w[i][j] = pg;
        __syncthreads();
        if (mine_too) g[i][j] = product(w, p);              // G <- P G P (they commute)
        __syncthreads();
    }
    if (mine_too) *to = mine;
}

// O = Q U: a column per thread and turn.
template <typename U, typename Out>
__global__ void __launch_bounds__(kBlock)
k_thin_apply(const U* update, int n_matrices, int first, const ThinTable table, const double* __restrict__ q, Out* out)
{
    __shared__ double lds[kThinSide][kThinSide];
    const int at = find_block(table.first, n_matrices, blockIdx.x);
    const ThinMatrix t = table.m[at];
    const ThinPlace o(t);
    lds[threadIdx.x / kThinSide][threadIdx.x % kThinSide] = q[static_cast<size_t>(first + at) * kThinGram + threadIdx.x];
    __syncthreads();
    const int64_t c0 = static_cast<int64_t>(blockIdx.x - table.first[at]) * kThinColumns;
    for (int64_t col = c0 + threadIdx.x; col < min(c0 + kThinColumns, static_cast<int64_t>(o.n)); col += kBlock) {
        double u[kThinSide];
        thin_column(update, t, o, col, u);
        for (int i = 0; i < o.m; ++i)                       // (a thread has read its column before it writes it: `out` may be `update`)
            put(out + t.src + i * o.row_step + col * o.col_step, static_cast<float>(thin_row(lds, i, o.m, u)));
    }
}

}  // namespace
