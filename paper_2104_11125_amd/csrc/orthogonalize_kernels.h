// Kernels that orthogonalise the matrices of an update by Newton-Schulz products.  Part of scalecom.hip's single
// translation unit.
//
// With m <= n the sides of a matrix (a tall one is worked on transposed) and X = U / (|U| + eps):
//
//   S = X X^T          m x m, symmetric: only tiles on and above the diagonal are computed, and written twice
//   B = b S + c S S    m x m, symmetric like S
//   X <- a X + B X     m x n
//
// Numbers.  The products run on the matrix units with 16-bit operands and 32-bit sums.  A value x is held as
// hi + lo, hi = half(s x), lo = half(s x - hi), with a power of two s that keeps every value the iteration can take
// (|x| <= 4, |S| <= 16, |B| <= 32, checked on the host from the coefficients) below the largest half and small ones
// away from the smallest.  SPLIT (32-bit results): hi hi + hi lo + lo hi, 22 bits per operand, the error of a product in
// binary32.  Otherwise (bfloat16 results): hi hi alone, 11 bits per operand.  In both, X enters a X with both
// halves, and the diagonals of S and B, about 1 and -2.5 where X is nearly orthogonal, are kept apart in binary32: their
// rounding to 11 bits would outweigh everything else.  Relative error of the result, 512 x 2048, before its rounding: 5e-4 (normal
// numbers) and 2.4e-4 (one direction a hundred times the others), where bfloat16 operands give 1.2e-2 and 1.6e-1.
// A matrix whose norm is small against eps starts from a small X: it is held times 2^e (OrthoMatrix::lift), and e falls
// with every step by the bits that the step can make X grow, so that it is used up before X reaches the range above.  (S and B
// need no such factor: beside a in a X + B X their absolute error counts.)
//
// Layout.  The scratch holds X, S and B (hi plane, then lo plane) as the LDS images that the products read: pieces of 64 rows x 32
// columns (4 KB), piece (r, c) of a row of pieces after the other, so a stage of a product is a few runs of whole
// kilobytes which the memory system copies to LDS as they are, and no pitch of a power of two hits one channel
// again and again.  Sides are padded with zeros to multiples of 128.  Inside a piece the four 16-byte chunks of a row are permuted
// (piece_chunk) so that neither the reads along rows (8 rows x 16 bytes at once) nor the transposing reads along
// columns (4 rows x 32 bytes) meet in a bank.
#pragma once

#include <hip/hip_runtime.h>

#include "device_helpers.h"
#include "geometry.h"
#include "optimizer_kernels.h"

namespace {

typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef float acc4_t __attribute__((ext_vector_type(4)));

constexpr int kOrthoTile = 128;                             // rows and columns of a block's tile; sides are multiples of it
constexpr int kPieceRows = 64, kPieceCols = 32;
constexpr int kPieceBytes = kPieceRows * kPieceCols * 2;
constexpr int kPiecesPerTile = kOrthoTile / kPieceCols;     // side by side
constexpr int kStageBytes = 32 * 1024;                      // both operands of a stage
constexpr int kOrthoPartsMax = 256;                         // partial sums of a norm
constexpr int kOrthoPartElements = 16384;
constexpr int kOrthoLiftMax = 100;
constexpr float kXScale = 4096.0f, kSScale = 2048.0f, kBScale = 1024.0f;

// One matrix, as the kernels see it.  Offsets into the scratch are bytes.
struct OrthoMatrix {
    int64_t src, stride;                                    // of the caller's vectors, in elements
    int64_t x, s;                                           // X (two copies of two planes), S (then B: two planes each, then the two diagonals)
    int32_t rows, cols;
    uint32_t part_first;                                    // its first partial sum = its first block of k_ortho_begin
    uint32_t tile_first, pair_first;                        // its first entries of the lists of tiles of X, and of S
    uint32_t parts;
    int32_t lift, pad;                                      // k_ortho_normalize leaves here: X is scaled up by 2^lift at first
};
constexpr int kOrthoMatrices = 60;                          // per launch of k_ortho_begin: 3840 bytes of arguments
static_assert(sizeof(OrthoMatrix) == 64, "");
struct OrthoTable {
    OrthoMatrix m[kOrthoMatrices];
};

struct OrthoTileRef {                                       // an entry of the lists of tiles
    uint32_t matrix;
    uint16_t row, col;                                      // in tiles
};

__host__ __device__ __forceinline__ int32_t pad_tile(int32_t n) { return (n + kOrthoTile - 1) / kOrthoTile * kOrthoTile; }

struct OrthoShape {                                         // what follows from a matrix's sides
    int32_t m, n, mp, np;                                   // short and long side, padded
    bool tall;
    size_t xplane, splane;                                  // bytes
};

__host__ __device__ __forceinline__ OrthoShape ortho_shape(int32_t rows, int32_t cols)
{
    OrthoShape o;
    o.tall = rows > cols;
    o.m = o.tall ? cols : rows;
    o.n = o.tall ? rows : cols;
    o.mp = pad_tile(o.m);
    o.np = pad_tile(o.n);
    o.xplane = static_cast<size_t>(o.mp) * o.np * 2;
    o.splane = static_cast<size_t>(o.mp) * o.mp * 2;
    return o;
}

// Byte offset of the 16-byte chunk `chunk` of row `row` inside a piece.
__device__ __forceinline__ uint32_t piece_chunk(uint32_t row, uint32_t chunk)
{
    const uint32_t f = (row & 2u) | ((row >> 2) & 1u);
    return row * (kPieceCols * 2) + ((chunk ^ f) << 4);
}

// Byte offset of element (row, col) in a plane of `pieces` pieces per row of pieces.
__device__ __forceinline__ size_t plane_offset(uint32_t row, uint32_t col, uint32_t pieces)
{
    const size_t piece = static_cast<size_t>(row / kPieceRows) * pieces + col / kPieceCols;
    return piece * kPieceBytes + piece_chunk(row % kPieceRows, col % kPieceCols / 8) + col % 8 * 2;
}

__device__ __forceinline__ void split_half(float x, _Float16& hi, _Float16& lo)   // x is scaled already
{
    hi = static_cast<_Float16>(x);
    lo = static_cast<_Float16>(x - static_cast<float>(hi));
}

// Sum over a block of 256 threads, in one order.
__device__ __forceinline__ double block_sum(double v, double* lds)
{
    lds[threadIdx.x] = v;
    __syncthreads();
    for (int w = kBlock / 2; w > 0; w /= 2) {
        if (static_cast<int>(threadIdx.x) < w) lds[threadIdx.x] += lds[threadIdx.x + w];
        __syncthreads();
    }
    return lds[0];
}

// First kernel of a call: partial sums of every matrix's squares (binary64: no overflow, no underflow), its entry of the table
// and its entries of the lists of tiles.  The matrices travel with the launch, so nothing is copied from the host.
template <typename U>
__global__ void __launch_bounds__(kBlock)
k_ortho_begin(const U* __restrict__ update, int n, int first, const OrthoTable table, OrthoMatrix* __restrict__ mats,
              OrthoTileRef* __restrict__ tiles, OrthoTileRef* __restrict__ pairs, double* __restrict__ partial)
{
    const uint32_t block = table.m[0].part_first + blockIdx.x;
    int at = 0;                                             // the last matrix that begins at or before this block
    for (int hi = n; hi - at > 1;) {
        const int mid = (at + hi) / 2;
        if (table.m[mid].part_first <= block)
            at = mid;
        else
            hi = mid;
    }
    const OrthoMatrix& t = table.m[at];
    const uint32_t part = block - t.part_first;
    const OrthoShape o = ortho_shape(t.rows, t.cols);
    if (part == 0 && threadIdx.x == 0) mats[first + at] = t;
    const uint32_t worker = part * kBlock + threadIdx.x, workers = t.parts * kBlock;
    const uint32_t tm = o.mp / kOrthoTile, tn = o.np / kOrthoTile;
    for (uint32_t i = worker; i < tm * tn; i += workers)
        tiles[t.tile_first + i] = OrthoTileRef{static_cast<uint32_t>(first + at), static_cast<uint16_t>(i % tm),
                                               static_cast<uint16_t>(i / tm)};
    // pairs (row <= col), column after column: col (col + 1) / 2 of them lie before column col
    for (uint32_t i = worker; i < tm * (tm + 1) / 2; i += workers) {
        uint32_t col = static_cast<uint32_t>((sqrtf(8.0f * i + 1.0f) - 1.0f) * 0.5f);
        while (col * (col + 1) / 2 > i) --col;
        while ((col + 1) * (col + 2) / 2 <= i) ++col;
        pairs[t.pair_first + i] = OrthoTileRef{static_cast<uint32_t>(first + at), static_cast<uint16_t>(i - col * (col + 1) / 2),
                                               static_cast<uint16_t>(col)};
    }
    const bool one = t.stride == t.cols;                    // rows without gaps are one row
    const int64_t len = one ? static_cast<int64_t>(t.rows) * t.cols : t.cols;
    const int64_t quads = one ? row_quads(t.src, len) : (len + 2) / kVec + 1, all = one ? quads : quads * t.rows;
    double sum = 0.0;
    for (int64_t q = worker; q < all; q += workers) {
        const int64_t row = one ? 0 : q / quads, begin = t.src + row * t.stride;
        const int64_t p = (begin & ~static_cast<int64_t>(kVec - 1)) + (q - row * quads) * kVec;
        if (p >= begin + len) continue;
        const float4 v = load_guarded(update, p, begin, begin + len, p >= begin && p + 3 < begin + len);
        sum += static_cast<double>(v.x) * v.x + static_cast<double>(v.y) * v.y + static_cast<double>(v.z) * v.z +
               static_cast<double>(v.w) * v.w;
    }
    __shared__ double lds[kBlock];
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) partial[block] = sum;
}

// X = U / (|U| + eps), split into halves, one tile per block; zeros where the sides are padded.
template <typename U>
__global__ void __launch_bounds__(kBlock)
k_ortho_normalize(const U* __restrict__ update, OrthoMatrix* __restrict__ mats, const OrthoTileRef* __restrict__ tiles,
                  const double* __restrict__ partial, float eps, char* __restrict__ scratch)
{
    const OrthoTileRef ref = tiles[blockIdx.x];
    const OrthoMatrix t = mats[ref.matrix];
    const OrthoShape o = ortho_shape(t.rows, t.cols);
    __shared__ double lds[kBlock];
    const double norm = sqrt(block_sum(threadIdx.x < t.parts ? partial[t.part_first + threadIdx.x] : 0.0, lds));
    const double size = norm / (norm + static_cast<double>(eps));   // of X
    int lift = 0;
    if (size > 0.0 && size < 0.5) lift = min(-ilogb(size) - 1, kOrthoLiftMax);
    if (ref.row == 0 && ref.col == 0 && threadIdx.x == 0) mats[ref.matrix].lift = lift;
    const double inv = ldexp(static_cast<double>(kXScale), lift) / (norm + static_cast<double>(eps));
    char* hi = scratch + t.x;
    char* lo = hi + o.xplane;
    const uint32_t pieces = o.np / kPieceCols;
    for (int r = 0; r < kOrthoTile * kOrthoTile / 8 / kBlock; ++r) {
        // a chunk of eight columns of one row; along the direction in which the caller's rows run
        const uint32_t c = r * kBlock + threadIdx.x;
        const uint32_t row = ref.row * kOrthoTile + (o.tall ? c % kOrthoTile : c / (kOrthoTile / 8));
        const uint32_t col = ref.col * kOrthoTile + (o.tall ? c / kOrthoTile : c % (kOrthoTile / 8)) * 8;
        half8_t h, l;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float x = 0.0f;
            if (row < static_cast<uint32_t>(o.m) && col + e < static_cast<uint32_t>(o.n)) {
                const int64_t p = o.tall ? t.src + static_cast<int64_t>(col + e) * t.stride + row
                                         : t.src + static_cast<int64_t>(row) * t.stride + col + e;
                x = static_cast<float>(static_cast<double>(widen(update[p])) * inv);
            }
            _Float16 a, b;
            split_half(x, a, b);
            h[e] = a;
            l[e] = b;
        }
        const size_t at = plane_offset(row, col, pieces);
        *reinterpret_cast<half8_t*>(hi + at) = h;
        *reinterpret_cast<half8_t*>(lo + at) = l;
    }
}

// The three products ------------------------------------------------------------------------------
// A block computes one tile of 128 x 128 with four waves of 64 x 64 (4 x 4 products of 16 x 16 x 32).  A stage takes 64 (SPLIT: 32)
// places of the inner dimension of both operands to LDS, 32 KB, while the one before is multiplied.
enum OrthoProduct { kGram = 0, kPoly = 1, kStep = 2, kLast = 3 };

template <bool SPLIT>
struct OrthoOut {
    using type = uint16_t;
};
template <>
struct OrthoOut<true> {
    using type = float;
};

typedef __attribute__((address_space(1))) const void* global_ptr_t;
typedef __attribute__((address_space(3))) void* lds_ptr_t;

// An operand whose rows are the tile's rows (two rows of pieces, `row_bytes` apart) or, TR, whose columns are (the inner
// dimension runs along its rows of pieces).  Copies one stage of 16 KB; wave w takes every fourth kilobyte.
template <bool SPLIT, bool TR>
__device__ __forceinline__ void copy_stage(char* lds, const char* src, size_t plane, size_t row_bytes, int stage, int wave, int lane)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 4 + wave;                         // kilobyte of the operand's image
        const int part = SPLIT ? c % 8 : c;
        size_t at;
        if (!TR)        // [row of pieces][piece]: 8 KB (SPLIT: 4 KB) in a run
            at = SPLIT ? (part / 4) * row_bytes + static_cast<size_t>(stage) * kPieceBytes + part % 4 * 1024
                       : (part / 8) * row_bytes + static_cast<size_t>(stage) * (2 * kPieceBytes) + part % 8 * 1024;
        else            // [piece]: 16 KB in a run (SPLIT: the upper or lower 32 rows of four pieces)
            at = SPLIT ? static_cast<size_t>(stage / 2) * row_bytes + (part / 2) * kPieceBytes + stage % 2 * (kPieceBytes / 2) + part % 2 * 1024
                       : static_cast<size_t>(stage) * row_bytes + part * 1024;
        if (SPLIT && c >= 8) at += plane;
        __builtin_amdgcn_global_load_lds((global_ptr_t)(src + at + lane * 16), (lds_ptr_t)(lds + c * 1024), 16, 0, 0);
    }
}

// Fragment f (16 rows) of a wave's 64: 8 values along the inner dimension per lane, from the image of copy_stage.
template <bool SPLIT>
__device__ __forceinline__ half8_t row_fragment(const char* lds, int side, int f, int ks, int lane)
{
    constexpr int run = SPLIT ? kPieceBytes : 2 * kPieceBytes;
    return *reinterpret_cast<const half8_t*>(lds + side * run + ks * kPieceBytes + f * 16 * (kPieceCols * 2) +
                                             piece_chunk(lane % 16, lane / 16));
}

// The same along columns: a transposing read gives a lane its column of four rows.
template <bool SPLIT>
__device__ __forceinline__ half8_t col_fragment(const char* lds, int side, int f, int ks, int lane)
{
    constexpr int piece = SPLIT ? kPieceBytes / 2 : kPieceBytes;
    const uint32_t row = lane / 16 * 8 + lane % 16 / 4;     // first of the two groups of four rows; the second begins 4 below
    const uint32_t chunk = f % 2 * 2 + lane % 4 / 2;
    const char* base = lds + (side * 2 + f / 2) * piece + ks * 32 * (kPieceCols * 2) + lane % 2 * 8;
    typedef __attribute__((address_space(3))) short4_t* lds_s4_t;
    const short4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t)(lds_ptr_t)(const_cast<char*>(base) + piece_chunk(row, chunk)));
    const short4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t)(lds_ptr_t)(const_cast<char*>(base) + piece_chunk(row + 4, chunk)));
    return __builtin_bit_cast(half8_t, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <bool SPLIT, bool TR>
__device__ __forceinline__ void multiply_stage(const char* lds, int wi, int wj, int lane, acc4_t acc[4][4])
{
    constexpr int kOperand = kStageBytes / 2, kLow = kOperand / 2;
#pragma unroll
    for (int ks = 0; ks < (SPLIT ? 1 : 2); ++ks) {
        half8_t a[4], b[4], al[4], bl[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            a[f] = TR ? col_fragment<SPLIT>(lds, wi, f, ks, lane) : row_fragment<SPLIT>(lds, wi, f, ks, lane);
            b[f] = row_fragment<SPLIT>(lds + kOperand, wj, f, ks, lane);
            if (SPLIT) {
                al[f] = TR ? col_fragment<SPLIT>(lds + kLow, wi, f, ks, lane) : row_fragment<SPLIT>(lds + kLow, wi, f, ks, lane);
                bl[f] = row_fragment<SPLIT>(lds + kOperand + kLow, wj, f, ks, lane);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (SPLIT) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al[i], b[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i], bl[j], acc[i][j], 0, 0, 0);
                }
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i], b[j], acc[i][j], 0, 0, 0);
            }
    }
}

// kGram and kPoly: pairs of tiles (row, col), row <= col, of S = X X^T and of B = b S + c S S.
// kStep and kLast: tiles of a X + B X; the last one goes to the caller's vector.
// `from`: which copy of X is read.  X is scaled up by 2^max(lift - spent, 0) more than usual, and in the next step, where it
// may be larger by 2^growth, by that much less.
template <OrthoProduct P, bool SPLIT>
__global__ void __launch_bounds__(kBlock)
k_ortho_product(char* __restrict__ scratch, const OrthoMatrix* __restrict__ mats, const OrthoTileRef* __restrict__ refs, uint32_t n_refs,
                int from, int spent, int growth, float ca, float cb, float cc, typename OrthoOut<SPLIT>::type* __restrict__ out)
{
    constexpr bool kPair = P == kGram || P == kPoly, TR = !kPair;
    __shared__ __attribute__((aligned(1024))) char buf0[kStageBytes];
    __shared__ __attribute__((aligned(1024))) char buf1[kStageBytes];
    const OrthoTileRef ref = refs[piece_by_xcd(blockIdx.x, n_refs)];
    const OrthoMatrix t = mats[ref.matrix];
    const OrthoShape o = ortho_shape(t.rows, t.cols);
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int wi = wave / 2, wj = wave % 2;
    char* x = scratch + t.x + (from ? 2 * o.xplane : 0);
    char* s = scratch + t.s;
    char* b = s + 2 * o.splane;
    float* ds = reinterpret_cast<float*>(b + 2 * o.splane);
    float* db = ds + o.mp;
    const size_t xrow = static_cast<size_t>(o.np) / kPieceCols * kPieceBytes, srow = static_cast<size_t>(o.mp) / kPieceCols * kPieceBytes;
    // operands: rows of X twice; rows of S twice; columns of X with rows of B
    const char* pa = P == kGram ? x + ref.row * 2 * xrow : P == kPoly ? s + ref.row * 2 * srow : x + ref.col * (kPiecesPerTile * kPieceBytes);
    const char* pb = P == kGram ? x + ref.col * 2 * xrow : P == kPoly ? s + ref.col * 2 * srow : b + ref.row * 2 * srow;
    const size_t plane_a = P == kPoly ? o.splane : o.xplane, plane_b = P == kGram ? o.xplane : o.splane;
    const size_t row_a = P == kPoly ? srow : xrow, row_b = P == kGram ? xrow : srow;
    const int lift = max(t.lift - spent, 0);
    const int stages = (P == kGram ? o.np : o.mp) / (SPLIT ? 32 : 64);   // even
    auto copy = [&](char* lds, int stage) {
        copy_stage<SPLIT, TR>(lds, pa, plane_a, row_a, stage, wave, lane);
        copy_stage<SPLIT, false>(lds + kStageBytes / 2, pb, plane_b, row_b, stage, wave, lane);
    };
    acc4_t acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = acc4_t{0.0f, 0.0f, 0.0f, 0.0f};
    copy(buf0, 0);
    for (int stage = 0; stage < stages; stage += 2) {
        __syncthreads();                                    // (waits for the copies too)
        copy(buf1, stage + 1);
        multiply_stage<SPLIT, TR>(buf0, wi, wj, lane, acc);
        __syncthreads();
        if (stage + 2 < stages) copy(buf0, stage + 2);
        multiply_stage<SPLIT, TR>(buf1, wi, wj, lane, acc);
    }
    // a lane holds four consecutive places of the first operand's side (i) at one of the second's (j)
    if constexpr (kPair) {
        const uint32_t pieces = o.mp / kPieceCols;
#pragma unroll
        for (int fi = 0; fi < 4; ++fi)
#pragma unroll
            for (int fj = 0; fj < 4; ++fj) {
                const uint32_t i = ref.row * kOrthoTile + wi * 64 + fi * 16 + lane / 16 * 4, j = ref.col * kOrthoTile + wj * 64 + fj * 16 + lane % 16;
                acc4_t& v = acc[fi][fj];
                if (P == kGram) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        v[r] = ldexpf(v[r] * (1.0f / (kXScale * kXScale)), -2 * lift);
                        if (i + r == j) {
                            ds[j] = v[r];
                            v[r] = 0.0f;
                        }
                        v[r] *= kSScale;
                    }
                } else {
                    const size_t at = plane_offset(j, i, pieces);                 // (S is symmetric)
                    const half4_t eh = *reinterpret_cast<const half4_t*>(s + at);
                    half4_t el = {0, 0, 0, 0};
                    if (SPLIT) el = *reinterpret_cast<const half4_t*>(s + o.splane + at);
                    const float dj = ds[j];
                    const float4 di = *reinterpret_cast<const float4*>(ds + i);
                    const float d[4] = {di.x, di.y, di.z, di.w};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        // S = D + E with a diagonal D: S S = D D + D E + E D + E E
                        const float e = (static_cast<float>(eh[r]) + static_cast<float>(el[r])) * (1.0f / kSScale);
                        const float q = v[r] * (1.0f / (kSScale * kSScale));
                        if (i + r == j) {
                            db[j] = fmaf(cb, dj, cc * fmaf(dj, dj, q));
                            v[r] = 0.0f;
                        } else {
                            v[r] = fmaf(cb, e, cc * fmaf(d[r] + dj, e, q)) * kBScale;
                        }
                    }
                }
            }
        // the tile's image, rows of the second side, then (for the other triangle) rows of the first
        char* to = P == kGram ? s : b;
        for (int turn = 0; turn < (ref.row == ref.col ? 1 : 2); ++turn) {
            __syncthreads();
#pragma unroll
            for (int fi = 0; fi < 4; ++fi)
#pragma unroll
                for (int fj = 0; fj < 4; ++fj) {
                    const uint32_t i = wi * 64 + fi * 16 + lane / 16 * 4, j = wj * 64 + fj * 16 + lane % 16;
                    half4_t h, l;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        _Float16 a, c;
                        split_half(acc[fi][fj][r], a, c);
                        h[r] = a;
                        l[r] = c;
                    }
                    if (turn == 0) {
                        const size_t at = plane_offset(j, i, kPiecesPerTile);
                        *reinterpret_cast<half4_t*>(buf0 + at) = h;
                        if (SPLIT) *reinterpret_cast<half4_t*>(buf1 + at) = l;
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const size_t at = plane_offset(i + r, j, kPiecesPerTile);
                            *reinterpret_cast<_Float16*>(buf0 + at) = h[r];
                            if (SPLIT) *reinterpret_cast<_Float16*>(buf1 + at) = l[r];
                        }
                    }
                }
            __syncthreads();
            const uint32_t row = turn == 0 ? ref.col : ref.row, col = turn == 0 ? ref.row : ref.col;
            for (uint32_t c = threadIdx.x; c < kStageBytes / 16; c += kBlock) {
                const size_t at = (row * 2 + c / (kStageBytes / 32)) * srow + col * (kPiecesPerTile * kPieceBytes) + c % (kStageBytes / 32) * 16;
                *reinterpret_cast<vf4_t*>(to + at) = *reinterpret_cast<const vf4_t*>(buf0 + c * 16);
                if (SPLIT) *reinterpret_cast<vf4_t*>(to + o.splane + at) = *reinterpret_cast<const vf4_t*>(buf1 + c * 16);
            }
        }
    } else {
        const uint32_t pieces = o.np / kPieceCols;
        char* next = scratch + t.x + (from ? 0 : 2 * o.xplane);
        const float rescale = P == kStep ? ldexpf(1.0f, max(lift - growth, 0) - lift) : ldexpf(1.0f / kXScale, -lift);
#pragma unroll
        for (int fj = 0; fj < 4; ++fj) {
            const uint32_t j = ref.row * kOrthoTile + wj * 64 + fj * 16 + lane % 16;   // row of X
            const float scale = ca + db[j];
#pragma unroll
            for (int fi = 0; fi < 4; ++fi) {
                const uint32_t i = ref.col * kOrthoTile + wi * 64 + fi * 16 + lane / 16 * 4;   // first of four columns
                const size_t at = plane_offset(j, i, pieces);
                const half4_t xh = *reinterpret_cast<const half4_t*>(x + at), xl = *reinterpret_cast<const half4_t*>(x + o.xplane + at);
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    v[r] = fmaf(scale, static_cast<float>(xh[r]) + static_cast<float>(xl[r]), acc[fi][fj][r] * (1.0f / kBScale));
                if (P == kStep) {
                    half4_t h, l;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        _Float16 a, c;
                        split_half(v[r] * rescale, a, c);
                        h[r] = a;
                        l[r] = c;
                    }
                    *reinterpret_cast<half4_t*>(next + at) = h;
                    *reinterpret_cast<half4_t*>(next + o.xplane + at) = l;
                } else if (j < static_cast<uint32_t>(o.m)) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (i + r < static_cast<uint32_t>(o.n))
                            put(out + (o.tall ? t.src + static_cast<int64_t>(i + r) * t.stride + j : t.src + static_cast<int64_t>(j) * t.stride + i + r), v[r] * rescale);
                }
            }
        }
    }
}

}  // namespace
