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
// (|x| <= 4, |S| <= 16, |B| <= 32) below the largest half; the host checks that from the coefficients, and that no steps make X so
// small that its halves come near the smallest.  SPLIT (32-bit results): hi hi + hi lo + lo hi, 22 bits per operand, the error of a product in
// binary32; X becomes (a I + B) X then.  Otherwise (bfloat16 results): hi hi alone, 11 bits per operand; X enters a X with
// both halves, and the diagonals of S and B, about 1 and -2.5 where X is nearly orthogonal, are kept apart in binary32: their
// rounding to 11 bits would outweigh everything else.  Relative error of the result, 512 x 2048, before its rounding: 5e-4 (normal
// numbers) and 2.4e-4 (one direction a hundred times the others), where bfloat16 operands give 1.2e-2 and 1.6e-1.  It is the rounding of what S
// and B hold off the diagonal that counts, against one large direction about 0.1 / sqrt(m) of it: 1.8e-2 for a 3 x 50 of rank 1, 6e-3 for a 60 x 600.
// A matrix whose norm is small against eps starts from a small X: it is held times 2^e (OrthoMatrix::lift), and e falls
// with every step by the bits that the step can make X grow, so that it is used up before X reaches the range above.  (S and B
// need no such factor: beside a in a X + B X their absolute error counts.)
//
// Layout.  The scratch holds X, S and B (hi plane, then lo plane) as the LDS images that the products read: pieces of 64 rows x 32
// columns (4 KB), piece (r, c) of a row of pieces after the other, so a stage of a product is a few runs of whole
// kilobytes which the memory system copies to LDS as they are, and no pitch of a power of two hits one channel
// again and again.  Sides are padded with zeros to multiples of the largest tile, 128 or 256.  Inside a piece the four 16-byte chunks of a row are permuted
// (piece_chunk) so that 8 rows x 16 bytes and, for the transposing reads along columns, 4 rows x 32 bytes lie in banks of their own.  A read takes
// twice as many rows at once and meets twofold: of the cycles in which the LDS is busy with the products' reads (SQ_LDS_IDX_ACTIVE) 46 to 50 % are
// bank conflicts (SQ_LDS_BANK_CONFLICT), in every product.
//
// What bounds it, us a launch: in tiles of 256 the matrix units, their power, and the LDS with its conflicts (bf16 16384 x 4096: X X^T 279 and its join
// 34, S S 106, B X 516, 1.07 PFLOP/s; matrix units busy 77, 71 and 63 % of the time that CUs are, the LDS 58, 58 and 51 %; f32 2048 x 8192: B X 179, 1.15
// PFLOP/s of 16-bit products; times rise by a third within a run as the clock falls); in tiles of 128 what a block takes before its first and
// after its last stage (72 x 512 x 512 and 24 x 512 x 2048, bf16: 52, 36, 105; matrix units busy 36, 27 and 23 %, B X 2.8 TB/s from and to HBM).
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

constexpr int kPieceRows = 64, kPieceCols = 32;
constexpr int kPieceBytes = kPieceRows * kPieceCols * 2;
constexpr int kPieceRowBytes = kPieceCols * 2;
constexpr int kOrthoPartsMax = 2048;                        // partial sums of a norm
constexpr int kOrthoPartElements = 8192;                    // of a matrix's elements, at least
constexpr int kOrthoLiftMax = 127;                          // 2^-22, of X's and B's scales, times 2^-127 is the last power of two that binary32 holds
constexpr float kXScale = 4096.0f, kSScale = 2048.0f, kBScale = 1024.0f;

enum OrthoProduct { kGram = 0, kPoly = 1, kStep = 2, kLast = 3 };

// One matrix, as the kernels see it.  Offsets into the scratch are bytes; `first`, `join_first` and `cell_first` index one list of
// tiles, in which every launch has a section of its own.
struct OrthoMatrix {
    int64_t src, stride;                                    // of the caller's vectors, in elements
    int64_t x, s;                                           // X (two copies of two planes), S (then B: two planes each, then the two diagonals)
    int32_t rows, cols;
    int32_t pad;                                            // the sides are padded to multiples of it: its largest tile
    int32_t lift;                                           // k_ortho_normalize leaves here: X is scaled up by 2^lift at first
    uint32_t part_first, parts;                             // partial sums of its norm = blocks of k_ortho_begin
    uint32_t cell_first;                                    // tiles of k_ortho_normalize
    uint32_t first[3];                                      // tiles of kGram (pairs), kPoly (pairs), kStep
    uint32_t join_first[2];                                 // kGram, kPoly with more than one split: pairs to be put together
    uint32_t slot_first[2];                                 // and their partial tiles, in units of 128 x 128
    uint16_t tile[3];                                       // rows and columns of these tiles: 128 or 256
    uint8_t splits[2];                                      // blocks that share the inner dimension of a pair
};
constexpr int kOrthoMatrices = 39;                          // per launch of k_ortho_begin: 3900 bytes of arguments
static_assert(sizeof(OrthoMatrix) == 96, "");
struct OrthoTable {
    uint32_t first[kOrthoMatrices];                         // block of k_ortho_begin
    OrthoMatrix m[kOrthoMatrices];
};

struct OrthoTileRef {                                       // an entry of the list of tiles
    uint32_t matrix : 24, split : 8;
    uint16_t row, col;                                      // in tiles
};
// A launch's entries, cut into one run of consecutive entries per XCD with like amounts of work (its matrices' tiles meet in that XCD's L2).
// Blocks go to the XCDs in turn.
struct OrthoRuns {
    uint32_t first[kXcds + 1];
};
__device__ __forceinline__ bool run_entry(const OrthoRuns& runs, uint32_t block, uint32_t& entry)
{
    const uint32_t xcd = block % kXcds;
    entry = runs.first[xcd] + block / kXcds;
    return entry < runs.first[xcd + 1];
}

constexpr int kOrthoMatricesMax = 1 << 24;
constexpr int kOrthoCell = 128;                             // rows and columns of a block of k_ortho_normalize

struct OrthoShape {                                         // what follows from a matrix's sides
    int32_t m, n, mp, np;                                   // short and long side, padded
    bool tall;
    size_t xplane, splane;                                  // bytes
};

__host__ __device__ __forceinline__ OrthoShape ortho_shape(int32_t rows, int32_t cols, int32_t pad)
{
    OrthoShape o;
    o.tall = rows > cols;
    o.m = o.tall ? cols : rows;
    o.n = o.tall ? rows : cols;
    o.mp = (o.m + pad - 1) / pad * pad;
    o.np = (o.n + pad - 1) / pad * pad;
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
              OrthoTileRef* __restrict__ refs, double* __restrict__ partial)
{
    const int at = find_block(table.first, n, blockIdx.x);
    const OrthoMatrix t = table.m[at];
    const uint32_t block = t.part_first + blockIdx.x - table.first[at];
    const uint32_t part = block - t.part_first;
    const OrthoShape o = ortho_shape(t.rows, t.cols, t.pad);
    const uint32_t matrix = first + at;
    if (part == 0 && threadIdx.x == 0) mats[matrix] = t;
    const uint32_t worker = part * kBlock + threadIdx.x, workers = t.parts * kBlock;
    // tiles of X, column after column
    for (int list = 0; list < 2; ++list) {
        const uint32_t side = list == 0 ? kOrthoCell : t.tile[kStep], tm = o.mp / side, n_tiles = tm * (o.np / side);
        OrthoTileRef* to = refs + (list == 0 ? t.cell_first : t.first[kStep]);
        for (uint32_t i = worker; i < n_tiles; i += workers)
            to[i] = OrthoTileRef{matrix, 0, static_cast<uint16_t>(i % tm), static_cast<uint16_t>(i / tm)};
    }
    // pairs (row <= col), column after column: col (col + 1) / 2 of them lie before column col
    for (int p = 0; p < 2; ++p) {
        const uint32_t tm = o.mp / t.tile[p], n_pairs = tm * (tm + 1) / 2, splits = t.splits[p];
        for (uint32_t i = worker; i < n_pairs * splits; i += workers) {
            const uint32_t pair = i / splits;
            uint32_t col = static_cast<uint32_t>((sqrtf(8.0f * pair + 1.0f) - 1.0f) * 0.5f);
            while (col * (col + 1) / 2 > pair) --col;
            while ((col + 1) * (col + 2) / 2 <= pair) ++col;
            const OrthoTileRef ref{matrix, i % splits, static_cast<uint16_t>(pair - col * (col + 1) / 2), static_cast<uint16_t>(col)};
            refs[t.first[p] + i] = ref;
            if (splits > 1 && i % splits == 0) refs[t.join_first[p] + pair] = ref;
        }
    }
    const bool one = t.stride == t.cols;                    // rows without gaps are one row
    const int64_t len = one ? static_cast<int64_t>(t.rows) * t.cols : t.cols;
    const int64_t quads = one ? row_quads(t.src, len) : (len + 2) / kVec + 1, all = one ? quads : quads * t.rows;
    double sum = 0.0;
#pragma unroll 8
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

// What U is multiplied by, from the sum of its squares: kXScale / (|U| + eps), times 2^lift where X is small.
struct OrthoScale {
    double factor;
    int lift;
    __device__ __forceinline__ OrthoScale(double squares, float eps)
    {
        const double norm = sqrt(squares), size = norm / (norm + static_cast<double>(eps));   // |X|
        lift = size > 0.0 && size < 0.5 ? min(-ilogb(size) - 1, kOrthoLiftMax) : 0;
        factor = ldexp(static_cast<double>(kXScale), lift) / (norm + static_cast<double>(eps));
    }
};

// Four consecutive elements of a row of the caller's matrix; zeros where it has none.
template <typename U>
__device__ __forceinline__ void four_of_row(const U* __restrict__ update, const OrthoMatrix& t, uint32_t row, uint32_t col, uint32_t rows, uint32_t cols,
                                            float* x)
{
    const int64_t p = t.src + static_cast<int64_t>(row) * t.stride + col;
    if (row < rows && col + 3 < cols && p % kVec == 0) {
        const float4 v = cached4(update + p);
        x[0] = v.x;
        x[1] = v.y;
        x[2] = v.z;
        x[3] = v.w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = row < rows && col + e < cols ? widen(update[p + e]) : 0.0f;
}

// X = U / (|U| + eps), split into halves, 128 x 128 per block; zeros where the sides are padded.
template <typename U>
__global__ void __launch_bounds__(kBlock)
k_ortho_normalize(const U* __restrict__ update, OrthoMatrix* __restrict__ mats, const OrthoTileRef* __restrict__ cells,
                  const double* __restrict__ partial, float eps, char* __restrict__ scratch)
{
    const OrthoTileRef ref = cells[blockIdx.x];
    const OrthoMatrix t = mats[ref.matrix];
    constexpr uint32_t side = kOrthoCell;
    const OrthoShape o = ortho_shape(t.rows, t.cols, t.pad);
    // Four rows and eight columns of X per thread and turn: along the caller's rows that is an access of 16 bytes at least.  All of them are
    // asked for before the norm is put together.
    constexpr int kTurns = kOrthoCell * kOrthoCell / 32 / kBlock;
    float x[kTurns][4][8];
    const auto row_of = [&](int turn) {                     // consecutive threads along the caller's rows
        const uint32_t c = turn * kBlock + threadIdx.x;
        return ref.row * side + (o.tall ? c % (side / 4) : c / (side / 8)) * 4;
    };
    const auto col_of = [&](int turn) {
        const uint32_t c = turn * kBlock + threadIdx.x;
        return ref.col * side + (o.tall ? c / (side / 4) : c % (side / 8)) * 8;
    };
#pragma unroll
    for (int turn = 0; turn < kTurns; ++turn) {
        const uint32_t row = row_of(turn), col = col_of(turn);
        if (!o.tall) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < 8; e += 4) four_of_row(update, t, row + r, col + e, o.m, o.n, x[turn][r] + e);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float v[4];
                four_of_row(update, t, col + e, row, o.n, o.m, v);
#pragma unroll
                for (int r = 0; r < 4; ++r) x[turn][r][e] = v[r];
            }
        }
    }
    __shared__ double lds[kBlock];
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < t.parts; i += kBlock) sum += partial[t.part_first + i];
    const OrthoScale scale(block_sum(sum, lds), eps);
    if (ref.row == 0 && ref.col == 0 && threadIdx.x == 0) mats[ref.matrix].lift = scale.lift;
    char* hi = scratch + t.x;
    char* lo = hi + o.xplane;
    const uint32_t pieces = o.np / kPieceCols;
#pragma unroll
    for (int turn = 0; turn < kTurns; ++turn)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            half8_t h, l;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                _Float16 a, b;
                split_half(static_cast<float>(static_cast<double>(x[turn][r][e]) * scale.factor), a, b);
                h[e] = a;
                l[e] = b;
            }
            const size_t at = plane_offset(row_of(turn) + r, col_of(turn), pieces);
            *reinterpret_cast<half8_t*>(hi + at) = h;
            *reinterpret_cast<half8_t*>(lo + at) = l;
        }
}

// The three products ------------------------------------------------------------------------------
// A block of WI x WJ waves computes a tile, every wave FI x FJ products of 16 x 16 x 32.  A stage takes 32 places of the inner
// dimension of both operands to LDS, which has room for B of them (four, SPLIT: two).
template <int WI_, int WJ_, int FI_, int FJ_, int B_, bool SPLIT_>
struct OrthoConfig {
    static constexpr int WI = WI_, WJ = WJ_, FI = FI_, FJ = FJ_, B = B_;
    static constexpr bool SPLIT = SPLIT_;
    static constexpr int TILE = WI * FI * 16;               // (square)
    static_assert(TILE == WJ * FJ * 16, "");
    static constexpr int WAVES = WI * WJ, THREADS = WAVES * kLanes;
    static constexpr int PLANE = TILE * kPieceRowBytes;     // bytes of one operand's plane in a stage
    static constexpr int OPERAND = PLANE * (SPLIT ? 2 : 1), STAGE = 2 * OPERAND;
    static constexpr int COPIES = OPERAND / 1024 / WAVES;   // of a kilobyte, per wave and operand
    static_assert(OPERAND % (1024 * WAVES) == 0, "");
    static_assert(B * STAGE <= 160 * 1024, "");
    static_assert(B * STAGE >= WAVES * FI * FJ * 512, "an image of every wave's part at the end");
    using Out = typename std::conditional<SPLIT, float, uint16_t>::type;
};

typedef __attribute__((address_space(1))) const void* global_ptr_t;
typedef __attribute__((address_space(3))) void* lds_ptr_t;

// One stage of an operand whose rows are the tile's rows (rows of pieces `row_bytes` apart, a piece of each) or, TR, whose columns
// are (the upper or lower 32 rows of consecutive pieces).  Wave w takes every WAVES-th kilobyte, a lane the 16 bytes at `mine`.
template <typename C, bool TR>
__device__ __forceinline__ void copy_stage(char* lds, const char* src, size_t plane, size_t row_bytes, int stage, int wave, uint32_t mine)
{
#pragma unroll
    for (int i = 0; i < C::COPIES; ++i) {
        const int c = i * C::WAVES + wave;                  // kilobyte of the operand's image
        const int part = c % (C::PLANE / 1024);
        size_t at = !TR ? (part / 4) * row_bytes + static_cast<size_t>(stage) * kPieceBytes + part % 4 * 1024
                        : static_cast<size_t>(stage / 2) * row_bytes + (part / 2) * kPieceBytes + stage % 2 * (kPieceBytes / 2) + part % 2 * 1024;
        if (C::SPLIT && c >= C::PLANE / 1024) at += plane;
        __builtin_amdgcn_global_load_lds((global_ptr_t)(src + at + mine), (lds_ptr_t)(lds + c * 1024), 16, 0, 0);
    }
}

// A transposing read: a lane's column of four rows, of 16 columns and the rows that its group of 16 lanes points to.
__device__ __forceinline__ short4_t read_columns(const char* at)
{
    typedef __attribute__((address_space(3))) short4_t* lds_s4_t;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t)(lds_ptr_t) const_cast<char*>(at));
}

__device__ __forceinline__ half8_t join_halves(short4_t a, short4_t b)
{
    return __builtin_bit_cast(half8_t, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Where a lane reads in an operand's plane: a fragment of 16 rows takes 8 values along the inner dimension at `row`; one of 16 columns
// (TR) four at `col[0]` and four in the rows that follow at `col[1]`, with the other half of a piece's columns at `col[2]`, `col[3]`.
// fresh(): the same, but as far as the compiler can tell values of its own; otherwise it keeps an address register for every
// combination with the stages' arrays through the whole loop, which costs more than there are.
struct LanePlaces {
    uint32_t row, col[4];
    __device__ __forceinline__ LanePlaces(int first, int lane)
    {
        row = first * kPieceRowBytes + piece_chunk(lane % 16, lane / 16);
        const uint32_t r = lane / 16 * 8 + lane % 16 / 4, base = first / kPieceCols * (kPieceBytes / 2) + lane % 2 * 8;
        col[0] = base + piece_chunk(r, lane % 4 / 2);
        col[1] = base + piece_chunk(r + 4, lane % 4 / 2);
        col[2] = base + piece_chunk(r, 2 + lane % 4 / 2);
        col[3] = base + piece_chunk(r + 4, 2 + lane % 4 / 2);
    }
    template <bool TR>
    __device__ __forceinline__ LanePlaces fresh() const
    {
        LanePlaces p = *this;
        if (TR)
            asm volatile("" : "+v"(p.col[0]), "+v"(p.col[1]), "+v"(p.col[2]), "+v"(p.col[3]));
        else
            asm volatile("" : "+v"(p.row));
        return p;
    }
};

// Fragment f of a wave's part of an operand's plane.
template <bool TR>
__device__ __forceinline__ half8_t read_fragment(const char* lds, int f, const LanePlaces& p)
{
    if (!TR) return *reinterpret_cast<const half8_t*>(lds + p.row + f * (16 * kPieceRowBytes));
    const char* at = lds + f / 2 * (kPieceBytes / 2);
    return join_halves(read_columns(at + p.col[f % 2 * 2]), read_columns(at + p.col[f % 2 * 2 + 1]));
}

// The fragments of a wave in one stage, of the hi planes or of the lo planes (which lie C::PLANE behind).
template <typename C>
struct OrthoFragments {
    half8_t a[C::FI], b[C::FJ];
};

template <typename C, bool TR>
__device__ __forceinline__ void read_first(const char* lds, const LanePlaces& p, OrthoFragments<C>& f)
{
#pragma unroll
    for (int i = 0; i < C::FI; ++i) f.a[i] = read_fragment<TR>(lds, i, p);
}

template <typename C>
__device__ __forceinline__ void read_second(const char* lds, const LanePlaces& p, OrthoFragments<C>& f)
{
#pragma unroll
    for (int j = 0; j < C::FJ; ++j) f.b[j] = read_fragment<false>(lds, j, p);
}

template <typename C>
__device__ __forceinline__ void multiply(const half8_t (&a)[C::FI], const half8_t (&b)[C::FJ], acc4_t (&acc)[C::FI][C::FJ])
{
#pragma unroll
    for (int i = 0; i < C::FI; ++i)
#pragma unroll
        for (int j = 0; j < C::FJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i], b[j], acc[i][j], 0, 0, 0);
}

// Lets the scheduler put a read of LDS between every EVERY products: all at once they fill the queue of the LDS, which eight waves
// share, and the products behind them would wait.
template <int READS, int EVERY>
__device__ __forceinline__ void spread_reads()
{
#pragma unroll
    for (int i = 0; i < READS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, EVERY, 0);
    }
}

// Waits until all but the last N copies that this wave asked for have arrived and its reads of LDS are done, then for the block.
template <int N>
__device__ __forceinline__ void stage_barrier()
{
    static_assert(N < 64, "");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);   // vmcnt(N) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Where things are in a wave's part of a tile.  A lane holds four consecutive places (r) of the first operand's side, i, at one of
// the second's, j: in the product (fi, fj) i = i0 + fi * 16 + lane / 16 * 4 + r, j = j0 + fj * 16 + lane % 16.  Where X, S
// or B lie row by row along j that is half a chunk, whose place differs between products by whole pieces and rows, and by one
// bit for odd fi.
struct OrthoPlaces {
    uint32_t i0, j0, i_lane, j_lane, even, odd;
    __device__ __forceinline__ OrthoPlaces(uint32_t i, uint32_t j, int lane)
        : i0(i), j0(j), i_lane(i + lane / 16 * 4), j_lane(j + lane % 16), even(piece_chunk(lane % 16, lane / 32) + lane / 16 % 2 * 8), odd(even ^ 32)
    {
    }
    __device__ __forceinline__ uint32_t operator()(int fi, int fj) const
    {
        return fi / 2 * kPieceBytes + fj % 4 * (16 * kPieceRowBytes) + (fi % 2 ? odd : even);
    }
};

// The sums of a pair of tiles, complete: S from X X^T, or B from S S, written on both sides of the diagonal.  `image`: LDS of this wave's own,
// which holds its part of S already, its first READY planes.
template <OrthoProduct P, typename C, int READY>
__device__ __forceinline__ void finish_pair(acc4_t (&acc)[C::FI][C::FJ], const OrthoTileRef& ref, const OrthoShape& o, char* s, int lift, float ca,
                                            float cb, float cc, char* image, int wi, int wj, int lane)
{
    constexpr bool SPLIT = C::SPLIT;
    char* b = s + 2 * o.splane;
    float* ds = reinterpret_cast<float*>(b + 2 * o.splane);
    float* db = ds + o.mp;
    const size_t srow = static_cast<size_t>(o.mp) / kPieceCols * kPieceBytes;
    const OrthoPlaces place(ref.row * C::TILE + wi * C::FI * 16, ref.col * C::TILE + wj * C::FJ * 16, lane);
    const uint32_t i0 = place.i0, j0 = place.j0;
    const char* s_part = s + (j0 / kPieceRows) * srow + (i0 / kPieceCols) * kPieceBytes;    // (S is symmetric)
    // the diagonal, in the products that hold some of it (one for every fj, at most)
    float on[C::FJ];                                        // what B holds there: nothing, or SPLIT: a I + B whole
#pragma unroll
    for (int fj = 0; fj < C::FJ; ++fj) on[fj] = 0.0f;
    if (ref.row == ref.col) {
#pragma unroll
        for (int fi = 0; fi < C::FI; ++fi)
#pragma unroll
            for (int fj = 0; fj < C::FJ; ++fj) {
                if (i0 + fi * 16 != j0 + fj * 16) continue;                  // (uniform)
                const int r = lane % 16 - lane / 16 * 4;
                const float v = r == 0 ? acc[fi][fj][0] : r == 1 ? acc[fi][fj][1] : r == 2 ? acc[fi][fj][2] : acc[fi][fj][3];
                if (r < 0 || r > 3) continue;
                const uint32_t j = place.j_lane + fj * 16;
                if (P == kGram) {
                    ds[j] = ldexpf(v * (1.0f / (kXScale * kXScale)), -2 * lift);
                } else {
                    const float d = ds[j];
                    const float all = ca + fmaf(cb, d, cc * fmaf(d, d, v * (1.0f / (kSScale * kSScale))));
                    if (SPLIT)
                        on[fj] = all * kBScale;
                    else
                        db[j] = all;
                }
            }
    }
#pragma unroll
    for (int fj = 0; fj < C::FJ; ++fj) {
        const uint32_t j = place.j_lane + fj * 16;
        const float dj = P == kPoly ? ds[j] : 0.0f;
#pragma unroll
        for (int fi = 0; fi < C::FI; ++fi) {
            const uint32_t i = place.i_lane + fi * 16;
            acc4_t& v = acc[fi][fj];
            if (P == kGram) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = ldexpf(v[r] * (kSScale / (kXScale * kXScale)), -2 * lift);
                    v[r] = i + r == j ? 0.0f : e;
                }
            } else {
                const char* at = s_part + (fj / 4) * srow + place(fi, fj);
                const half4_t eh = *reinterpret_cast<const half4_t*>(READY > 0 ? image + place(fi, fj) : at);
                half4_t el = {0, 0, 0, 0};
                if (SPLIT) el = *reinterpret_cast<const half4_t*>(READY > 1 ? image + C::FI * C::FJ * 512 + place(fi, fj) : at + o.splane);
                const float4 di = *reinterpret_cast<const float4*>(ds + i);
                const float d[4] = {di.x, di.y, di.z, di.w};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    // S = D + E with a diagonal D: S S = D D + D E + E D + E E
                    const float e = (static_cast<float>(eh[r]) + static_cast<float>(el[r])) * (1.0f / kSScale);
                    const float off = fmaf(cb, e, cc * fmaf(d[r] + dj, e, v[r] * (1.0f / (kSScale * kSScale)))) * kBScale;
                    v[r] = i + r == j ? on[fj] : off;
                }
            }
        }
        if (P == kPoly) __builtin_amdgcn_sched_barrier(0);   // (all loads at once would take more registers than there are)
    }
    // every wave puts an image of its part together in LDS, plane by plane: rows along j, then (for the other triangle)
    // rows along i
    constexpr int kImage = C::FI * C::FJ * 512;
    char* to = P == kGram ? s : b;
    const uint32_t across = lane / 16 * (4 * kPieceRowBytes) + ((lane % 16 / 8 ^ lane / 16 % 2) << 4) + lane % 8 * 2;
#pragma unroll 1
    for (int turn = 0; turn < (ref.row == ref.col ? 1 : 2); ++turn) {
        const uint32_t run = (turn == 0 ? C::FI : C::FJ) * (kPieceBytes / 32);   // 16-byte words of a row of pieces
        char* begin = to + ((turn == 0 ? j0 : i0) / kPieceRows) * srow + ((turn == 0 ? i0 : j0) / kPieceCols) * kPieceBytes;
#pragma unroll
        for (int plane = 0; plane < (SPLIT ? 2 : 1); ++plane) {
#pragma unroll
            for (int fi = 0; fi < C::FI; ++fi)
#pragma unroll
                for (int fj = 0; fj < C::FJ; ++fj) {
                    half4_t h;
                    asm volatile("" : "+v"(acc[fi][fj]));            // (split anew in every turn, not kept)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        _Float16 hi, lo;
                        split_half(acc[fi][fj][r], hi, lo);
                        h[r] = plane == 0 ? hi : lo;
                    }
                    if (turn == 0) {
                        *reinterpret_cast<half4_t*>(image + fj / 4 * (C::FI / 2 * kPieceBytes) + place(fi, fj)) = h;
                    } else {
                        char* at = image + fi / 4 * (C::FJ / 2 * kPieceBytes) + fj / 2 * kPieceBytes + fi % 4 * (16 * kPieceRowBytes);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            *reinterpret_cast<_Float16*>(at + r * kPieceRowBytes + ((fj + r / 2) % 2 ? across ^ 32 : across)) = h[r];
                    }
                }
            wave_lds_fence();
#pragma unroll 4
            for (uint32_t c = lane; c < kImage / 16; c += kLanes)
                *reinterpret_cast<vf4_t*>(begin + plane * o.splane + (c / run) * srow + c % run * 16) = *reinterpret_cast<const vf4_t*>(image + c * 16);
            wave_lds_fence();
        }
    }
}

// Waits for everything that this wave has asked for.
__device__ __forceinline__ void wave_copies_done()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(7 << 4);                     // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

// kGram and kPoly: pairs of tiles (row, col), row <= col, of S = X X^T and of B = b S + c S S; a matrix's inner dimension may be split
// over several blocks, whose sums go to `slots` then.
// kStep and kLast: tiles of a X + B X; the last one goes to the caller's vector.
// `from`: which copy of X is read.  X is scaled up by 2^max(lift - spent, 0) more than usual, and in the next step, where it
// may be larger by 2^growth, by that much less.
template <OrthoProduct P, typename C>
__global__ void __launch_bounds__(C::THREADS, 2)        // (two waves per SIMD: 256 registers)
k_ortho_product(char* __restrict__ scratch, char* __restrict__ slots, const OrthoMatrix* __restrict__ mats, const OrthoTileRef* __restrict__ refs, const OrthoRuns runs,
                int from, int spent, int growth, float ca, float cb, float cc, typename C::Out* __restrict__ out)
{
    constexpr bool kPair = P == kGram || P == kPoly, TR = !kPair, SPLIT = C::SPLIT, kShared = P == kGram || (P == kPoly && SPLIT);
    // An array per stage and operand: the compiler waits for copies to the array that it reads from, not for all of them, and the first
    // operand's four lie within the 64 KB that one address register reaches.
    static_assert(C::B == (SPLIT ? 2 : 4), "");
    __shared__ __attribute__((aligned(1024))) char a0[C::OPERAND], a1[C::OPERAND], a2[C::B > 2 ? C::OPERAND : 16], a3[C::B > 2 ? C::OPERAND : 16];
    __shared__ __attribute__((aligned(1024))) char b0[C::OPERAND], b1[C::OPERAND], b2[C::B > 2 ? C::OPERAND : 16], b3[C::B > 2 ? C::OPERAND : 16];
    uint32_t entry;
    if (!run_entry(runs, blockIdx.x, entry)) return;        // (whole block)
    const OrthoTileRef ref = refs[entry];
    const OrthoMatrix t = mats[ref.matrix];
    const OrthoShape o = ortho_shape(t.rows, t.cols, t.pad);
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int wi = wave / C::WJ, wj = wave % C::WJ;
    char* x = scratch + t.x + (from ? 2 * o.xplane : 0);
    char* s = scratch + t.s;
    char* b = s + 2 * o.splane;
    const float* db = reinterpret_cast<const float*>(b + 2 * o.splane) + o.mp;
    const size_t xrow = static_cast<size_t>(o.np) / kPieceCols * kPieceBytes, srow = static_cast<size_t>(o.mp) / kPieceCols * kPieceBytes;
    constexpr int kRowPieces = C::TILE / kPieceRows, kColPieces = C::TILE / kPieceCols;
    // operands: rows of X twice; rows of S twice; columns of X with rows of B
    const char* pa = P == kGram ? x + ref.row * kRowPieces * xrow : P == kPoly ? s + ref.row * kRowPieces * srow : x + ref.col * (kColPieces * kPieceBytes);
    const char* pb = P == kGram ? x + ref.col * kRowPieces * xrow : P == kPoly ? s + ref.col * kRowPieces * srow : b + ref.row * kRowPieces * srow;
    const size_t plane_a = P == kPoly ? o.splane : o.xplane, plane_b = P == kGram ? o.xplane : o.splane;
    const size_t row_a = P == kPoly ? srow : xrow, row_b = P == kGram ? xrow : srow;
    const int lift = max(t.lift - spent, 0);
    // the part of the inner dimension that this block takes: a multiple of four stages
    const int quarters = (P == kGram ? o.np : o.mp) / 128, splits = kShared ? t.splits[P] : 1;
    const int stage0 = kShared ? quarters * ref.split / splits * 4 : 0, stages = (kShared ? quarters * (ref.split + 1) / splits * 4 : quarters * 4) - stage0;
    auto copy = [&](char* lds_a, char* lds_b, int stage) {
        const int from_stage = stage0 + stage;
        uint32_t mine = lane * 16;
        asm volatile("" : "+v"(mine));                      // (one register beside a scalar address, not an address of two kept for the loop)
        copy_stage<C, TR>(lds_a, pa, plane_a, row_a, from_stage, wave, mine);
        copy_stage<C, false>(lds_b, pb, plane_b, row_b, from_stage, wave, mine);
    };
    acc4_t acc[C::FI][C::FJ];
#pragma unroll
    for (int i = 0; i < C::FI; ++i)
#pragma unroll
        for (int j = 0; j < C::FJ; ++j) acc[i][j] = acc4_t{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kCopies = 2 * C::COPIES;                  // of a stage, per wave
    copy(a0, b0, 0);
    OrthoFragments<C> f, g;
    constexpr int kReads = C::FI * (TR ? 2 : 1) + C::FJ, kProducts = C::FI * C::FJ;
    const LanePlaces first(wi * C::FI * 16, lane), second(wj * C::FJ * 16, lane);
    // At the end every wave has LDS of its own, of all stages: room for images of its part of the tile, of one plane or of two.
    constexpr int kImage = C::FI * C::FJ * 512, kPlanes = C::B * C::STAGE / C::WAVES / kImage, kPerArray = C::OPERAND / kImage;
    static_assert(C::OPERAND % kImage == 0 && (kPlanes == 1 || kPlanes == 2), "");
    static_assert(C::FJ * 16 == kPieceRows && kImage / 1024 % C::COPIES == 0, "a wave's part of X or S is one run of pieces");
    // Behind the last stage come the waves' parts of what the sums are joined with, X or S, into the arrays that their images will
    // have; `n` counts these arrays.
    const auto copy_part = [&](char* array, int n) {
        const int begin = wave * C::COPIES, slot = n * kPerArray + (kPerArray > 1 ? begin / (kImage / 1024) : 0), w = slot / kPlanes, plane = slot % kPlanes;
        const uint32_t row = (kPair ? ref.col : ref.row) * kRowPieces + w % C::WJ;
        const uint32_t piece = (kPair ? ref.row : ref.col) * kColPieces + w / C::WJ * (C::FI * 16 / kPieceCols);
        uint32_t mine = lane * 16;
        asm volatile("" : "+v"(mine));
        const char* at = (kPair ? s + plane * o.splane : x + plane * o.xplane) + row * (kPair ? srow : xrow) + piece * kPieceBytes + (kPerArray > 1 ? begin % (kImage / 1024) : begin) * 1024;
#pragma unroll
        for (int c = 0; c < C::COPIES; ++c)
            __builtin_amdgcn_global_load_lds((global_ptr_t)(at + c * 1024 + mine), (lds_ptr_t)(array + (begin + c) * 1024), 16, 0, 0);
    };
    if constexpr (!SPLIT) {
        // Four stages in turn.  While a stage is multiplied the fragments of the next one are read and the copies of the two or
        // three after it are under way.
        copy(a1, b1, 1);
        copy(a2, b2, 2);
        copy(a3, b3, 3);
        stage_barrier<3 * kCopies>();
        read_first<C, TR>(a0, first, f);
        read_second<C>(b0, second, f);
        const auto read_next = [&](OrthoFragments<C>& next, const char* ready_a, const char* ready_b) {
            read_first<C, TR>(ready_a, first.fresh<TR>(), next);
            read_second<C>(ready_b, second.fresh<false>(), next);
        };
        const auto step = [&](OrthoFragments<C>& now, OrthoFragments<C>& next, char* free_a, char* free_b, const char* ready_a,
                              const char* ready_b, int stage) {
            stage_barrier<2 * kCopies>();                   // what is ready has arrived; everybody has read what is free
            copy(free_a, free_b, stage);
            read_next(next, ready_a, ready_b);
            multiply<C>(now.a, now.b, acc);
            spread_reads<kReads, kProducts / kReads>();
            __builtin_amdgcn_sched_barrier(0);
        };
        // One of the last four.  (Of two planes of S the upper one is all there is.)
        const auto last_step = [&](OrthoFragments<C>& now, OrthoFragments<C>& next, char* free_a, char* free_b, const char* ready_a,
                                   const char* ready_b, auto step_number) {
            constexpr int t = decltype(step_number)::value;
            constexpr auto parts = [](int step) { return P != kGram && (P != kPoly || kPlanes == 1 || step % 2 == 0); };
            constexpr int since = t == 0 ? 2 : t == 1 ? 1 + parts(0) : t == 2 ? parts(0) + parts(1) : 2;   // behind the stage that is read now
            if (t < 3 || parts(3)) stage_barrier<since * kCopies>();
            if constexpr (parts(t)) {
                copy_part(free_a, t);
                copy_part(free_b, t + 4);
            }
            if (t < 3) read_next(next, ready_a, ready_b);
            multiply<C>(now.a, now.b, acc);
            if (t < 3) spread_reads<kReads, kProducts / kReads>();
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int stage = 0; stage < stages - 4; stage += 4) {
            step(f, g, a0, b0, a1, b1, stage + 4);
            step(g, f, a1, b1, a2, b2, stage + 5);
            step(f, g, a2, b2, a3, b3, stage + 6);
            step(g, f, a3, b3, a0, b0, stage + 7);
        }
        last_step(f, g, a0, b0, a1, b1, std::integral_constant<int, 0>{});
        last_step(g, f, a1, b1, a2, b2, std::integral_constant<int, 1>{});
        last_step(f, g, a2, b2, a3, b3, std::integral_constant<int, 2>{});
        last_step(g, f, a3, b3, a0, b0, std::integral_constant<int, 3>{});
    } else {
        // Two stages in turn.  The lo planes of a stage are read beside hi hi and hi lo; then its LDS is free for the one after the
        // next, and the hi planes of the next are read beside lo hi.
        stage_barrier<0>();
        copy(a1, b1, 1);
        read_first<C, TR>(a0, first, f);
        read_second<C>(b0, second, f);
        const auto step = [&](char* now_a, char* now_b, const char* next_a, const char* next_b, int stage, auto to_go) {
            constexpr int left = decltype(to_go)::value;    // 2: stages enough, 1 and 0: behind this one
            constexpr bool parts = left < 2 && P == kPoly;
            OrthoFragments<C> low;
            int anew = lane;                                // (a dozen instructions a stage instead of registers that are needed)
            asm volatile("" : "+v"(anew));
            const LanePlaces p(wi * C::FI * 16, anew), q(wj * C::FJ * 16, anew);
            read_second<C>(now_b + C::PLANE, q, low);
            multiply<C>(f.a, f.b, acc);
            spread_reads<C::FJ, kProducts / C::FJ>();
            __builtin_amdgcn_sched_barrier(0);
            read_first<C, TR>(now_a + C::PLANE, p, low);
            multiply<C>(f.a, low.b, acc);
            spread_reads<kReads - C::FJ, kProducts / (kReads - C::FJ)>();
            __builtin_amdgcn_sched_barrier(0);
            if (left > 0 || parts) stage_barrier<(left > 0 ? 0 : kCopies)>();   // the next stage has arrived; everybody has read this one
            if (left == 2) copy(now_a, now_b, stage);
            if (parts) {
                copy_part(now_a, 1 - left);
                copy_part(now_b, 3 - left);
            }
            if (left > 0) {
                read_first<C, TR>(next_a, p, f);
                read_second<C>(next_b, q, g);
            }
            multiply<C>(low.a, f.b, acc);
            if (left > 0) spread_reads<kReads, kProducts / kReads>();
            __builtin_amdgcn_sched_barrier(0);
            if (left > 0) {
#pragma unroll
                for (int j = 0; j < C::FJ; ++j) f.b[j] = g.b[j];
            }
        };
        for (int stage = 0; stage < stages - 2; stage += 2) {
            step(a0, b0, a1, b1, stage + 2, std::integral_constant<int, 2>{});
            step(a1, b1, a0, b0, stage + 3, std::integral_constant<int, 2>{});
        }
        step(a0, b0, a1, b1, 0, std::integral_constant<int, 1>{});
        step(a1, b1, a0, b0, 0, std::integral_constant<int, 0>{});
    }
    stage_barrier<0>();                                     // nothing under way any more, LDS free
    char* image[kPlanes];
#pragma unroll
    for (int plane = 0; plane < kPlanes; ++plane) {
        const int slot = wave * kPlanes + plane, n = slot / kPerArray;
        char* array = C::B > 2 ? (n == 0 ? a0 : n == 1 ? a1 : n == 2 ? a2 : n == 3 ? a3 : n == 4 ? b0 : n == 5 ? b1 : n == 6 ? b2 : b3)
                               : (n == 0 ? a0 : n == 1 ? a1 : n == 2 ? b0 : b1);
        image[plane] = array + slot % kPerArray * kImage;
    }
    if constexpr (kPair) {
        if (kShared && splits > 1) {                        // left for k_ortho_join
            const uint32_t pair = ref.col * (ref.col + 1) / 2 + ref.row;
            char* to = slots + (t.slot_first[P] + static_cast<size_t>(pair * splits + ref.split) * (C::TILE * C::TILE / 16384)) * 65536;
            const uint32_t mine = threadIdx.x * sizeof(acc4_t);
#pragma unroll
            for (int fi = 0; fi < C::FI; ++fi) {
#pragma unroll
                for (int fj = 0; fj < C::FJ; ++fj) *reinterpret_cast<acc4_t*>(to + (fi * C::FJ + fj) * C::THREADS * sizeof(acc4_t) + mine) = acc[fi][fj];
                __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
        finish_pair<P, C, SPLIT ? kPlanes : 1>(acc, ref, o, s, lift, ca, cb, cc, image[0], wi, wj, lane);
    } else {
        const OrthoPlaces place(ref.col * C::TILE + wi * C::FI * 16, ref.row * C::TILE + wj * C::FJ * 16, lane);
        const size_t part = (place.j0 / kPieceRows) * xrow + (place.i0 / kPieceCols) * kPieceBytes;
        const float rescale = P == kStep ? ldexpf(1.0f / kBScale, max(lift - growth, 0) - lift) : ldexpf(1.0f / (kXScale * kBScale), -lift);
        if constexpr (!SPLIT) {
            // (a + B's diagonal) X, from both planes.  They come by way of LDS, in whole kilobytes: a lane's halves of chunks, straight
            // from memory, took the units that work out addresses longer than the products took (129 us a step, now 114, Transformer-base).
            float scale[C::FJ];
#pragma unroll
            for (int fj = 0; fj < C::FJ; ++fj) scale[fj] = db[place.j_lane + fj * 16] * kBScale;
#pragma unroll
            for (int turn = 0; turn < 2 / kPlanes; ++turn) {
                if (turn > 0) {                             // (room for one plane: the other one)
#pragma unroll
                    for (int c = 0; c < kImage / 1024; ++c)
                        __builtin_amdgcn_global_load_lds((global_ptr_t)(x + part + o.xplane + c * 1024 + lane * 16),
                                                         (lds_ptr_t)(image[0] + c * 1024), 16, 0, 0);
                    wave_copies_done();
                }
#pragma unroll
                for (int plane = 0; plane < kPlanes; ++plane)
#pragma unroll
                    for (int fj = 0; fj < C::FJ; ++fj)
#pragma unroll
                        for (int fi = 0; fi < C::FI; ++fi) {
                            const half4_t v = *reinterpret_cast<const half4_t*>(image[plane] + place(fi, fj));
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[fi][fj][r] = fmaf(scale[fj], static_cast<float>(v[r]), acc[fi][fj][r]);
                        }
                wave_lds_fence();
            }
        }
        if constexpr (P == kStep) {
            char* next = scratch + t.x + (from ? 0 : 2 * o.xplane) + part;
#pragma unroll
            for (int plane = 0; plane < 2; ++plane) {
#pragma unroll
                for (int fj = 0; fj < C::FJ; ++fj)
#pragma unroll
                    for (int fi = 0; fi < C::FI; ++fi) {
                        half4_t v;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {       // (split_half of acc * rescale, without rounding that product)
                            const _Float16 hi = static_cast<_Float16>(acc[fi][fj][r] * rescale);
                            v[r] = plane == 0 ? hi : static_cast<_Float16>(fmaf(acc[fi][fj][r], rescale, -static_cast<float>(hi)));
                        }
                        *reinterpret_cast<half4_t*>(image[0] + place(fi, fj)) = v;
                    }
                wave_lds_fence();
#pragma unroll
                for (int c = 0; c < kImage / 1024; ++c)
                    *reinterpret_cast<vf4_t*>(next + plane * o.xplane + c * 1024 + lane * 16) = *reinterpret_cast<const vf4_t*>(image[0] + c * 1024 + lane * 16);
                wave_lds_fence();
            }
        } else {
            if constexpr (!SPLIT) {
                if (t.src % kVec == 0 && t.stride % kVec == 0) {
                    // Whole lines of the caller's rows, by way of LDS: rows of units of four values, permuted so that writes down a column of
                    // units meet in no bank.  (us a call, four values a lane straight to memory / so: Transformer-base 1009 / 977, 16384 x 4096
                    // 4434 / 4397.)
                    const uint32_t shift = o.tall ? 4 : C::FI == 8 ? 5 : 4, pitch = 8u << shift;
#pragma unroll
                    for (int fj = 0; fj < C::FJ; ++fj)
#pragma unroll
                        for (int fi = 0; fi < C::FI; ++fi) {
                            const acc4_t v = acc[fi][fj] * rescale;
                            const uint32_t i = fi * 16 + lane / 16 * 4, j = fj * 16 + lane % 16;
                            if (!o.tall) {
                                *reinterpret_cast<vu2_t*>(image[0] + j * pitch + ((i / 4 ^ j % 16) << 3)) =
                                    vu2_t{bf16_bits(v[0]) | static_cast<uint32_t>(bf16_bits(v[1])) << 16, bf16_bits(v[2]) | static_cast<uint32_t>(bf16_bits(v[3])) << 16};
                            } else {
#pragma unroll
                                for (uint32_t r = 0; r < 4; ++r)
                                    *reinterpret_cast<uint16_t*>(image[0] + (i + r) * pitch + ((j / 4 ^ (i + r) % 16) << 3) + j % 4 * 2) = bf16_bits(v[r]);
                            }
                        }
                    wave_lds_fence();
                    const uint32_t row0 = o.tall ? place.i0 : place.j0, col0 = o.tall ? place.j0 : place.i0;
#pragma unroll 4
                    for (uint32_t c = lane; c < kImage / 8; c += kLanes) {
                        const uint32_t row = c >> shift, unit = c & ((1u << shift) - 1), col = col0 + unit * 4;
                        const vu2_t v = *reinterpret_cast<const vu2_t*>(image[0] + row * pitch + ((unit ^ row % 16) << 3));
                        if (row0 + row >= static_cast<uint32_t>(t.rows)) continue;
                        uint16_t* to = out + t.src + static_cast<int64_t>(row0 + row) * t.stride + col;
                        if (col + 3 < static_cast<uint32_t>(t.cols)) {
                            __builtin_nontemporal_store(v, reinterpret_cast<vu2_t*>(to));
                        } else {
#pragma unroll
                            for (uint32_t e = 0; e < 4; ++e)
                                if (col + e < static_cast<uint32_t>(t.cols)) to[e] = static_cast<uint16_t>(v[e / 2] >> e % 2 * 16);
                        }
                    }
                    return;
                }
            }
            const bool wide = SPLIT && !o.tall && t.src % 4 == 0 && t.stride % 4 == 0;    // four columns of `out` are one access
#pragma unroll
            for (int fj = 0; fj < C::FJ; ++fj) {
                const uint32_t j = place.j_lane + fj * 16;  // row of X
                if (j >= static_cast<uint32_t>(o.m)) continue;
#pragma unroll
                for (int fi = 0; fi < C::FI; ++fi) {
                    const uint32_t i = place.i_lane + fi * 16;   // first of four columns
                    const acc4_t v = acc[fi][fj] * rescale;
                    if (wide && i + 3 < static_cast<uint32_t>(o.n)) {
                        store4(out + t.src + static_cast<int64_t>(j) * t.stride + i, make_float4(v[0], v[1], v[2], v[3]));
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (i + r < static_cast<uint32_t>(o.n))
                                put(out + (o.tall ? t.src + static_cast<int64_t>(i + r) * t.stride + j : t.src + static_cast<int64_t>(j) * t.stride + i + r), v[r]);
                    }
                }
            }
        }
    }
}

// Adds the sums of a pair's blocks up, in their order, and finishes the pair; a wave's part of a tile per block.  Four waves share the sums, so
// that the parts of four blocks are on their way at once, and one of them finishes.
template <OrthoProduct P, typename C>
__global__ void __launch_bounds__(kBlock)
k_ortho_join(char* __restrict__ scratch, const char* __restrict__ slots, const OrthoMatrix* __restrict__ mats, const OrthoTileRef* __restrict__ refs,
             int spent, float ca, float cb, float cc)
{
    constexpr int kFragments = C::FI * C::FJ, kEach = kFragments / kWaves, kTogether = 4;
    __shared__ __attribute__((aligned(1024))) char image[kFragments * 512];
    __shared__ acc4_t sums[kFragments][kLanes];
    const OrthoTileRef ref = refs[blockIdx.x / C::WAVES];
    const OrthoMatrix t = mats[ref.matrix];
    const int lane = threadIdx.x % kLanes, part = blockIdx.x % C::WAVES, share = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const uint32_t pair = ref.col * (ref.col + 1) / 2 + ref.row;
    const int splits = t.splits[P];
    constexpr size_t kSlot = C::TILE * C::TILE * sizeof(float), kRow = C::THREADS * sizeof(acc4_t);
    const char* from = slots + static_cast<size_t>(t.slot_first[P]) * 65536 + static_cast<size_t>(pair) * splits * kSlot + share * kEach * kRow;
    const uint32_t mine = (part * kLanes + lane) * sizeof(acc4_t);
    acc4_t v[kEach];
#pragma unroll
    for (int f = 0; f < kEach; ++f) v[f] = *reinterpret_cast<const acc4_t*>(from + f * kRow + mine);
    for (int split = 1; split < splits; split += kTogether) {
        acc4_t w[kTogether][kEach];
#pragma unroll
        for (int k = 0; k < kTogether; ++k)
#pragma unroll
            for (int f = 0; f < kEach; ++f)                 // (past the last one the last one again, not added)
                w[k][f] = *reinterpret_cast<const acc4_t*>(from + min(split + k, splits - 1) * kSlot + f * kRow + mine);
#pragma unroll
        for (int k = 0; k < kTogether; ++k)
            if (split + k < splits)
#pragma unroll
                for (int f = 0; f < kEach; ++f) v[f] += w[k][f];
    }
#pragma unroll
    for (int f = 0; f < kEach; ++f) sums[share * kEach + f][lane] = v[f];
    __syncthreads();
    if (share > 0) return;                                  // (whole waves, nothing is awaited any more)
    acc4_t acc[C::FI][C::FJ];
#pragma unroll
    for (int fi = 0; fi < C::FI; ++fi)
#pragma unroll
        for (int fj = 0; fj < C::FJ; ++fj) acc[fi][fj] = sums[fi * C::FJ + fj][lane];
    const OrthoShape o = ortho_shape(t.rows, t.cols, t.pad);
    finish_pair<P, C, 0>(acc, ref, o, scratch + t.s, max(t.lift - spent, 0), ca, cb, cc, image, part / C::WJ, part % C::WJ, lane);
}

}  // namespace
