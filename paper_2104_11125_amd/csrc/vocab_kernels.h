// Kernels of the losses over a vocabulary: softmax cross entropy and distillation from a teacher's listed logits, from the
// last hidden states x (T x D) and the output matrix w (V x D), with their gradients.  Part of scalecom.hip's single
// translation unit.
//
//   z = x w^T / tau                               T x V, never held as a whole
//   lse_t = log sum_v exp z_tv
//   cross entropy (tau = 1):  loss_t = lse_t - z_t,y = softplus(log sum_{v != y} exp z_tv - z_ty)
//   distillation:             loss_t = tau^2 sum_j q_tj (log q_tj - z_t,i(j) + lse_t),  q the teacher's softmax over its list
//   dz = c_t (exp(z_tv - lse_t) - target_tv)      of a piece of the vocabulary at a time
//   dx = dz w,   dw = dz^T x
//
// Rows without a target are left out: k_vocab_rows copies the others, one behind the other, so they cost nothing and what they
// hold (NaN too) reaches no product.
//
// Numbers.  The products run on the matrix units with bfloat16 operands and binary32 sums.  A binary32 operand is held as three
// bfloat16 planes, hi + mid + lo, 24 bits and binary32's range, and a product is six products of planes (the dropped ones are at most
// 2^-23 of it, mostly a few 2^-27); a plane pair is a segment of a longer inner dimension, so one loop serves all types.  dz, in binary32, is
// held in two planes for gradients in bfloat16 and in three for binary32 ones.  With one plane less every term is rounded a second time, which few
// tokens, or tokens that all count the same, do not average out: 12 of 150 calls of random sizes then had a bfloat16 gradient more than 1.5 times as far from the
// exact one as products in binary32 are (up to 2.6 times, with 344 tokens 1.8); so none of 300 has.  (8192 x 131072 x 4096, loss and gradient: 35.0 ms instead of 24.0;
// 4096 x 32768 x 512, dw in binary32, 0.90 instead of 0.83.)  A binary32 dw of bfloat16 operands with two planes, a third less work in dw, was three times as far.
//
// What bounds it: the matrix units and their power, and what a tile takes at its end.  7168 x 131072 x 4096 (bf16): sums 6.1 ms (1.26 PFLOP/s), dz 6.5, dx 11.6 (two
// products, 1.33), dw 10.8 (two, 1.43; a large product of the library 1.45), matrix units busy 68, 63, 80 and 76 % of the CUs' time at some 1.75 GHz; no bank conflicts; every
// line of an operand asked for once a tile; the ends of large tiles of dx and dw keep 170 to 210 bytes a lane in scratch memory.  With 512 places of the inner dimension a tile's 16 stages take 11 us and the exponentials behind them half as long:
// sums of 3584 x 32768 x 512 159 us (0.76 PFLOP/s).  Few tokens: w's bytes and three launches (8 x 32768 x 512: 18 us, of which the sums 8).
#pragma once

#include <hip/hip_runtime.h>

#include "device_helpers.h"
#include "embed_kernels.h"
#include "geometry.h"
#include "optimizer_kernels.h"
#include "orthogonalize_kernels.h"

namespace {

typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));

constexpr int kVocabStage = 32;                             // places of the inner dimension that a stage holds
constexpr int kVocabQuarter = 4 * kVocabStage;              // inner dimensions are padded to multiples of it
constexpr int kVocabPad = 32;                               // columns behind the rows of planes, so that their blocks do not all begin on one memory channel
constexpr int kVocabPieceMax = 1 << 18, kVocabPieceLeast = 2048;
static_assert((kVocabPieceMax + kVocabPad) * 32 < 1 << 24 && (SCALECOM_DIM_MAX + kVocabQuarter + kVocabPad) * 32 < 1 << 24, "rows times a pitch, in 24 bits");
constexpr int kVocabPieceRows = 256;                        // pieces of the vocabulary are multiples of it

// The operands' plane pairs, one nibble per segment (first operand's plane, then the second's, two bits each), the smallest first: a sum is rounded at
// every addition, and only hi times hi, last, adds to large ones.
struct VocabSegments {
    uint32_t pairs;
    int32_t n;
};
constexpr VocabSegments kOnePlane{0x0, 1}, kSecondInTwo{0x04, 2}, kSecondInThree{0x048, 3}, kThreeOfNine{0x014, 3}, kSixOfNine{0x014582, 6};

// An operand: planes `plane` bytes apart, of `rows` rows and `cols` columns.  Its tile is of rows (inner dimension along a row), or, TR, of
// columns (inner dimension across rows).  As the caller's matrix lies: rows of `pitch` bytes; places behind its rows or columns are never read: the
// last one stands in.  Blocked, as this file lays out what it makes itself: blocks of 16 rows, `pitch` bytes each, in which 32 columns
// of all 16 rows are a kilobyte (rows are padded to whole tiles, and zeros are there), so a copy to LDS takes whole lines whichever way the operand is read.
struct VocabOperand {
    const char* at;
    int64_t plane;
    uint32_t pitch;
    int32_t rows, cols;
};
__device__ __forceinline__ int64_t blocked(int64_t row, int64_t col, uint32_t pitch)
{
    return row / 16 * pitch + col / 32 * 1024 + row % 16 * 64 + col % 32 * 2;
}

// A block of WI x WJ waves computes a tile of TI x TJ, every wave FI x FJ products of 16 x 16 x 32.
template <int WI_, int WJ_, int FI_, int FJ_>
struct VocabConfig {
    static constexpr int WI = WI_, WJ = WJ_, FI = FI_, FJ = FJ_;
    static constexpr int TI = WI * FI * 16, TJ = WJ * FJ * 16;
    static constexpr int WAVES = WI * WJ, THREADS = WAVES * kLanes;
    static constexpr int A = TI * kVocabStage * 2, B = TJ * kVocabStage * 2;    // bytes of an operand's stage
    static constexpr int COPIES_A = A / 1024 / WAVES, COPIES_B = B / 1024 / WAVES, COPIES = COPIES_A + COPIES_B;
    static_assert(A % (1024 * WAVES) == 0 && B % (1024 * WAVES) == 0, "");
    static constexpr bool WIDE = FI * FJ > 32;              // sums in accumulation registers of their own, one wave per SIMD
    static constexpr int PER_SIMD = WIDE ? 1 : 2;
    static_assert((FI & (FI - 1)) == 0 && (FJ & (FJ - 1)) == 0 && FI <= 8 && FJ <= 8, "");
};
using VocabLarge = VocabConfig<2, 2, 8, 8>;                 // 256 x 256, one block of 4 waves per CU
using VocabMedium = VocabConfig<2, 2, 4, 4>;                // 128 x 128, two of 4 waves
using VocabThin = VocabConfig<4, 1, 2, 4>;                  // 128 x 64, three of 4 waves: few tokens

// In LDS a stage of an operand with rows of 64 bytes (four chunks of 16; two stages: 128, eight) holds chunk c of row r in place c ^ row_swizzle(r), one with
// columns (TR: 32 rows of TILE elements) the 16 columns u of row r in place u ^ column_swizzle(r), so that the lanes that read at
// once meet in no bank.
__device__ __forceinline__ uint32_t row_swizzle(uint32_t r) { return (r >> 2) & 2u; }
__device__ __forceinline__ uint32_t pair_swizzle(uint32_t r) { return (r >> 1) & 7u; }      // of two stages: rows of 128 bytes
__device__ __forceinline__ uint32_t column_swizzle(uint32_t r) { return (r & 3u) | ((r >> 1) & 4u); }

// What a wave copies of an operand: a lane's 16 bytes of every kilobyte that the wave takes, at an offset of 32 bits beside a scalar address.
template <int TILE, int COPIES, int WAVES, bool TR, bool BLOCKED>
struct VocabCopies {
    static constexpr int kChunks = TILE / 8;                // TR: of 16 bytes in a row
    static constexpr int kStep = WAVES * kLanes / kChunks;  // TR: rows from one of the wave's kilobytes to the next
    static constexpr bool kOne = TR && kStep % 16 == 0;     // the swizzle is the same in all of them
    uint32_t at[kOne ? 1 : COPIES];                         // !TR: from the tile's first row; TR: of the column
    int32_t row;                                            // TR: of the first kilobyte
    __device__ __forceinline__ VocabCopies(const VocabOperand& o, int first, int wave, int lane)
    {
        row = (wave * kLanes + lane) / kChunks;
#pragma unroll
        for (int i = 0; i < (kOne ? 1 : COPIES); ++i) {
            if (TR) {
                const int chunk = min(first / 8 + ((lane % kChunks) ^ static_cast<int>(column_swizzle(row + i * kStep) << 1)), o.cols / 8 - 1);
                at[i] = BLOCKED ? static_cast<uint32_t>(chunk / 4 * 1024 + chunk % 4 * 16) : static_cast<uint32_t>(chunk) * 16;
                continue;
            }
            if (BLOCKED) {
                at[i] = static_cast<uint32_t>(i * WAVES + wave) * o.pitch + lane / 4 * 64 + ((lane % 4) ^ row_swizzle(lane / 4)) * 16;
            } else {                                        // two stages at once: eight rows of 128 bytes
                const int r = (i * WAVES + wave) * 8 + lane / 8;
                at[i] = static_cast<uint32_t>(min(r, o.rows - 1 - first)) * o.pitch + ((lane % 8) ^ pair_swizzle(r)) * 16;
            }
        }
    }
    // Where four stages from stage `stage` on begin, of the tile with the first row or column `first`.
    __device__ __forceinline__ static const char* begin(const VocabOperand& o, int plane, int first, int stage)
    {
        const char* p = o.at + plane * o.plane;
        if (TR) return p + static_cast<int64_t>(stage) * (BLOCKED ? kVocabStage / 16 : kVocabStage) * o.pitch;
        return BLOCKED ? p + static_cast<int64_t>(first / 16) * o.pitch + stage * 1024 : p + static_cast<int64_t>(first) * o.pitch + stage * 64;
    }
    // One of the wave's kilobytes of one of the four stages behind `base`; TR, not blocked: the operand's last row is `last` rows behind it.
    template <int K>
    __device__ __forceinline__ void copy(char* lds, const char* base, uint32_t pitch, int last, int wave, int i) const
    {
        uint32_t mine = at[kOne ? 0 : i];
        if (!TR) {
            mine += K * (BLOCKED ? 1024 : 64);
        } else if (BLOCKED) {
            const uint32_t r = row + i * kStep;
            mine += __umul24(r / 16 + K * (kVocabStage / 16), pitch) + r % 16 * 64;
        } else {
            mine += __umul24(static_cast<uint32_t>(min(row + i * kStep + K * kVocabStage, last)), pitch);
        }
        asm volatile("" : "+v"(mine));                      // (beside the scalar address, not an address of two registers kept for the loop)
        __builtin_amdgcn_global_load_lds((global_ptr_t)(base + mine), (lds_ptr_t)(lds + (i * WAVES + wave) * 1024), 16, 0, 0);
    }
};

// Where a lane reads in a stage: a fragment of 16 rows takes 8 values along the inner dimension; one of 16 columns (TR) four, and four of the
// rows that follow.
// PAIRED: rows of two stages; the second one's chunks are 64 bytes on, as far as the swizzle goes.
template <int TILE, bool TR, bool PAIRED>
struct VocabReads {
    uint32_t at;
    __device__ __forceinline__ VocabReads(int first, int lane)
    {
        if (PAIRED) {
            at = (first + lane % 16) * 128 + ((lane / 16) ^ pair_swizzle(lane % 16)) * 16;
        } else if (!TR) {
            at = (first + lane % 16) * 64 + ((lane / 16) ^ row_swizzle(lane % 16)) * 16;
        } else {
            const uint32_t r = lane / 16 * 8 + lane % 16 / 4;
            at = r * (TILE * 2) + ((first / 16) ^ column_swizzle(r)) * 32 + lane % 4 * 8;
        }
    }
    // Where fragment 0 is, in the second of two stages or else.  (One register, not one for every fragment and stage.)
    __device__ __forceinline__ uint32_t here(bool second) const
    {
        uint32_t mine = PAIRED && second ? at ^ 64u : at;
        asm volatile("" : "+v"(mine));
        return mine;
    }
    __device__ __forceinline__ static bf8_t fragment(const char* lds, uint32_t from, int i)
    {
        if (!TR) return *reinterpret_cast<const bf8_t*>(lds + from + i * (PAIRED ? 2048 : 1024));
        const char* p = lds + (from ^ (i * 32));
        return __builtin_bit_cast(bf8_t, __builtin_shufflevector(read_columns(p), read_columns(p + 4 * TILE * 2), 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // Fragments [FIRST, FIRST + N) of the wave's part.
    template <int FIRST, int N>
    __device__ __forceinline__ void read(const char* lds, bool second, bf8_t (&f)[N]) const
    {
        const uint32_t from = here(second);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = fragment(lds, from, FIRST + i);
    }
};

// The order of a half stage's instructions: products first, then reads of LDS between them (two at a time where there are many), then copies.
template <int PRODUCTS, int READS, int COPIES>
__device__ __forceinline__ void order()
{
    constexpr int kAtOnce = 2 * READS > PRODUCTS ? 2 : 1, kFirst = PRODUCTS >= 16 ? 2 : 1;    // (few products: what is left over follows)
    __builtin_amdgcn_sched_group_barrier(0x008, kFirst, 0);
#pragma unroll
    for (int i = 0; i < READS / kAtOnce; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, kAtOnce, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS, 0);
    __builtin_amdgcn_sched_barrier(0);
}

// The tiles of a launch, n_i x n_j of them, `splits` times: tile number e, and its part of the inner dimension, which is `quarters` times four
// stages long over all segments.  They are numbered in groups of four along j, so that the 32 blocks that an XCD runs at once
// share rows of both operands.
struct VocabTiles {
    uint32_t n_i, n_j, splits;
    int32_t quarters;
    __device__ __forceinline__ uint32_t all() const { return n_i * n_j * splits; }
};
struct VocabTile {
    int i, j, split, stage0, stages;
    __device__ __forceinline__ VocabTile(const VocabTiles& t, uint32_t e)
    {
        const uint32_t per = t.n_i * t.n_j, rest = e % per;
        split = static_cast<int>(e / per);
        const uint32_t group = rest / (4 * t.n_i), width = min(4u, t.n_j - group * 4), in = rest - group * 4 * t.n_i;
        i = static_cast<int>(in / width);
        j = static_cast<int>(group * 4 + in % width);
        stage0 = static_cast<int>(static_cast<int64_t>(t.quarters) * split / t.splits) * 4;
        stages = static_cast<int>(static_cast<int64_t>(t.quarters) * (split + 1) / t.splits) * 4 - stage0;
    }
};

// What a block does: an eighth of consecutive tiles for every XCD (blocks go to the XCDs in turn), of these every so many-th.  For each, sums over the
// inner dimension (segments of `per_segment` stages one behind the other; the tile's stages, a multiple of four and four at least) and
// finish(tile, acc).  Four stages are in LDS in turn: while one is multiplied the copies of the two or three after it are under way, and those behind a
// tile's last one are the next tile's first, so neither a block's start nor the end of a tile leaves the memory idle.
template <typename C, bool TRA, bool TRB, bool BLOCKED_A, bool BLOCKED_B, typename Finish>
__device__ __forceinline__ void vocab_products(const VocabOperand& a, const VocabOperand& b, const VocabSegments& seg, const VocabTiles& tiles, int per_segment,
                                               int wave, int lane, const Finish& finish)
{
    // The caller's matrix along its rows comes in pairs of stages, 128 bytes of a row, a whole line; what is free is asked for at once where a stage is
    // odd.  (One stage at a time, every line twice: dz of 7168 x 131072 x 4096 took 6.47 ms instead of 6.15.)
    constexpr bool PAIRED = !TRA && !BLOCKED_A;
    constexpr int kFirstA = PAIRED ? 2 * C::A : C::A, kSecondA = PAIRED ? 16 : C::A, kCopiesA = PAIRED ? 2 * C::COPIES_A : C::COPIES_A;
    __shared__ __attribute__((aligned(1024))) char a0[kFirstA], a1[kSecondA], a2[kFirstA], a3[kSecondA];
    __shared__ __attribute__((aligned(1024))) char b0[C::B], b1[C::B], b2[C::B], b3[C::B];
    const uint32_t xcd = blockIdx.x % kXcds, every = gridDim.x / kXcds;             // (the grid is a multiple of kXcds)
    const uint64_t all = tiles.all();
    const uint32_t end = static_cast<uint32_t>(all * (xcd + 1) / kXcds);
    uint32_t e = static_cast<uint32_t>(all * xcd / kXcds) + blockIdx.x / kXcds;
    if (e >= end) return;                                   // (whole block)
    const int wi = wave / C::WJ, wj = wave % C::WJ;
    const VocabReads<C::TI, TRA, PAIRED> ra(wi * C::FI * 16, lane);
    const VocabReads<C::TJ, TRB, false> rb(wj * C::FJ * 16, lane);
    // Where the next copies come from, four stages at a time.
    using CopiesA = VocabCopies<C::TI, kCopiesA, C::WAVES, TRA, BLOCKED_A>;
    static_assert(TRB || BLOCKED_B, "");
    using CopiesB = VocabCopies<C::TJ, C::COPIES_B, C::WAVES, TRB, BLOCKED_B>;
    VocabTile ahead(tiles, e);
    CopiesA ca(a, ahead.i * C::TI, wave, lane);
    CopiesB cb(b, ahead.j * C::TJ, wave, lane);
    int segment = ahead.stage0 / per_segment, at = ahead.stage0 % per_segment, left = ahead.stages, last_a = 0, last_b = 0;
    const char *from_a = nullptr, *from_b = nullptr;
    const auto four_stages = [&]() {
        if (left == 0) {                                    // the next tile; behind the last one its stages once more
            e += every;
            if (e < end) ahead = VocabTile(tiles, e);
            ca = CopiesA(a, ahead.i * C::TI, wave, lane);
            cb = CopiesB(b, ahead.j * C::TJ, wave, lane);
            segment = ahead.stage0 / per_segment;
            at = ahead.stage0 % per_segment;
            left = ahead.stages;
        } else if (at == per_segment) {
            at = 0;
            ++segment;
        }
        const uint32_t pair = seg.pairs >> (segment * 4);
        from_a = CopiesA::begin(a, pair & 3u, ahead.i * C::TI, at);
        from_b = CopiesB::begin(b, pair >> 2 & 3u, ahead.j * C::TJ, at);
        last_a = a.rows - 1 - at * kVocabStage;
        last_b = b.rows - 1 - at * kVocabStage;
        at += 4;
        left -= 4;
    };
    // Copies of a step: of the first operand (PAIRED: of both its stages where k is odd), then of the second.
    const auto copy_one = [&](char* lds_a, char* lds_b, auto k, int i) {
        constexpr int kOfA = PAIRED ? decltype(k)::value % 2 * kCopiesA : kCopiesA;
        if (i < kOfA)
            ca.template copy<PAIRED ? decltype(k)::value / 2 * 2 : decltype(k)::value>(lds_a, from_a, a.pitch, last_a, wave, i);
        else
            cb.template copy<decltype(k)::value>(lds_b, from_b, b.pitch, last_b, wave, i - kOfA);
    };
    // A stage is multiplied in two halves of the first operand's fragments.  Beside the first half the other half's fragments are read, beside
    // the second the next stage's first half and its second operand: 64 registers of fragments, where two whole stages' were
    // 96 and the transposing reads' addresses went to scratch memory (k_vocab_dx 2.4 ms instead of 0.8 for 7168 x 16384 x 4096).
    constexpr int H = C::FI / 2, kProducts = H * C::FJ, kReadsA = H * (TRA ? 2 : 1), kReadsB = C::FJ * (TRB ? 2 : 1);
    acc4_t acc[C::FI][C::FJ];
    bf8_t low[H], high[H], even[C::FJ], odd[C::FJ];
    const auto multiply = [&](const bf8_t (&fa)[H], const bf8_t (&fb)[C::FJ], auto first) {
        constexpr int i0 = decltype(first)::value;
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int j = 0; j < C::FJ; ++j) acc[i0 + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[j], acc[i0 + i][j], 0, 0, 0);
    };
    // WIDE: 256 sums a lane have to stay in the accumulation registers, where the compiler does not leave them by itself (it moves them to others
    // and back in every turn), so the instruction is written out, in the order of the source.  What the compiler then cannot know, the
    // waits between these instructions and others that touch the sums, settle() provides at either end of a tile.  (Their operands come straight from
    // reads of LDS, which it does wait for; two idle cycles before each product, for a move that it might put there and does not, cost 7 %.  That no move
    // is there, and that the waits are long enough, is looked for in the built code: tests/test_matrix_waits.py.)
    const auto product = [](acc4_t& sum, const bf8_t& x, const bf8_t& y) {
        typedef int int4_t __attribute__((ext_vector_type(4)));
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(sum) : "v"(__builtin_bit_cast(int4_t, x)), "v"(__builtin_bit_cast(int4_t, y)));
    };
    const auto settle = [&]() {
        if constexpr (C::WIDE) {
#pragma unroll
            for (int i = 0; i < C::FI; ++i)
#pragma unroll
                for (int j = 0; j < C::FJ; j += 8)
                    asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[i][j]), "+a"(acc[i][j + 1]), "+a"(acc[i][j + 2]), "+a"(acc[i][j + 3]), "+a"(acc[i][j + 4]),
                                 "+a"(acc[i][j + 5]), "+a"(acc[i][j + 6]), "+a"(acc[i][j + 7]));
        }
    };
    // The stage in (now_a, now_b), whose second operand is in `fb`; the next one in (next_a, next_b).  The order of instructions is given: a
    // half begins with products whose operands have been read, and what is read or asked for comes well before its end.
    const auto step = [&](char* now_a, char* now_b, const char* next_a, const char* next_b, bf8_t (&fb)[C::FJ], bf8_t (&next_fb)[C::FJ], auto k) {
        constexpr bool kOdd = decltype(k)::value % 2 != 0;
        constexpr int kCopies = (!PAIRED || kOdd ? kCopiesA : 0) + C::COPIES_B;
        // What may be under way when the next stage has arrived, the last copies asked for: of two stages.  PAIRED, k even: those of the second operand
        // behind the next stage's, and the pair behind it; k odd: the pair that is needed came before them.
        constexpr int kUnderWay = !PAIRED ? 2 * C::COPIES : kOdd ? 2 * C::COPIES_B : 2 * C::COPIES_B + kCopiesA;
        if constexpr (C::WIDE) {
            uint32_t from = ra.here(kOdd);
#pragma unroll
            for (int p = 0; p < kProducts; ++p) {
                product(acc[p / C::FJ][p % C::FJ], low[p / C::FJ], fb[p % C::FJ]);
                if (p % 4 == 1 && p / 4 < H) high[p / 4] = ra.fragment(now_a, from, H + p / 4);
                __builtin_amdgcn_sched_barrier(0);
            }
            stage_barrier<kUnderWay>();
            from = ra.here(!kOdd);
            const uint32_t from_b = rb.here(false);
#pragma unroll
            for (int p = 0; p < kProducts; ++p) {
                product(acc[H + p / C::FJ][p % C::FJ], high[p / C::FJ], fb[p % C::FJ]);
                constexpr int kFragments = H + C::FJ;       // one behind every other product
                if (p % 2 == 1 && p / 2 < C::FJ) next_fb[p / 2] = rb.fragment(next_b, from_b, p / 2);
                if (p % 2 == 1 && p / 2 >= C::FJ && p / 2 < kFragments) low[p / 2 - C::FJ] = ra.fragment(next_a, from, p / 2 - C::FJ);
                if (p % 2 == 0 && p >= 2 && p / 2 - 1 < kCopies) copy_one(now_a, now_b, k, p / 2 - 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
        ra.template read<H>(now_a, kOdd, high);
        multiply(low, fb, std::integral_constant<int, 0>{});
        order<kProducts, kReadsA, 0>();
        stage_barrier<kUnderWay>();                         // the next stage has arrived; everybody has read this one
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_one(now_a, now_b, k, i);
        rb.template read<0>(next_b, false, next_fb);
        ra.template read<0>(next_a, !kOdd, low);
        multiply(high, fb, std::integral_constant<int, H>{});
        order<kProducts, kReadsA + kReadsB, kCopies>();
    };
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    constexpr std::integral_constant<int, 2> k2{};
    constexpr std::integral_constant<int, 3> k3{};
    four_stages();
    const auto copies = [&](char* lds_a, char* lds_b, auto k, int from, int to) {
#pragma unroll
        for (int i = 0; i < kCopiesA + C::COPIES_B; ++i)
            if (i >= from && i < to) copy_one(lds_a, lds_b, k, i);
    };
    if constexpr (PAIRED) {                                 // the pairs before the second operand's stages that they go with
        copies(a0, b1, k1, 0, kCopiesA);
        copies(a0, b0, k0, 0, C::COPIES_B);
        copies(a0, b1, k1, kCopiesA, kCopiesA + C::COPIES_B);
        copies(a2, b3, k3, 0, kCopiesA);
        copies(a2, b2, k2, 0, C::COPIES_B);
        copies(a2, b3, k3, kCopiesA, kCopiesA + C::COPIES_B);
        stage_barrier<3 * C::COPIES_B + kCopiesA>();
    } else {
        copies(a0, b0, k0, 0, C::COPIES);
        copies(a1, b1, k1, 0, C::COPIES);
        copies(a2, b2, k2, 0, C::COPIES);
        copies(a3, b3, k3, 0, C::COPIES);
        stage_barrier<3 * C::COPIES>();
    }
    ra.template read<0>(a0, false, low);
    rb.template read<0>(b0, false, even);
    // PAIRED: a0 holds the stages 0 and 1, a2 the others
    char* const second_a = PAIRED ? a0 : a1;
    char* const fourth_a = PAIRED ? a2 : a3;
    while (true) {
        const VocabTile tile = ahead;
#pragma unroll
        for (int i = 0; i < C::FI; ++i)
#pragma unroll
            for (int j = 0; j < C::FJ; ++j) acc[i][j] = acc4_t{0.0f, 0.0f, 0.0f, 0.0f};
        settle();
        for (int stage = 0; stage < tile.stages; stage += 4) {
            four_stages();
            step(a0, b0, second_a, b1, even, odd, k0);
            step(second_a, b1, a2, b2, odd, even, k1);
            step(a2, b2, fourth_a, b3, even, odd, k2);
            step(fourth_a, b3, a0, b0, odd, even, k3);
        }
        settle();
        finish(tile, acc);
        if (e >= end) break;
    }
    stage_barrier<0>();                                     // (nothing arrives in LDS behind the block's end)
}

// What the kernels know of the rows that take part.
struct VocabRow {
    float lse, factor, target_dz;                           // of the gradient: c_t, and what dz is at the target (cross entropy)
    int32_t target;                                         // -1: none (distillation)
};

typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
typedef float f2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t two_bf16(float a, float b)      // rounded to nearest even, one instruction
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2_t{a, b}, bf2_t));
}

// Four values to consecutive places of every plane: hi, mid, lo.  WIDE: also for values whose hi is infinite; mid and lo are zero then.
template <int PLANES, bool WIDE>
__device__ __forceinline__ void store_planes4(char* at, int64_t plane, const float* v)
{
    float rest[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
        uint2 w;
        w.x = two_bf16(rest[0], rest[1]);
        w.y = two_bf16(rest[2], rest[3]);
        *reinterpret_cast<uint2*>(at + p * plane) = w;
        if (p + 1 == PLANES) break;
        const float hi[4] = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
#pragma unroll
        for (int c = 0; c < 4; ++c) rest[c] = !WIDE || fabsf(hi[c]) < __builtin_huge_valf() ? rest[c] - hi[c] : 0.0f;
    }
}

// Four consecutive elements of a row from column `col` on, zeros behind its end.
template <typename T>
__device__ __forceinline__ void four_of(const T* row, int64_t col, int64_t cols, float* v)
{
    T e[4];
    load_row(row + col, static_cast<int>(min(cols - col, int64_t{4})), e);
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = widen(e[c]);
}

struct VocabRowsArgs {
    const int32_t* targets;                                 // one per token; out of [0, vocab): no part
    int32_t n, padded, vocab, dim, dim_padded;
    uint32_t pitch;                                         // of the planes' blocks
    int64_t stride;
    int32_t one_target;                                     // cross entropy; otherwise distillation, and `targets` says who takes part
    const float *loss, *lse, *dloss;                        // of the gradient, or NULL
    float temperature;
    int32_t* inverse;                                       // token -> row, -1
    VocabRow* rows;
    int32_t* count;
    const int32_t* tile_counts;                             // of kVocabCountTile tokens each, or NULL: every block looks at all tokens
    int64_t plane;
    char* planes;                                           // blocked
    float* zero[2];                                         // outputs that are zero for tokens that take no part, or NULL
};
constexpr int kVocabRowsBlock = 16;                         // tokens per block

// How many of each kVocabCountTile tokens take part, where there are many tokens.
constexpr int kVocabCountTile = 4096;
__global__ void __launch_bounds__(kBlock)
k_vocab_count(const int32_t* __restrict__ targets, int n, int vocab, int32_t* __restrict__ tile_counts)
{
    __shared__ uint32_t sums[kWaves];
    uint32_t all = 0;
    for (int i = threadIdx.x; i < kVocabCountTile; i += kBlock) {
        const int64_t t = static_cast<int64_t>(blockIdx.x) * kVocabCountTile + i;
        all += t < n && static_cast<uint32_t>(targets[t]) < static_cast<uint32_t>(vocab);
    }
    all = wave_sum(all);
    if (threadIdx.x % kLanes == 0) sums[threadIdx.x / kLanes] = all;
    __syncthreads();
    if (threadIdx.x == 0) tile_counts[blockIdx.x] = static_cast<int32_t>(sums[0] + sums[1] + sums[2] + sums[3]);
}
static_assert(kWaves == 4, "");

// The rows that take part, one behind the other, as planes of bfloat16; zeros behind them and behind their ends.  Every block
// counts the tokens before its own for itself (up to 32768 reads of 4 bytes from L2, beyond that the tiles' counts), so up to there it is one launch.
template <typename T, int PLANES>
__global__ void __launch_bounds__(kBlock)
k_vocab_rows(const T* __restrict__ x, const VocabRowsArgs a)
{
    __shared__ uint32_t sums[2][kWaves];
    __shared__ int32_t place[kVocabRowsBlock];
    const int first = blockIdx.x * kVocabRowsBlock, lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    const auto there = [&](int t) { return t < a.n && static_cast<uint32_t>(a.targets[t]) < static_cast<uint32_t>(a.vocab); };
    uint32_t before = 0, all = 0;
    if (!a.tile_counts) {
        for (int t = threadIdx.x; t < a.n; t += kBlock) {
            const uint32_t one = there(t);
            all += one;
            before += t < first ? one : 0u;
        }
    } else {
        const int tile = first / kVocabCountTile, tiles = (a.n + kVocabCountTile - 1) / kVocabCountTile;
        for (int i = threadIdx.x; i < tiles; i += kBlock) {
            all += a.tile_counts[i];
            before += i < tile ? a.tile_counts[i] : 0;
        }
        for (int t = tile * kVocabCountTile + threadIdx.x; t < first; t += kBlock) before += there(t);
    }
    before = wave_sum(before);
    all = wave_sum(all);
    if (lane == 0) {
        sums[0][wave] = before;
        sums[1][wave] = all;
    }
    __syncthreads();
    before = all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before += sums[0][w];
        all += sums[1][w];
    }
    if (wave == 0) {
        const int t = first + lane;
        const bool mine = lane < kVocabRowsBlock && there(t);
        const uint64_t ballot = __ballot(mine);
        const int row = static_cast<int>(before + lanes_below(ballot));
        if (lane < kVocabRowsBlock) place[lane] = mine ? row : -1;
        if (lane < kVocabRowsBlock && t < a.n) {
            a.inverse[t] = mine ? row : -1;
            if (!mine) {
                if (a.zero[0]) a.zero[0][t] = 0.0f;
                if (a.zero[1]) a.zero[1][t] = 0.0f;
            }
        }
        if (mine) {
            VocabRow r{0.0f, 0.0f, 0.0f, a.one_target ? a.targets[t] : -1};
            if (a.dloss) {
                r.lse = a.lse[t];
                r.factor = a.dloss[t] * a.temperature;
                r.target_dz = a.one_target ? r.factor * expm1f(-a.loss[t]) : 0.0f;
            }
            a.rows[row] = r;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = static_cast<int32_t>(all);
    __syncthreads();
    const int quads = a.dim_padded / kVec;
    for (int i = threadIdx.x; i < quads * kVocabRowsBlock; i += kBlock) {
        const int r = i / quads, q = i % quads;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        int row = place[r];
        if (row >= 0) {
            four_of(x + static_cast<int64_t>(first + r) * a.stride, q * kVec, a.dim, v);
            store_planes4<PLANES, true>(a.planes + blocked(row, q * kVec, a.pitch), a.plane, v);
        }
        row = first + r;                                    // (a row behind the last one, perhaps)
        if (row >= static_cast<int>(all) && row < a.padded) {
            const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            store_planes4<PLANES, true>(a.planes + blocked(row, q * kVec, a.pitch), a.plane, none);
        }
    }
}

// A piece of the output matrix as planes of bfloat16, zeros behind its last row and behind the rows' ends.  One row per block in turn.
template <typename T, int PLANES>
__global__ void __launch_bounds__(kBlock)
k_vocab_planes(const T* __restrict__ w, int64_t stride, int rows, int padded, int dim, int dim_padded, int pitch, char* __restrict__ planes)
{
    const int64_t plane = static_cast<int64_t>(padded) * pitch * 2;
    const uint32_t quads = dim_padded / kVec;
    const uint64_t all = static_cast<uint64_t>(padded) * quads;
#pragma unroll 4
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kBlock + threadIdx.x; i < all; i += static_cast<uint64_t>(gridDim.x) * kBlock) {
        const uint32_t r = static_cast<uint32_t>(i / quads), q = static_cast<uint32_t>(i % quads);
        float v[4];
        four_of(w + static_cast<int64_t>(min(static_cast<int>(r), rows - 1)) * stride, q * kVec, static_cast<int>(r) < rows ? dim : 0, v);
        store_planes4<PLANES, true>(planes + (static_cast<int64_t>(r) * pitch + q * kVec) * 2, plane, v);
    }
}

// Whether one of 16 rows (those of the lanes) has its target among the wave's part of the vocabulary, which starts at `first`.
template <typename C>
__device__ __forceinline__ bool target_here(int target, int first)
{
    return __ballot(static_cast<uint32_t>(target - first) < static_cast<uint32_t>(C::FI * 16)) != 0;
}

// Loss: what a wave's part of a tile of logits adds to a row's sum of exponentials, as (largest logit, sum over exp(logit - largest)),
// without the target's.  i: vocabulary, j: rows.
template <typename C>
__global__ void __launch_bounds__(C::THREADS, C::PER_SIMD)
k_vocab_sums(const VocabOperand w, const VocabOperand x, const VocabSegments seg, int stages, int n_i, int vocab, int v0, float scale,
             const int32_t* __restrict__ count, const VocabRow* __restrict__ rows, float2* __restrict__ parts, int n_parts)
{
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int n = *count;
    const int wi = wave / C::WJ, wj = wave % C::WJ;
    const VocabTiles tiles{static_cast<uint32_t>(n_i), static_cast<uint32_t>((n + C::TJ - 1) / C::TJ), 1, stages * seg.n / 4};
    vocab_products<C, false, false, false, true>(w, x, seg, tiles, stages, wave, lane, [&](const VocabTile& t, acc4_t (&acc)[C::FI][C::FJ]) {
    const int i0 = v0 + t.i * C::TI + wi * C::FI * 16, i = i0 + lane / 16 * 4, part = i0 / (C::FI * 16);
    constexpr float kNone = -__builtin_huge_valf();
#pragma unroll
    for (int fj = 0; fj < C::FJ; ++fj) {
        const int j = t.j * C::TJ + wj * C::FJ * 16 + fj * 16 + lane % 16;
        const int target = j < n ? rows[j].target : -1;
        if (i0 + C::FI * 16 > vocab || target_here<C>(target, i0)) {
#pragma unroll
            for (int fi = 0; fi < C::FI; ++fi)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int v = i + fi * 16 + r;
                    if (v >= vocab || v == target) acc[fi][fj][r] = kNone;
                }
        }
        float top = kNone;
#pragma unroll
        for (int fi = 0; fi < C::FI; ++fi)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[fi][fj][r]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        float sum = 0.0f;
        top *= scale;                                       // (positive)
        const float from = top > kNone ? top : 0.0f;
#pragma unroll
        for (int fi = 0; fi < C::FI; ++fi)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += __expf(fmaf(acc[fi][fj][r], scale, -from));
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16 && j < n) parts[static_cast<int64_t>(j) * n_parts + part] = make_float2(top, sum);
    }
    });
}

// Gradient: a tile of dz of a piece of the vocabulary, as planes of bfloat16, zero behind the last row and the vocabulary's end.
template <typename C, int PLANES>
__global__ void __launch_bounds__(C::THREADS, C::PER_SIMD)
k_vocab_dz(const VocabOperand w, const VocabOperand x, const VocabSegments seg, int stages, int n_i, int vocab, int v0, float scale,
           const int32_t* __restrict__ count, const VocabRow* __restrict__ rows, char* __restrict__ dz, int64_t plane, uint32_t pitch)
{
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int n = *count;
    const int wi = wave / C::WJ, wj = wave % C::WJ;
    const VocabTiles tiles{static_cast<uint32_t>(n_i), static_cast<uint32_t>((n + C::TJ - 1) / C::TJ), 1, stages * seg.n / 4};
    vocab_products<C, false, false, false, true>(w, x, seg, tiles, stages, wave, lane, [&](const VocabTile& t, acc4_t (&acc)[C::FI][C::FJ]) {
    const int i0 = t.i * C::TI + wi * C::FI * 16, i = i0 + lane / 16 * 4;
#pragma unroll
    for (int fj = 0; fj < C::FJ; ++fj) {
        const int j0 = t.j * C::TJ + wj * C::FJ * 16 + fj * 16, j = j0 + lane % 16;
        const VocabRow row = j < n ? rows[j] : VocabRow{0.0f, 0.0f, 0.0f, -1};
#pragma unroll
        for (int fi = 0; fi < C::FI; ++fi)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[fi][fj][r] = row.factor * __expf(fmaf(acc[fi][fj][r], scale, -row.lse));
        if (v0 + i0 + C::FI * 16 > vocab || j0 + 16 > n || target_here<C>(row.target, v0 + i0)) {
#pragma unroll
            for (int fi = 0; fi < C::FI; ++fi)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int v = v0 + i + fi * 16 + r;
                    if (v == row.target) acc[fi][fj][r] = row.target_dz;
                    if (v >= vocab || j >= n) acc[fi][fj][r] = 0.0f;
                }
        }
#pragma unroll
        for (int fi = 0; fi < C::FI; ++fi) {
            const float d[4] = {acc[fi][fj][0], acc[fi][fj][1], acc[fi][fj][2], acc[fi][fj][3]};
            store_planes4<PLANES, false>(dz + blocked(j, i + fi * 16, pitch), plane, d);
        }
    }
    });
}

// Rows of zeros behind those that thin tiles write: dw's inner dimension goes on to a multiple of kVocabQuarter.
__global__ void __launch_bounds__(kBlock)
k_vocab_zero(char* __restrict__ at, int64_t words)
{
    const vf4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t w = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; w < words; w += static_cast<int64_t>(gridDim.x) * kBlock)
        reinterpret_cast<vf4_t*>(at)[w] = zero;
}

// dx += dz w over a piece of the vocabulary, in binary32.  i: columns of w, j: rows.  Blocks that share the inner dimension have a copy each.
template <typename C>
__global__ void __launch_bounds__(C::THREADS, C::PER_SIMD)
k_vocab_dx(const VocabOperand w, const VocabOperand dz, const VocabSegments seg, int stages, int n_i, int splits,
           const int32_t* __restrict__ count, float* __restrict__ sums, int padded, int dim_padded, int add)
{
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int n = *count;
    const int wi = wave / C::WJ, wj = wave % C::WJ;
    const VocabTiles tiles{static_cast<uint32_t>(n_i), static_cast<uint32_t>((n + C::TJ - 1) / C::TJ), static_cast<uint32_t>(splits), stages * seg.n / 4};
    vocab_products<C, true, false, false, true>(w, dz, seg, tiles, stages, wave, lane, [&](const VocabTile& t, acc4_t (&acc)[C::FI][C::FJ]) {
        const int i = t.i * C::TI + wi * C::FI * 16 + lane / 16 * 4;
#pragma unroll
        for (int fj = 0; fj < C::FJ; ++fj) {
            const int j = t.j * C::TJ + wj * C::FJ * 16 + fj * 16 + lane % 16;
            if (j >= n) continue;
            float* out = sums + (static_cast<int64_t>(t.split) * padded + j) * dim_padded;
#pragma unroll
            for (int fi = 0; fi < C::FI; ++fi) {
                const int d = i + fi * 16;
                if (d >= dim_padded) continue;
                acc4_t v = acc[fi][fj];
                if (add) v += *reinterpret_cast<const acc4_t*>(out + d);
                *reinterpret_cast<acc4_t*>(out + d) = v;
            }
            __builtin_amdgcn_sched_barrier(0);              // (all loads at once would take more registers than there are)
        }
    });
}

// The sums of dx in the caller's rows and type; zeros in those that take no part.
template <typename T>
__global__ void __launch_bounds__(kBlock)
k_vocab_dx_out(const float* __restrict__ sums, int splits, int padded, int dim, int dim_padded, const int32_t* __restrict__ inverse, int n,
               T* __restrict__ dx, int64_t stride)
{
    const uint32_t quads = (dim + kVec - 1) / kVec;
    const uint64_t all = static_cast<uint64_t>(n) * quads;
    for (uint64_t e = static_cast<uint64_t>(blockIdx.x) * kBlock + threadIdx.x; e < all; e += static_cast<uint64_t>(gridDim.x) * kBlock) {
        const uint32_t t = static_cast<uint32_t>(e / quads), d = static_cast<uint32_t>(e % quads) * kVec;
        const int row = inverse[t];
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (row >= 0) {
#pragma unroll 4
            for (int s = 0; s < splits; ++s) {
                const float4 p = cached4(sums + (static_cast<int64_t>(s) * padded + row) * dim_padded + d);
                v.x += p.x;
                v.y += p.y;
                v.z += p.z;
                v.w += p.w;
            }
        }
        const float f[4] = {v.x, v.y, v.z, v.w};
        store_row<false>(dx + static_cast<int64_t>(t) * stride + d, dim - static_cast<int>(d), f);
    }
}

// Four consecutive elements of a row of dw: written, or added to what is there (one rounding behind the sum in binary32).
template <typename T>
__device__ __forceinline__ void put_dw(T* to, int n, bool add, const acc4_t& v)
{
    float f[4] = {v[0], v[1], v[2], v[3]};
    if (add) {
        T old[4];
        load_row(to, n, old);
#pragma unroll
        for (int c = 0; c < 4; ++c) f[c] += widen(old[c]);
    }
    store_row<false>(to, n, f);
}

struct VocabDwArgs {
    float* slots;                                           // a copy of the piece's sums for each split, or NULL: straight into dw (one split, dim a multiple of four)
    int64_t stride;
    int32_t v0, vocab, dim, dim_padded, piece;              // (piece: rows of a copy)
    int32_t add, splits;
};

// How many blocks share the inner dimension of a tile of dw, of at most `splits`: n rows may be fewer than the call's tokens.
__device__ __forceinline__ int dw_parts(int n, int segments, int splits)
{
    return max(min((n + kVocabQuarter - 1) / kVocabQuarter * segments, splits), 1);
}

// dw = dz^T x of a piece of the vocabulary.  i: columns of x, j: vocabulary, inner dimension: rows.
template <typename C, typename T>
__global__ void __launch_bounds__(C::THREADS, C::PER_SIMD)
k_vocab_dw(const VocabOperand x, const VocabOperand dz, const VocabSegments seg, int n_i, int n_j, const int32_t* __restrict__ count, T* __restrict__ dw,
           const VocabDwArgs a)
{
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int n = *count;
    const int wi = wave / C::WJ, wj = wave % C::WJ;
    const int per = (n + kVocabQuarter - 1) / kVocabQuarter, splits = dw_parts(n, seg.n, a.splits);
    if (n == 0) {                                           // nothing to add up
        const int64_t rows = min(a.piece, a.vocab - a.v0), quads = (a.dim + kVec - 1) / kVec;
        for (int64_t q = static_cast<int64_t>(blockIdx.x) * C::THREADS + threadIdx.x; q < rows * quads; q += static_cast<int64_t>(gridDim.x) * C::THREADS) {
            const int64_t row = q / quads, d = (q - row * quads) * kVec;
            const acc4_t none = {0.0f, 0.0f, 0.0f, 0.0f};
            if (a.slots)
                *reinterpret_cast<acc4_t*>(a.slots + row * a.dim_padded + d) = none;
            else if (a.add == 0)
                put_dw(dw + (a.v0 + row) * a.stride + d, 4, false, none);
        }
        return;
    }
    const VocabTiles tiles{static_cast<uint32_t>(n_i), static_cast<uint32_t>(n_j), static_cast<uint32_t>(splits), per * seg.n};
    vocab_products<C, true, true, true, true>(x, dz, seg, tiles, per * 4, wave, lane, [&](const VocabTile& t, acc4_t (&acc)[C::FI][C::FJ]) {
        const int i = t.i * C::TI + wi * C::FI * 16 + lane / 16 * 4;
#pragma unroll
        for (int fj = 0; fj < C::FJ; ++fj) {
            const int j = t.j * C::TJ + wj * C::FJ * 16 + fj * 16 + lane % 16;
            if (a.v0 + j >= a.vocab) continue;
            if (a.slots) {
                float* to = a.slots + (static_cast<int64_t>(t.split) * a.piece + j) * a.dim_padded + i;
#pragma unroll
                for (int fi = 0; fi < C::FI; ++fi)
                    if (i + fi * 16 < a.dim) *reinterpret_cast<acc4_t*>(to + fi * 16) = acc[fi][fj];
            } else {
                T* to = dw + static_cast<int64_t>(a.v0 + j) * a.stride + i;
#pragma unroll
                for (int fi = 0; fi < C::FI; ++fi)
                    if (i + fi * 16 < a.dim) put_dw(to + fi * 16, 4, a.add != 0, acc[fi][fj]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    });
}

// Sums that blocks shared, joined in one order.
template <typename T>
__global__ void __launch_bounds__(kBlock)
k_vocab_dw_join(T* __restrict__ dw, const VocabDwArgs a, int rows, int segments, const int32_t* __restrict__ count)
{
    const int splits = dw_parts(*count, segments, a.splits);
    const uint32_t quads = (a.dim + kVec - 1) / kVec;
    const uint64_t all = static_cast<uint64_t>(rows) * quads;
    for (uint64_t e = static_cast<uint64_t>(blockIdx.x) * kBlock + threadIdx.x; e < all; e += static_cast<uint64_t>(gridDim.x) * kBlock) {
        const uint32_t j = static_cast<uint32_t>(e / quads), d = static_cast<uint32_t>(e % quads) * kVec;
        acc4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const acc4_t*>(a.slots + (static_cast<int64_t>(s) * a.piece + j) * a.dim_padded + d);
        put_dw(dw + static_cast<int64_t>(a.v0 + j) * a.stride + d, a.dim - static_cast<int>(d), a.add != 0, v);
    }
}

// Sum, or largest, over a block, in one order, for all its threads.
__device__ __forceinline__ float block_fold(float v, bool largest, float* lds)
{
#pragma unroll
    for (int m = 32; m >= 1; m /= 2) {
        const float other = __shfl_xor(v, m);
        v = largest ? fmaxf(v, other) : v + other;
    }
    __syncthreads();                                        // (lds is read by no one any more)
    if (threadIdx.x % kLanes == 0) lds[threadIdx.x / kLanes] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = largest ? fmaxf(v, lds[w]) : v + lds[w];
    return v;
}

// log sum exp of a row from its parts, by a block: the largest logit, and the logarithm of the sum beside it.
struct RowSum {
    float top, log_sum;
    __device__ __forceinline__ RowSum(const float2* __restrict__ parts, int n, float* lds)
    {
        constexpr int kHeld = 4;                            // parts of a thread that are read once
        float2 held[kHeld];
        top = -__builtin_huge_valf();
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int p = i * kBlock + static_cast<int>(threadIdx.x);
            held[i] = p < n ? parts[p] : make_float2(-__builtin_huge_valf(), 0.0f);
            top = fmaxf(top, held[i].x);
        }
        for (int p = kHeld * kBlock + threadIdx.x; p < n; p += kBlock) top = fmaxf(top, parts[p].x);
        top = block_fold(top, true, lds);
        const float from = top > -__builtin_huge_valf() ? top : 0.0f;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) sum += held[i].y * expf(held[i].x - from);
        for (int p = kHeld * kBlock + threadIdx.x; p < n; p += kBlock) sum += parts[p].y * expf(parts[p].x - from);
        log_sum = logf(block_fold(sum, false, lds));
    }
};

// Cross entropy of a token by a block, from the parts of the other tokens and its target's logit.
template <typename T>
__global__ void __launch_bounds__(kBlock)
k_entropy_join(const T* __restrict__ x, int64_t x_stride, const T* __restrict__ w, int64_t w_stride, int dim, const int32_t* __restrict__ targets,
               const int32_t* __restrict__ inverse, const float2* __restrict__ parts, int n_parts, float* __restrict__ loss, float* __restrict__ lse)
{
    __shared__ float lds[kWaves];
    const int64_t t = blockIdx.x;
    const int row = inverse[t];
    if (row < 0) return;                                    // (whole block; k_vocab_rows left zeros)
    const T* a = x + t * x_stride;
    const T* b = w + targets[t] * w_stride;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int d = threadIdx.x * kVec; d < dim; d += kBlock * kVec) {
        float u[4], v[4];
        four_of(a, d, dim, u);
        four_of(b, d, dim, v);
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] = fmaf(u[c], v[c], sum[c]);
    }
    const RowSum others(parts + static_cast<int64_t>(row) * n_parts, n_parts, lds);
    const float z = block_fold((sum[0] + sum[1]) + (sum[2] + sum[3]), false, lds);
    if (threadIdx.x != 0) return;
    const float all = others.top + others.log_sum, far = all - z, more = log1pf(expf(-fabsf(far)));
    // (a target's logit of infinity leaves no distribution, as an infinity elsewhere, whose exponential made `all` NaN; it is not the certain
    // token that `far` of minus infinity would make of it)
    loss[t] = z < __builtin_huge_valf() ? fmaxf(far, 0.0f) + more : __builtin_nanf("");
    lse[t] = (far > 0.0f ? all : z) + more;
}

// Logits at listed tokens in the rows of `w` (vocabulary from v0 on), 16 of a token's list per wave, formed by the same matrix instructions in the same
// order as in k_vocab_sums, so they have the very bits that lse was formed from: where a listed token has most of the
// probability, the errors of its logit and of lse are one and leave p (formed apart they made the gradients of a binary32 case
// twice as inexact, 4e-6 of their norm).  One row of the second operand would do, the instruction has 16: the products are few.
__global__ void __launch_bounds__(kBlock)
k_distill_listed(const VocabOperand w, int v0, int v1, int vocab, const int32_t* __restrict__ ids, int n, int per_token, const int32_t* __restrict__ inverse,
                 const VocabOperand x, int stages, const VocabSegments seg, float scale, float* __restrict__ out)
{
    const int lane = threadIdx.x % kLanes, groups = (per_token + 15) / 16;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    if (item >= static_cast<int64_t>(n) * groups) return;
    const int t = static_cast<int>(item / groups), first = static_cast<int>(item % groups) * 16;
    const int row = inverse[t];
    const int32_t* list = ids + static_cast<int64_t>(t) * per_token;
    const int entry = first + lane % 16;
    const int32_t id = entry < per_token ? list[entry] : -1;
    const bool known = row >= 0 && static_cast<uint32_t>(id) < static_cast<uint32_t>(vocab), here = known && id >= v0 && id < v1;
    float* to = out + static_cast<int64_t>(t) * per_token + entry;
    if (v0 == 0 && lane < 16 && entry < per_token && !known) *to = 0.0f;
    if (__ballot(here) == 0) return;                        // (whole wave)
    const char* of = w.at + static_cast<int64_t>(here ? id - v0 : 0) * w.pitch + lane / 16 * 16;
    const char* with = x.at + blocked(row, lane / 16 * 8, x.pitch);
    acc4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < seg.n; ++s) {
        const uint32_t pair = seg.pairs >> (s * 4);
        const char* a = of + (pair & 3u) * w.plane;
        const char* b = with + (pair >> 2 & 3u) * x.plane;
        bf8_t u[4], v[4];                                   // (stages are a multiple of four)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            u[k] = *reinterpret_cast<const bf8_t*>(a + k * 64);
            v[k] = *reinterpret_cast<const bf8_t*>(b + k * 1024);
        }
        for (int k0 = 4; k0 <= stages; k0 += 4) {           // (the last turn asks for the first places again)
            const int next = k0 < stages ? k0 : 0;
            bf8_t u_next[4], v_next[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                u_next[k] = *reinterpret_cast<const bf8_t*>(a + (next + k) * 64);
                v_next[k] = *reinterpret_cast<const bf8_t*>(b + (next + k) * 1024);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u[k], v[k], acc, 0, 0, 0);
                u[k] = u_next[k];
                v[k] = v_next[k];
            }
        }
    }
    // A lane holds entries lane / 16 * 4 + r, the same ones as the others of its 16; lane e of the first 16 looks after entry e.
    const int from = lane % 16 / 4 * 16;
    float z = 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float v = __shfl(acc[r], from);
        if (lane % 4 == r) z = v;
    }
    if (lane < 16 && here) *to = z * scale;
}

// The teacher's distribution over a token's list, by a wave: q = softmax over the entries that are there (in the vocabulary), of logits / tau.  The
// temperature is applied to what a logit is below the largest one: logits / tau may be out of range (lowest values of their type as a mask, tau < 1).
constexpr int kListedMax = 1024;
template <typename U>
struct TeacherList {
    float top, sum, inverse_tau;                            // top: the largest logit; -inf if there is nothing
    __device__ __forceinline__ float logit(const U* teacher, const int32_t* ids, int j, int n, int vocab) const
    {
        return j < n && static_cast<uint32_t>(ids[j]) < static_cast<uint32_t>(vocab) ? widen(teacher[j]) : -__builtin_huge_valf();
    }
    // (logit - top) / tau; -inf for an entry that is none
    __device__ __forceinline__ float below(const U* teacher, const int32_t* ids, int j, int n, int vocab) const
    {
        return (logit(teacher, ids, j, n, vocab) - top) * inverse_tau;
    }
    __device__ __forceinline__ TeacherList(const U* teacher, const int32_t* ids, int n, int vocab, float inverse_tau_, int lane) : inverse_tau(inverse_tau_)
    {
        top = -__builtin_huge_valf();
        bool odd = false;                                   // a NaN, which the maximum would skip
        for (int j = lane; j < n; j += kLanes) {
            const float u = logit(teacher, ids, j, n, vocab);
            odd |= u != u;
            top = fmaxf(top, u);
        }
#pragma unroll
        for (int m = 32; m >= 1; m /= 2) top = fmaxf(top, __shfl_xor(top, m));
        if (__ballot(odd) != 0) top = __builtin_nanf("");
        sum = 0.0f;
        for (int j = lane; j < n; j += kLanes) sum += expf(below(teacher, ids, j, n, vocab));
#pragma unroll
        for (int m = 32; m >= 1; m /= 2) sum += __shfl_xor(sum, m);
    }
    __device__ __forceinline__ bool empty() const { return top == -__builtin_huge_valf(); }
};

// Which tokens have a distribution (0) and which not (-1).
template <typename U>
__global__ void __launch_bounds__(kBlock)
k_distill_there(const int32_t* __restrict__ ids, const U* __restrict__ teacher, int n, int per_token, int vocab, float inverse_tau, int32_t* __restrict__ there)
{
    const int lane = threadIdx.x % kLanes;
    const int t = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    if (t >= n) return;
    const int64_t at = static_cast<int64_t>(t) * per_token;
    const TeacherList<U> list(teacher + at, ids + at, per_token, vocab, inverse_tau, lane);
    if (lane == 0) there[t] = list.empty() ? -1 : 0;
}

// lse and loss = tau^2 sum_j q_j (log q_j - z_j + lse), a block per token, of which one wave looks after the list.
template <typename U>
__global__ void __launch_bounds__(kBlock)
k_distill_join(const int32_t* __restrict__ ids, const U* __restrict__ teacher, const float* __restrict__ listed, int per_token, int vocab, float tau,
               const int32_t* __restrict__ inverse, const float2* __restrict__ parts, int n_parts, float* __restrict__ loss, float* __restrict__ lse)
{
    __shared__ float lds[kWaves];
    const int lane = threadIdx.x % kLanes;
    const int64_t t = blockIdx.x, at = t * per_token;
    const int row = inverse[t];
    if (row < 0) return;                                    // (whole block; k_vocab_rows left zeros)
    const RowSum all_of(parts + static_cast<int64_t>(row) * n_parts, n_parts, lds);
    if (threadIdx.x >= kLanes) return;
    const float all = all_of.top + all_of.log_sum;
    const TeacherList<U> list(teacher + at, ids + at, per_token, vocab, 1.0f / tau, lane);
    const float log_sum = logf(list.sum);
    float s = 0.0f;
    for (int j = lane; j < per_token; j += kLanes) {
        const float u = list.below(teacher + at, ids + at, j, per_token, vocab), q = expf(u) / list.sum;
        if (!(q == 0.0f)) s = fmaf(q, (u - log_sum) - ((listed[at + j] - all_of.top) - all_of.log_sum), s);   // (lse's rounding stays out)
    }
#pragma unroll
    for (int m = 32; m >= 1; m /= 2) s += __shfl_xor(s, m);
    if (lane != 0) return;
    lse[t] = all;
    loss[t] = tau * tau * s;
}

// What dz is at the listed tokens: c (exp(z - lse) - sum of q over the entries with that token).
template <typename U>
__global__ void __launch_bounds__(kBlock)
k_distill_targets(const int32_t* __restrict__ ids, const U* __restrict__ teacher, const float* __restrict__ listed, int n, int per_token, int vocab, float tau,
                  const float* __restrict__ lse, const float* __restrict__ dloss, float* __restrict__ values)
{
    __shared__ float q_of[kWaves][kListedMax];
    __shared__ int32_t id_of[kWaves][kListedMax];
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int t = blockIdx.x * kWaves + wave;
    if (t >= n) return;                                     // (whole wave; no barrier follows)
    const int64_t at = static_cast<int64_t>(t) * per_token;
    const TeacherList<U> list(teacher + at, ids + at, per_token, vocab, 1.0f / tau, lane);
    if (list.empty()) return;
    for (int j = lane; j < per_token; j += kLanes) {
        q_of[wave][j] = expf(list.below(teacher + at, ids + at, j, per_token, vocab)) / list.sum;
        id_of[wave][j] = ids[at + j];
    }
    wave_lds_fence();
    const float all = lse[t], factor = dloss[t] * tau;
    for (int j = lane; j < per_token; j += kLanes) {
        const int32_t id = id_of[wave][j];
        float q = 0.0f;
        for (int i = 0; i < per_token; ++i) q += id_of[wave][i] == id ? q_of[wave][i] : 0.0f;
        values[at + j] = factor * (expf(listed[at + j] - all) - q);
    }
}

// Those values into a piece of dz (an entry that is there twice writes the same value twice).
template <int PLANES>
__global__ void __launch_bounds__(kBlock)
k_distill_put(const int32_t* __restrict__ ids, const float* __restrict__ values, int64_t n, int per_token, const int32_t* __restrict__ inverse, int vocab,
              int v0, int piece, char* __restrict__ dz, int64_t plane, uint32_t pitch)
{
    const int64_t e = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
    if (e >= n) return;
    const int32_t id = ids[e];
    if (id < v0 || id >= min(v0 + piece, vocab)) return;
    const int row = inverse[e / per_token];
    if (row < 0) return;
    float rest = values[e];
#pragma unroll
    for (int p = 0; p < PLANES; ++p) {
        const uint16_t bits = bf16_bits(rest);
        *reinterpret_cast<uint16_t*>(dz + p * plane + blocked(row, id - v0, pitch)) = bits;
        rest -= widen(bits);
    }
}

}  // namespace
