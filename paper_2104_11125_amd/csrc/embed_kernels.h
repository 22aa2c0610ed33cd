// Kernels of the embedding: rows of a table by token, and the table's gradient by sorted tokens.  Part of scalecom.hip's
// single translation unit.
//
//   out_t = scale * table[token_t]                       zeros for a token outside the table (padding)
//   grad_v (+)= scale * sum over t with token_t = v of dout_t
//
// The gradient needs no float atomics, so its bits do not depend on the order in which blocks run.  Positions are sorted by (token, position);
// a run of one token is summed in binary32 in the order of its positions, in tiles of them, and what a
// run leaves in several tiles is put together by k_embed_join.  A gradient that replaces what was there is zeroed by blocks that ride along with
// the sorting launches, which leave most of the chip idle.
//
// What bounds it.  Lookup: HBM, 65536 rows of 1024 f32 to bf16 39 us, 4.8 TB/s of the rows that are distinct and the output (28 us at the rate of a copy); 512 rows
// of 512 take 4 us, a launch and two dependent loads.  Gradient: 65536 x 2048 bf16 into 131072 rows 214 us, half of it zeros at 5.2 TB/s beside four sorting
// launches, 83 us the sums (335 MB), 14 the joins; 4096 x 512 f32 into 32768 rows 23.5 us: 13 zeros beside the sort, 5.5 and 4 two launches of dependent loads.
#pragma once

#include <hip/hip_runtime.h>

#include "device_helpers.h"
#include "geometry.h"
#include "optimizer_kernels.h"

namespace {

constexpr int kEmbedBatch = 16;                             // sorted positions whose rows a wave of k_embed_sums has under way
constexpr int kEmbedManyWaves = 8192;                       // with so many a wave takes two batches: half of the parts to be joined
constexpr int kEmbedDigit = 9, kEmbedDigits = 1 << kEmbedDigit;
constexpr int kEmbedSortBlock = 1024, kEmbedSortRows = 4, kEmbedSortTile = kEmbedSortBlock * kEmbedSortRows;
constexpr int kEmbedOneMax = 4096;                          // positions that one block sorts

// A matrix that is zeroed by the blocks [first, first + blocks) of a launch, `part` of `parts` of it.
struct EmbedFill {
    char* at;
    int64_t rows, row_bytes, stride_bytes;
    uint32_t blocks, part, parts;
};
constexpr int64_t kEmbedFillBytes = 65536;                  // of a block

// Zeroes the block's share, in words of 16 bytes where rows lie back to back.  `block` of fill.blocks; any number of threads.
__device__ __forceinline__ void embed_fill(const EmbedFill& f, uint32_t block)
{
    const uint32_t threads = blockDim.x;
    if (f.stride_bytes == f.row_bytes) {
        char* begin = f.at;
        char* end = begin + f.rows * f.row_bytes;
        char* a = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(begin) + 15) & ~static_cast<uintptr_t>(15));
        if (a > end) a = end;
        const int64_t words = (end - a) / 16;
        const vf4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
        const int64_t from = words * f.part / f.parts, to = words * (f.part + 1) / f.parts;
        for (int64_t w = from + static_cast<int64_t>(block) * threads + threadIdx.x; w < to; w += static_cast<int64_t>(f.blocks) * threads)
            __builtin_nontemporal_store(zero, reinterpret_cast<vf4_t*>(a) + w);
        if (block == 0 && f.part == 0) {                    // (elements are of two bytes at least)
            for (char* p = begin + threadIdx.x * 2; p < a; p += threads * 2) *reinterpret_cast<uint16_t*>(p) = 0;
            for (char* p = a + words * 16 + threadIdx.x * 2; p < end; p += threads * 2) *reinterpret_cast<uint16_t*>(p) = 0;
        }
        return;
    }
    const int64_t from = f.rows * f.part / f.parts, to = f.rows * (f.part + 1) / f.parts;
    for (int64_t r = from + block; r < to; r += f.blocks)
        for (int64_t b = threadIdx.x * 2; b < f.row_bytes; b += threads * 2) *reinterpret_cast<uint16_t*>(f.at + r * f.stride_bytes + b) = 0;
}

// What a token is sorted by: itself, or `vocab`, behind all others, if it is not in the table.
__device__ __forceinline__ uint32_t embed_key(int32_t token, uint32_t vocab) { return min(static_cast<uint32_t>(token), vocab); }

// A lane's elements of a row: 16 bytes of the narrower kind, which the memory system takes at any element's address (four-byte ones at full
// rate).  Held as they lie until they are used.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) ElementsAt {
    T v[N];
};
template <typename T, int N>
__device__ __forceinline__ void load_row(const T* from, int left, T (&v)[N])    // `left` elements are there; zeros behind
{
    if (left >= N) {
        const ElementsAt<T, N> e = *reinterpret_cast<const ElementsAt<T, N>*>(from);
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = e.v[c];
        return;
    }
#pragma unroll
    for (int c = 0; c < N; ++c) v[c] = c < left ? from[c] : T(0);
}
__device__ __forceinline__ float as_type(float x, float) { return x; }
__device__ __forceinline__ uint16_t as_type(float x, uint16_t) { return bf16_bits(x); }
// STREAM: with the nontemporal hint, for what is not read again soon (65536 rows of 1024 bfloat16 39 us, without it 54).
template <bool STREAM, typename T, int N>
__device__ __forceinline__ void store_row(T* to, int left, const float (&v)[N])
{
    if (left >= N) {
        ElementsAt<T, N> e;
#pragma unroll
        for (int c = 0; c < N; ++c) e.v[c] = as_type(v[c], T());
        if constexpr (STREAM) {
            typedef uint32_t two_t __attribute__((ext_vector_type(2)));
            typedef two_t two_at_t __attribute__((aligned(2)));
            typedef uint32_t four_t __attribute__((ext_vector_type(4)));
            typedef four_t four_at_t __attribute__((aligned(2)));
            constexpr int kBytes = N * sizeof(T);
            if constexpr (kBytes == 8) {
                __builtin_nontemporal_store(__builtin_bit_cast(two_t, e), reinterpret_cast<two_at_t*>(to));
            } else {
                static_assert(kBytes % 16 == 0, "");
                struct {
                    four_t w[kBytes / 16];
                } words = __builtin_bit_cast(decltype(words), e);
#pragma unroll
                for (int c = 0; c < kBytes / 16; ++c) __builtin_nontemporal_store(words.w[c], reinterpret_cast<four_at_t*>(to) + c);
            }
        } else {
            *reinterpret_cast<ElementsAt<T, N>*>(to) = e;
        }
        return;
    }
#pragma unroll
    for (int c = 0; c < N; ++c)
        if (c < left) put(to + c, v[c]);
}

// 2^shift lanes take a row's columns, eight each and in turns, kEmbedRows rows a lane, whose loads are under way together.
constexpr int kEmbedRows = 4, kEmbedCols = 8;
template <typename T, typename O>
__global__ void __launch_bounds__(kBlock)
k_embed(const T* __restrict__ table, int64_t stride, uint32_t vocab, int dim, const int32_t* __restrict__ tokens, uint32_t n, int shift, float scale,
        O* __restrict__ out, int64_t out_stride)
{
    const uint32_t per_block = kBlock >> shift, first = blockIdx.x * per_block * kEmbedRows + (threadIdx.x >> shift);
    uint32_t id[kEmbedRows];
#pragma unroll
    for (int i = 0; i < kEmbedRows; ++i) {
        const uint32_t t = first + i * per_block;
        id[i] = t < n ? static_cast<uint32_t>(tokens[t]) : vocab;
    }
    for (int col = (threadIdx.x & ((1 << shift) - 1)) * kEmbedCols; col < dim; col += kEmbedCols << shift) {
        T v[kEmbedRows][kEmbedCols];
#pragma unroll
        for (int i = 0; i < kEmbedRows; ++i) load_row(table + (id[i] < vocab ? id[i] : 0) * stride + col, id[i] < vocab ? dim - col : 0, v[i]);
#pragma unroll
        for (int i = 0; i < kEmbedRows; ++i) {
            const uint32_t t = first + i * per_block;
            if (t >= n) continue;
            float x[kEmbedCols];
#pragma unroll
            for (int c = 0; c < kEmbedCols; ++c) x[c] = widen(v[i][c]) * scale;
            store_row<true>(out + t * out_stride + col, dim - col, x);
        }
    }
}

// Sorting is by digits of up to 9 bits, lowest first, equal digits in their order.
struct EmbedDigit {
    int shift, bits;
    __device__ __forceinline__ uint32_t operator()(uint32_t key) const { return key >> shift & ((1u << bits) - 1); }
};

// A wave's positions come row after row of 64: how many of its earlier ones have a lane's digit, row after row.  `counts` (zero at first; how often the
// wave has every digit) is the wave's own.  Lanes of one digit find each other by a ballot a bit.
template <typename Count>
__device__ __forceinline__ uint32_t embed_rank(uint32_t key, bool there, const EmbedDigit& of, Count* counts)
{
    const uint64_t all = __ballot(there);
    const uint32_t digit = of(key), before = counts[digit];
    uint32_t low = static_cast<uint32_t>(all), high = static_cast<uint32_t>(all >> 32);         // the lanes with the same digit
#pragma unroll
    for (int b = 0; b < kEmbedDigit; ++b) {
        const uint32_t mine = static_cast<uint32_t>(static_cast<int32_t>(digit << (31 - b)) >> 31);          // the bit, 32 times
        const uint64_t ones = __ballot(mine != 0);
        low &= ~(static_cast<uint32_t>(ones) ^ mine);
        high &= ~(static_cast<uint32_t>(ones >> 32) ^ mine);
    }
    const uint32_t below = __builtin_amdgcn_mbcnt_hi(high, __builtin_amdgcn_mbcnt_lo(low, 0u));
    wave_lds_fence();
    if (there && below == 0) counts[digit] = static_cast<Count>(before + static_cast<uint32_t>(__popc(low) + __popc(high)));
    wave_lds_fence();
    return before + below;
}

// The digits' first places: digit d < kEmbedDigits, of the first threads of a block, has `count` positions.
__device__ __forceinline__ uint32_t embed_digit_scan(uint32_t count, uint32_t* wave_total)
{
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    uint32_t inclusive = count;
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) {
        const uint32_t v = __shfl_up(inclusive, m);
        if (lane >= m) inclusive += v;
    }
    if (lane == kLanes - 1 && wave < kEmbedDigits / kLanes) wave_total[wave] = inclusive;
    __syncthreads();
    uint32_t first = inclusive - count;
    for (int w = 0; w < min(wave, kEmbedDigits / kLanes); ++w) first += wave_total[w];
    return first;
}

// Few positions: one block sorts them, held in registers and exchanged through LDS, the others zero the gradient meanwhile.  Bound by that block's
// instructions, some 2.4 us for 1000 positions in two digits: with 10007 it takes 24 us, as long as the four launches below do, with 4096 less than zeroing
// a gradient of 64 MB.  (At 10007: counting, for every position, those before it, by comparison and all over the chip, 22 to 27; masks of equal digits
// joined in LDS instead of by ballots 24; rows in a loop, with positions in memory, 35.)
constexpr int kEmbedSortWaves = kEmbedSortBlock / kLanes, kEmbedOneRows = kEmbedOneMax / kEmbedSortBlock;
__global__ void __launch_bounds__(kEmbedSortBlock)
k_embed_sort(const int32_t* __restrict__ tokens, int n, uint32_t vocab, int digits, int bits, const EmbedFill fill, int32_t* __restrict__ keys,
             int32_t* __restrict__ positions)
{
    if (blockIdx.x > 0) {
        embed_fill(fill, blockIdx.x - 1);
        return;
    }
    __shared__ uint32_t key_at[kEmbedOneMax], wave_total[kEmbedDigits / kLanes];
    __shared__ uint16_t counts[kEmbedSortWaves][kEmbedDigits], position_at[kEmbedOneMax];
    static_assert(kEmbedOneMax <= 65536, "positions in 16 bits");
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    const int rows = (n + kEmbedSortBlock - 1) / kEmbedSortBlock;           // of a wave: few positions are spread over the waves
    uint32_t key[kEmbedOneRows], rank[kEmbedOneRows];
    int32_t position[kEmbedOneRows];
    bool there[kEmbedOneRows];
#pragma unroll
    for (int r = 0; r < kEmbedOneRows; ++r) {
        position[r] = (wave * rows + r) * kLanes + lane;
        there[r] = r < rows && position[r] < n;
        key[r] = there[r] ? embed_key(tokens[position[r]], vocab) : 0u;
    }
    for (int d = 0; d < digits; ++d) {
        const EmbedDigit of{d * bits, bits};
        for (int i = threadIdx.x; i < kEmbedSortWaves * kEmbedDigits; i += kEmbedSortBlock) counts[0][i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kEmbedOneRows; ++r)
            if (r < rows) rank[r] = embed_rank(key[r], there[r], of, counts[wave]);              // (uniform)
        __syncthreads();
        uint32_t count = 0;
        if (threadIdx.x < kEmbedDigits) {
#pragma unroll
            for (int w = 0; w < kEmbedSortWaves; ++w) count += counts[w][threadIdx.x];
        }
        uint32_t first = embed_digit_scan(count, wave_total);
        if (threadIdx.x < kEmbedDigits) {
#pragma unroll
            for (int w = 0; w < kEmbedSortWaves; ++w) {     // counts become the first places of every wave
                const uint32_t c = counts[w][threadIdx.x];
                counts[w][threadIdx.x] = static_cast<uint16_t>(first);
                first += c;
            }
        }
        __syncthreads();
        const bool last = d + 1 == digits;
#pragma unroll
        for (int r = 0; r < kEmbedOneRows; ++r) {
            if (!there[r]) continue;
            const uint32_t to = counts[wave][of(key[r])] + rank[r];         // (places before those of n positions: each of 0 .. n - 1 once)
            if (last) {
                keys[to] = static_cast<int32_t>(key[r]);
                positions[to] = position[r];
            } else {
                key_at[to] = key[r];
                position_at[to] = static_cast<uint16_t>(position[r]);
            }
        }
        if (last) break;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kEmbedOneRows; ++r) {
            const int at = (wave * rows + r) * kLanes + lane;
            if (!there[r]) continue;
            key[r] = key_at[at];
            position[r] = position_at[at];
        }
    }
}

// More positions: two launches a digit.  k_embed_count: how often a block's tile has every digit.
template <bool FIRST>
__device__ __forceinline__ void embed_tile_keys(const int32_t* __restrict__ tokens, const int32_t* __restrict__ keys, const int32_t* __restrict__ positions,
                                                int n, uint32_t vocab, int wave, int lane, uint32_t (&key)[kEmbedSortRows],
                                                int32_t (&position)[kEmbedSortRows], bool (&there)[kEmbedSortRows])
{
#pragma unroll
    for (int r = 0; r < kEmbedSortRows; ++r) {
        const int t = blockIdx.x * kEmbedSortTile + (wave * kEmbedSortRows + r) * kLanes + lane;
        there[r] = t < n;
        key[r] = 0;
        position[r] = t;
        if (!there[r]) continue;
        if (FIRST) {
            key[r] = embed_key(tokens[t], vocab);
        } else {
            key[r] = static_cast<uint32_t>(keys[t]);
            position[r] = positions[t];
        }
    }
}

template <bool FIRST>
__global__ void __launch_bounds__(kEmbedSortBlock)
k_embed_count(const int32_t* __restrict__ tokens, const int32_t* __restrict__ keys, int n, uint32_t vocab, const EmbedDigit of, uint32_t sort_blocks,
              const EmbedFill fill, uint32_t* __restrict__ table)
{
    if (blockIdx.x >= sort_blocks) {
        embed_fill(fill, blockIdx.x - sort_blocks);
        return;
    }
    __shared__ uint32_t counts[kEmbedDigits];
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;     // (positions in the order of k_embed_place's)
    if (threadIdx.x < kEmbedDigits) counts[threadIdx.x] = 0;
    __syncthreads();
    uint32_t key[kEmbedSortRows];
    int32_t position[kEmbedSortRows];
    bool there[kEmbedSortRows];
    embed_tile_keys<FIRST>(tokens, keys, keys, n, vocab, wave, lane, key, position, there);
#pragma unroll
    for (int r = 0; r < kEmbedSortRows; ++r)
        if (there[r]) atomicAdd(&counts[of(key[r])], 1u);
    __syncthreads();
    if (threadIdx.x < kEmbedDigits) table[blockIdx.x * kEmbedDigits + threadIdx.x] = counts[threadIdx.x];
}

// k_embed_place: every block adds up the tiles before its own and the digits before each (the table is a few kilobytes per tile) and
// moves its positions, equal digits in their order.
template <bool FIRST>
__global__ void __launch_bounds__(kEmbedSortBlock)
k_embed_place(const int32_t* __restrict__ tokens, const int32_t* __restrict__ keys, const int32_t* __restrict__ positions, int n, uint32_t vocab, const EmbedDigit of,
              uint32_t sort_blocks, const EmbedFill fill, const uint32_t* __restrict__ table, int32_t* __restrict__ keys_out,
              int32_t* __restrict__ positions_out)
{
    if (blockIdx.x >= sort_blocks) {
        embed_fill(fill, blockIdx.x - sort_blocks);
        return;
    }
    __shared__ uint32_t counts[kEmbedSortWaves][kEmbedDigits], halves[2][2][kEmbedDigits], wave_total[kEmbedDigits / kLanes];
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    for (int i = threadIdx.x; i < kEmbedSortWaves * kEmbedDigits; i += kEmbedSortBlock) counts[0][i] = 0;
    uint32_t key[kEmbedSortRows], rank[kEmbedSortRows];
    int32_t position[kEmbedSortRows];
    bool there[kEmbedSortRows];
    embed_tile_keys<FIRST>(tokens, keys, positions, n, vocab, wave, lane, key, position, there);
    {
        // two halves of the block share the tiles of the table
        const uint32_t digit = threadIdx.x % kEmbedDigits, half = threadIdx.x / kEmbedDigits;
        uint32_t before = 0, all = 0;
#pragma unroll 4
        for (uint32_t b = half; b < sort_blocks; b += 2) {
            const uint32_t c = table[b * kEmbedDigits + digit];
            all += c;
            before += b < blockIdx.x ? c : 0u;
        }
        halves[half][0][digit] = before;
        halves[half][1][digit] = all;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kEmbedSortRows; ++r) rank[r] = embed_rank(key[r], there[r], of, counts[wave]);
    const bool mine = threadIdx.x < kEmbedDigits;
    uint32_t first = embed_digit_scan(mine ? halves[0][1][threadIdx.x] + halves[1][1][threadIdx.x] : 0u, wave_total);
    if (mine) {                                             // counts become the first places of every wave
        first += halves[0][0][threadIdx.x] + halves[1][0][threadIdx.x];
        for (int w = 0; w < kEmbedSortWaves; ++w) {
            const uint32_t c = counts[w][threadIdx.x];
            counts[w][threadIdx.x] = first;
            first += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kEmbedSortRows; ++r) {
        if (!there[r]) continue;
        const uint32_t to = counts[wave][of(key[r])] + rank[r];
        if (to >= static_cast<uint32_t>(n)) continue;       // (tokens that change between the launches would make it no permutation)
        keys_out[to] = static_cast<int32_t>(key[r]);
        positions_out[to] = position[r];
    }
}

// Elements of a row of the gradient: written, or added to what is there.
template <typename G, int N>
__device__ __forceinline__ void embed_put(G* to, int left, bool add, float scale, const float (&s)[N])
{
    float v[N];
    if (add) {
        G old[N];
        load_row(to, left, old);
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = fmaf(scale, s[c], widen(old[c]));
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = scale * s[c];
    }
    store_row<true>(to, left, v);
}

constexpr int kEmbedPartCols = 512;                         // rows of partial sums are padded to multiples of it
struct EmbedSums {
    const int32_t *keys, *positions;
    int32_t n, dim;
    uint32_t vocab, tiles;
    int32_t run;                                            // sorted positions of a tile: a multiple of kEmbedBatch
    int64_t dout_stride, grad_stride;
    float scale;
    int32_t add;
    int64_t part_stride;                                    // per tile two rows of partial sums: of the run that began before it, of the one that goes on behind it
    float* partial;
};

// Sums of the runs in a tile of sorted positions, 64 N columns per wave.  A run that lies in one tile goes to the gradient, the
// parts of longer ones to `partial`.
template <typename T, typename G, int N>
__device__ __forceinline__ void embed_sums(const T* __restrict__ dout, G* __restrict__ grad, const EmbedSums& a, uint32_t tile, uint32_t chunk, int lane)
{
    const int begin = static_cast<int>(tile) * a.run, end = min(begin + a.run, a.n), col = (static_cast<int>(chunk) * kLanes + lane) * N;
    const int left = a.dim - col;                           // columns from here on; none: the lane reads and writes nothing
    // lane i of the first ones has the batch's i-th key and position, and the key behind them
    const auto keys_from = [&](int p) { return p + lane < a.n && lane <= kEmbedBatch ? a.keys[p + lane] : -1; };
    const auto positions_from = [&](int p) { return p + lane < a.n && lane < kEmbedBatch ? a.positions[p + lane] : 0; };
    int32_t keys = keys_from(begin), positions = positions_from(begin);
    float s[N];
#pragma unroll
    for (int c = 0; c < N; ++c) s[c] = 0.0f;
    bool from_before = begin > 0 && a.keys[begin > 0 ? begin - 1 : 0] == __builtin_amdgcn_readlane(keys, 0);
    float* partial = a.partial + tile * 2 * a.part_stride + col;
    for (int p0 = begin; p0 < end; p0 += kEmbedBatch) {
        T v[kEmbedBatch][N];
        uint32_t key[kEmbedBatch + 1];
#pragma unroll
        for (int i = 0; i <= kEmbedBatch; ++i) key[i] = static_cast<uint32_t>(__builtin_amdgcn_readlane(keys, i));
#pragma unroll
        for (int i = 0; i < kEmbedBatch; ++i)
            load_row(dout + __builtin_amdgcn_readlane(positions, i) * a.dout_stride + col, key[i] < a.vocab ? left : 0, v[i]);
        if (p0 + kEmbedBatch < end) {
            keys = keys_from(p0 + kEmbedBatch);
            positions = positions_from(p0 + kEmbedBatch);
        }
#pragma unroll
        for (int i = 0; i < kEmbedBatch; ++i) {
#pragma unroll
            for (int c = 0; c < N; ++c) s[c] += widen(v[i][c]);
            if (key[i] >= a.vocab) continue;                // (uniform)
            const bool last = p0 + i + 1 == end;
            if (!last && key[i + 1] == key[i]) continue;
            if (from_before)
                store_row<false>(partial, N, s);
            else if (last && key[i + 1] == key[i])
                store_row<false>(partial + a.part_stride, N, s);
            else if (left > 0)
                embed_put(grad + key[i] * a.grad_stride + col, left, a.add != 0, a.scale, s);
#pragma unroll
            for (int c = 0; c < N; ++c) s[c] = 0.0f;
            from_before = false;
        }
    }
}
template <typename T, typename G>
__global__ void __launch_bounds__(kBlock)
k_embed_sums(const T* __restrict__ dout, G* __restrict__ grad, const EmbedSums a)
{
    constexpr int N = 16 / sizeof(T);
    const uint32_t chunks = (a.dim + kLanes * N - 1) / (kLanes * N);
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    if (item < a.tiles * chunks) embed_sums<T, G, N>(dout, grad, a, item / chunks, item % chunks, threadIdx.x % kLanes);
}

// Runs over several tiles, put together for the tile in which they begin, 256 columns per wave.  Most reach one tile more and are
// the wave's own work; a block's waves share the parts of longer ones.  One order whatever the timing.
constexpr int kEmbedJoinWaves = 4, kEmbedJoinOwn = 8;       // parts that a wave adds up by itself
template <typename G>
__global__ void __launch_bounds__(kEmbedJoinWaves * kLanes)
k_embed_join(G* __restrict__ grad, const EmbedSums a)
{
    __shared__ float4 lds[kEmbedJoinWaves][kLanes];
    __shared__ uint32_t shared_tile[kEmbedJoinWaves], shared_last[kEmbedJoinWaves], shared_chunk[kEmbedJoinWaves];
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const uint32_t chunks = (a.dim + kWaveTile - 1) / kWaveTile, item = blockIdx.x * kEmbedJoinWaves + wave;
    const uint32_t tile = item % a.tiles, chunk = item / a.tiles;   // (neighbours: tiles of one chunk, of which few begin long runs)
    const auto add_up = [&](uint32_t from, uint32_t last, uint32_t step, uint32_t at_chunk, float4 s) {
#pragma unroll 8
        for (uint32_t t = from; t <= last; t += step) {
            const float4 v = cached4(a.partial + t * 2 * a.part_stride + at_chunk * kWaveTile + lane * kVec);
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
        return s;
    };
    const auto first_part = [&](uint32_t t, uint32_t at_chunk) { return cached4(a.partial + (static_cast<int64_t>(t) * 2 + 1) * a.part_stride + at_chunk * kWaveTile + lane * kVec); };
    const auto finish = [&](uint32_t t, uint32_t at_chunk, const float4& v) {
        const int col = static_cast<int>(at_chunk) * kWaveTile + lane * kVec;
        const float s[4] = {v.x, v.y, v.z, v.w};
        if (col < a.dim) embed_put(grad + a.keys[(t + 1) * a.run - 1] * a.grad_stride + col, a.dim - col, a.add != 0, a.scale, s);
    };
    uint32_t last = 0;                                      // the last tile that the run reaches; 0: no run begins here that goes on
    if (tile + 1 < a.tiles && chunk < chunks) {
        const int end = static_cast<int>(tile + 1) * a.run;
        const uint32_t key = static_cast<uint32_t>(a.keys[end - 1]);
        const bool earlier = tile > 0 && static_cast<uint32_t>(a.keys[end - a.run]) == key && static_cast<uint32_t>(a.keys[end - a.run - 1]) == key;
        if (key < a.vocab && static_cast<uint32_t>(a.keys[end]) == key && !earlier) {
            const int near = min(end + a.run, a.n) - 1;
            const int64_t behind = static_cast<uint32_t>(a.keys[near]) != key ? near : end + wave_lower_bound(a.keys + end, a.n - end, static_cast<int64_t>(key) + 1);
            last = static_cast<uint32_t>((behind - 1) / a.run);
        }
    }
    const bool own = last > 0 && last - tile <= kEmbedJoinOwn;
    if (own) finish(tile, chunk, add_up(tile + 1, last, 1, chunk, first_part(tile, chunk)));
    if (lane == 0) {
        shared_tile[wave] = tile;
        shared_last[wave] = own ? 0 : last;
        shared_chunk[wave] = chunk;
    }
    __syncthreads();
    for (int w = 0; w < kEmbedJoinWaves; ++w) {
        const uint32_t to = shared_last[w], from = shared_tile[w], at_chunk = shared_chunk[w];
        if (to == 0) continue;                              // (the same for all)
        const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        lds[wave][lane] = add_up(from + 1 + wave, to, kEmbedJoinWaves, at_chunk, wave == 0 ? first_part(from, at_chunk) : none);
        __syncthreads();
        if (wave == 0) {
            float4 s = lds[0][lane];
            for (int i = 1; i < kEmbedJoinWaves; ++i) {
                const float4 v = lds[i][lane];
                s.x += v.x;
                s.y += v.y;
                s.z += v.z;
                s.w += v.w;
            }
            finish(from, at_chunk, s);
        }
        __syncthreads();
    }
}

}  // namespace
