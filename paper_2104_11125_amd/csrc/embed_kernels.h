// Kernels of the embedding: rows of a table by token, and the table's gradient by sorted tokens.  Part of scalecom.hip's
// single translation unit.
//
//   out_t = scale * table[token_t]                       zeros for a token outside the table (padding)
//   grad_v (+)= scale * sum over t with token_t = v of dout_t
//
// The gradient needs no float atomics, so its bits do not depend on the order in which blocks run.  Positions are sorted by (token, position);
// a run of one token is summed in binary32 in the order of its positions, in tiles of kEmbedRun of them, and what a
// run leaves in several tiles is put together by k_embed_join.  A gradient that replaces what was there is zeroed by blocks that ride along with
// the sorting launches, which leave most of the chip idle.
#pragma once

#include <hip/hip_runtime.h>

#include "device_helpers.h"
#include "geometry.h"
#include "optimizer_kernels.h"

namespace {

constexpr int kEmbedRun = 16;                               // sorted positions of a wave of k_embed_sums
constexpr int kEmbedDigit = 9, kEmbedDigits = 1 << kEmbedDigit;
constexpr int kEmbedSortBlock = 1024, kEmbedSortRows = 4, kEmbedSortTile = kEmbedSortBlock * kEmbedSortRows;
constexpr int kEmbedRankWaves = 16;

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

// One wave takes 256 columns of a row, several rows in flight.
constexpr int kEmbedRows = 4;
template <typename T, typename O>
__global__ void __launch_bounds__(kBlock)
k_embed(const T* __restrict__ table, int64_t stride, uint32_t vocab, int dim, const int32_t* __restrict__ tokens, uint32_t n, uint32_t chunks, float scale,
        O* __restrict__ out, int64_t out_stride, int aligned)
{
    const int lane = threadIdx.x % kLanes;
    const uint32_t items = n * chunks, first = (blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes)) * kEmbedRows;
    float4 v[kEmbedRows];
    int64_t row[kEmbedRows];
    int col[kEmbedRows];
#pragma unroll
    for (int i = 0; i < kEmbedRows; ++i) {
        const uint32_t item = first + i;
        row[i] = item < items ? static_cast<int64_t>(item / chunks) : -1;
        col[i] = static_cast<int>(item % chunks) * kWaveTile + lane * kVec;
        v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (row[i] < 0 || col[i] >= dim) continue;
        const uint32_t id = static_cast<uint32_t>(tokens[row[i]]);
        if (id >= vocab) continue;
        const T* from = table + id * stride + col[i];
        if (aligned && col[i] + 3 < dim) {
            v[i] = cached4(from);
        } else {
            float e[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) e[c] = col[i] + c < dim ? widen(from[c]) : 0.0f;
            v[i] = make_float4(e[0], e[1], e[2], e[3]);
        }
    }
#pragma unroll
    for (int i = 0; i < kEmbedRows; ++i) {
        if (row[i] < 0 || col[i] >= dim) continue;
        const float4 s = make_float4(v[i].x * scale, v[i].y * scale, v[i].z * scale, v[i].w * scale);
        O* to = out + row[i] * out_stride + col[i];
        if (aligned && col[i] + 3 < dim)
            store4(to, s);
        else
            store_first(to, dim - col[i], s);
    }
}

// Sorting by comparison, for few positions: a position's place is the number of positions before it in the order (token, position).  A block takes
// 64 positions, its waves a part of all positions each, 64 at a time against uniform keys: two instructions a pair.
__global__ void __launch_bounds__(kEmbedRankWaves * kLanes)
k_embed_rank(const int32_t* __restrict__ tokens, int n, uint32_t vocab, uint32_t rank_blocks, const EmbedFill fill, int32_t* __restrict__ keys,
             int32_t* __restrict__ positions)
{
    if (blockIdx.x >= rank_blocks) {
        embed_fill(fill, blockIdx.x - rank_blocks);
        return;
    }
    __shared__ uint32_t part[kEmbedRankWaves][kLanes];
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const int block = blockIdx.x, t = block * kLanes + lane;
    const uint32_t key = t < n ? embed_key(tokens[t], vocab) : 0xffffffffu;
    const int chunks = (n + kLanes - 1) / kLanes;
    uint32_t before = 0;
    for (int c = wave; c < chunks; c += kEmbedRankWaves) {
        const int s0 = c * kLanes, len = min(kLanes, n - s0);
        const uint32_t limit = c < block ? key + 1 : key;   // positions of an earlier chunk come before equal ones of this
        if (c == block) {
            for (int s = 0; s < len; ++s) {
                const uint32_t other = embed_key(tokens[s0 + s], vocab);
                before += other < key || (other == key && s < lane);
            }
        } else if (len == kLanes) {
#pragma unroll 16
            for (int s = 0; s < kLanes; ++s) before += embed_key(tokens[s0 + s], vocab) < limit;
        } else {
            for (int s = 0; s < len; ++s) before += embed_key(tokens[s0 + s], vocab) < limit;
        }
    }
    part[wave][lane] = before;
    __syncthreads();
    if (wave > 0 || t >= n) return;
    before = 0;
#pragma unroll
    for (int w = 0; w < kEmbedRankWaves; ++w) before += part[w][lane];
    keys[before] = static_cast<int32_t>(key);               // (a permutation: below n)
    positions[before] = t;
}

// Sorting by digits of 9 bits, lowest first, two launches a digit.  k_embed_count: how often a block's tile has every digit.
__device__ __forceinline__ void embed_tile_counts(const uint32_t (&key)[kEmbedSortRows], bool (&there)[kEmbedSortRows], int shift, uint32_t* counts,
                                                  uint32_t (&rank)[kEmbedSortRows])
{
    // `counts`: this wave's, zero at first.  A wave's positions come in order: row after row of 64.
#pragma unroll
    for (int r = 0; r < kEmbedSortRows; ++r) {
        const uint32_t digit = key[r] >> shift & (kEmbedDigits - 1);
        uint64_t same = __ballot(there[r]);
#pragma unroll
        for (int b = 0; b < kEmbedDigit; ++b) {
            const uint64_t ones = __ballot(digit >> b & 1u);
            same &= digit >> b & 1u ? ones : ~ones;
        }
        rank[r] = 0;
        const uint32_t below = lanes_below(same);
        if (there[r]) rank[r] = counts[digit] + below;
        wave_lds_fence();
        if (there[r] && below == 0) counts[digit] += static_cast<uint32_t>(__popcll(same));
        wave_lds_fence();
    }
}

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
k_embed_count(const int32_t* __restrict__ tokens, const int32_t* __restrict__ keys, int n, uint32_t vocab, int shift, uint32_t sort_blocks,
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
        if (there[r]) atomicAdd(&counts[key[r] >> shift & (kEmbedDigits - 1)], 1u);
    __syncthreads();
    if (threadIdx.x < kEmbedDigits) table[blockIdx.x * kEmbedDigits + threadIdx.x] = counts[threadIdx.x];
}

// k_embed_place: every block adds up the tiles before its own and the digits before each (the table is a few kilobytes per tile) and
// moves its positions, equal digits in their order.
template <bool FIRST>
__global__ void __launch_bounds__(kEmbedSortBlock)
k_embed_place(const int32_t* __restrict__ tokens, const int32_t* __restrict__ keys, const int32_t* __restrict__ positions, int n, uint32_t vocab, int shift,
              uint32_t sort_blocks, const EmbedFill fill, const uint32_t* __restrict__ table, int32_t* __restrict__ keys_out,
              int32_t* __restrict__ positions_out)
{
    if (blockIdx.x >= sort_blocks) {
        embed_fill(fill, blockIdx.x - sort_blocks);
        return;
    }
    constexpr int kSortWaves = kEmbedSortBlock / kLanes;
    __shared__ uint32_t counts[kSortWaves][kEmbedDigits];
    __shared__ uint32_t halves[2][2][kEmbedDigits], base[kEmbedDigits], wave_total[kEmbedDigits / kLanes];
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    for (int i = threadIdx.x; i < kSortWaves * kEmbedDigits; i += kEmbedSortBlock) counts[0][i] = 0;
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
    uint32_t inclusive = 0, all = 0;
    if (threadIdx.x < kEmbedDigits) {
        all = halves[0][1][threadIdx.x] + halves[1][1][threadIdx.x];
        inclusive = all;
#pragma unroll
        for (int m = 1; m < kLanes; m *= 2) {
            const uint32_t v = __shfl_up(inclusive, m);
            if (lane >= m) inclusive += v;
        }
        if (lane == kLanes - 1) wave_total[wave] = inclusive;
    }
    __syncthreads();
    if (threadIdx.x < kEmbedDigits) {
        uint32_t first = inclusive - all + halves[0][0][threadIdx.x] + halves[1][0][threadIdx.x];
        for (int w = 0; w < wave; ++w) first += wave_total[w];
        base[threadIdx.x] = first;
    }
    uint32_t key[kEmbedSortRows], rank[kEmbedSortRows];
    int32_t position[kEmbedSortRows];
    bool there[kEmbedSortRows];
    embed_tile_keys<FIRST>(tokens, keys, positions, n, vocab, wave, lane, key, position, there);
    embed_tile_counts(key, there, shift, counts[wave], rank);
    __syncthreads();
    if (threadIdx.x < kEmbedDigits) {                       // counts become the first places of every wave
        uint32_t sum = base[threadIdx.x];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = counts[w][threadIdx.x];
            counts[w][threadIdx.x] = sum;
            sum += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kEmbedSortRows; ++r) {
        if (!there[r]) continue;
        const uint32_t to = counts[wave][key[r] >> shift & (kEmbedDigits - 1)] + rank[r];
        if (to >= static_cast<uint32_t>(n)) continue;       // (never: a permutation)
        keys_out[to] = static_cast<int32_t>(key[r]);
        positions_out[to] = position[r];
    }
}

// A row of the gradient: written, or added to what is there.
template <typename G>
__device__ __forceinline__ void embed_put(G* to, int n, bool aligned, bool add, float scale, const float4& s)
{
    if (aligned && n >= 4) {
        const float4 old = add ? cached4(to) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const float4 v = add ? make_float4(fmaf(scale, s.x, old.x), fmaf(scale, s.y, old.y), fmaf(scale, s.z, old.z), fmaf(scale, s.w, old.w))
                             : make_float4(scale * s.x, scale * s.y, scale * s.z, scale * s.w);
        store4(to, v);
        return;
    }
    const float e[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (c < n) put(to + c, add ? fmaf(scale, e[c], widen(to[c])) : scale * e[c]);
}

struct EmbedSums {
    const int32_t *keys, *positions;
    int32_t n, dim;
    uint32_t vocab, chunks;
    int64_t dout_stride, grad_stride;
    float scale;
    int32_t add, dout_aligned, grad_aligned;
    float* partial;                                         // per tile two rows of chunks * 256: of the run that began before it, of the one that goes on behind it
};

// Sums of the runs in a tile of kEmbedRun sorted positions, 256 columns per wave.  A run that lies in one tile goes to the gradient, the
// parts of longer ones to `partial`.
template <typename T, typename G>
__global__ void __launch_bounds__(kBlock)
k_embed_sums(const T* __restrict__ dout, G* __restrict__ grad, const EmbedSums a)
{
    const int lane = threadIdx.x % kLanes;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const uint32_t tile = item / a.chunks, chunk = item % a.chunks;
    const int p0 = static_cast<int>(tile) * kEmbedRun;
    if (p0 >= a.n) return;
    const int len = min(kEmbedRun, a.n - p0), col = static_cast<int>(chunk) * kWaveTile + lane * kVec;
    const int left = a.dim - col;                           // columns from here on; none: the lane reads and writes nothing
    const uint32_t before = p0 > 0 ? static_cast<uint32_t>(a.keys[p0 - 1]) : 0xffffffffu;
    const uint32_t after = p0 + len < a.n ? static_cast<uint32_t>(a.keys[p0 + len]) : 0xffffffffu;
    float4 v[kEmbedRun];
    uint32_t key[kEmbedRun];
#pragma unroll
    for (int i = 0; i < kEmbedRun; ++i) {
        key[i] = i < len ? static_cast<uint32_t>(a.keys[p0 + i]) : 0xffffffffu;
        v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (key[i] >= a.vocab || left <= 0) continue;
        const T* from = dout + a.positions[p0 + i] * a.dout_stride + col;
        if (a.dout_aligned && left >= 4) {
            v[i] = cached4(from);
        } else {
            float e[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) e[c] = c < left ? widen(from[c]) : 0.0f;
            v[i] = make_float4(e[0], e[1], e[2], e[3]);
        }
    }
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    bool from_before = key[0] == before;
    float* partial = a.partial + (static_cast<int64_t>(tile) * 2 * a.chunks + chunk) * kWaveTile + lane * kVec;
#pragma unroll
    for (int i = 0; i < kEmbedRun; ++i) {
        s.x += v[i].x;
        s.y += v[i].y;
        s.z += v[i].z;
        s.w += v[i].w;
        const uint32_t next = i + 1 < len ? key[i + 1 < kEmbedRun ? i + 1 : i] : after;
        if (i >= len || key[i] >= a.vocab) continue;        // (uniform)
        const bool last = i + 1 >= len;
        if (!last && next == key[i]) continue;
        const bool goes_on = last && next == key[i];
        if (from_before)
            *reinterpret_cast<float4*>(partial) = s;
        else if (goes_on)
            *reinterpret_cast<float4*>(partial + a.chunks * kWaveTile) = s;
        else if (left > 0)
            embed_put(grad + key[i] * a.grad_stride + col, left, a.grad_aligned != 0, a.add != 0, a.scale, s);
        s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        from_before = false;
    }
}

// Runs over several tiles: the block of the tile in which a run begins adds up its parts, every wave a quarter of the tiles in turn, in one order.
template <typename G>
__global__ void __launch_bounds__(kBlock)
k_embed_join(G* __restrict__ grad, const EmbedSums a, uint32_t tiles)
{
    __shared__ float4 lds[kWaves][kLanes];
    const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const uint32_t tile = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const int end = static_cast<int>(tile + 1) * kEmbedRun; // first position behind the tile (there is one: the last tile begins no such run)
    if (tile + 1 >= tiles) return;
    const uint32_t key = static_cast<uint32_t>(a.keys[end - 1]);
    if (key >= a.vocab || static_cast<uint32_t>(a.keys[end]) != key) return;
    if (end > kEmbedRun && static_cast<uint32_t>(a.keys[end - kEmbedRun]) == key && static_cast<uint32_t>(a.keys[end - kEmbedRun - 1]) == key)
        return;                                             // (it began in an earlier one)
    // the last tile that the run reaches: it holds the last position with this key
    const int64_t behind = end + wave_lower_bound(a.keys + end, a.n - end, static_cast<int64_t>(key) + 1);
    const uint32_t last = static_cast<uint32_t>((behind - 1) / kEmbedRun);
    const int64_t row = static_cast<int64_t>(a.chunks) * kWaveTile, at = static_cast<int64_t>(chunk) * kWaveTile + lane * kVec;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (wave == 0) s = cached4(a.partial + (static_cast<int64_t>(tile) * 2 + 1) * row + at);
#pragma unroll 8
    for (uint32_t t = tile + 1 + wave; t <= last; t += kWaves) {
        const float4 v = cached4(a.partial + static_cast<int64_t>(t) * 2 * row + at);
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
    }
    lds[wave][lane] = s;
    __syncthreads();
    const int col = static_cast<int>(at), left = a.dim - col;
    if (wave > 0 || left <= 0) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        const float4 v = lds[w][lane];
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
    }
    embed_put(grad + key * a.grad_stride + col, left, a.grad_aligned != 0, a.add != 0, a.scale, s);
}

}  // namespace
