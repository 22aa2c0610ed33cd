// Kernels of the dense optimiser operators: momentum from a compressed gradient, and the weight update per
// tensor.  Both are one pass over their vectors, bound by HBM traffic.  Part of scalecom.hip's single translation unit.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "device_helpers.h"
#include "geometry.h"

namespace {

__device__ __forceinline__ uint16_t bf16_bits(float x)      // round to nearest even; a NaN stays one
{
    const uint32_t b = __float_as_uint(x);
    if ((b & 0x7fffffffu) > 0x7f800000u) return static_cast<uint16_t>((b >> 16) | 0x40u);
    return static_cast<uint16_t>((b + 0x7fffu + ((b >> 16) & 1u)) >> 16);
}

__device__ __forceinline__ void store4(uint16_t* p, const float4& v)
{
    vu2_t w;
    w.x = bf16_bits(v.x) | static_cast<uint32_t>(bf16_bits(v.y)) << 16;
    w.y = bf16_bits(v.z) | static_cast<uint32_t>(bf16_bits(v.w)) << 16;
    __builtin_nontemporal_store(w, reinterpret_cast<vu2_t*>(p));
}

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = bf16_bits(x); }

template <typename T>
__device__ __forceinline__ void store_first(T* p, int64_t n, const float4& v)   // the first n of four values
{
    const float a[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (c < n) put(p + c, a[c]);
}

// First t in [0, k) with idx[t] >= target, k if there is none, for ascending idx: the 64 lanes of a wave probe 64 places at
// once, so a billion positions take five dependent loads.  Stays inside [0, k) whatever idx holds.
__device__ __forceinline__ int64_t wave_lower_bound(const int32_t* __restrict__ idx, int64_t k, int64_t target)
{
    const int lane = threadIdx.x % kLanes;
    int64_t lo = 0, hi = k;
    while (lo < hi) {                                       // (ends: what is left is shorter than one step)
        const int64_t step = (hi - lo + kLanes - 1) / kLanes, p = lo + lane * step;
        const int below = __popcll(__ballot(p < hi && idx[p] < target));
        if (below == 0) return lo;
        const int64_t end = lo + below * step;
        lo = end - step + 1;
        hi = end < hi ? end : hi;
    }
    return lo;
}

// The last of n ascending entries (the first is 0) that is not above `block`: where a block of a launch over several tensors
// belongs.  The lanes look at all entries at once, so a block waits for the arguments of its launch twice and not once per
// halving.  The same for all lanes.
__device__ __forceinline__ int find_block(const uint32_t* first, int n, uint32_t block)
{
    int below = 0;
    for (int base = 0; base < n; base += kLanes) {
        const int i = base + static_cast<int>(threadIdx.x % kLanes);
        below += __popcll(__ballot(i < n && first[i] <= block));
    }
    return __builtin_amdgcn_readfirstlane(below - 1);
}

// Momentum from a compressed gradient g (scale * vals[t] at idx[t], zero elsewhere):
//   m' = fma(mu, m, g);  u = NESTEROV ? fma(mu, m', g) : m'
// One pass: a block takes kMomentumTile positions, asks for their momentum, finds the members among them (idx is ascending,
// two waves search for the two ends while the loads are under way), spreads these over a tile of zeros in LDS and then
// goes over the tile.  U = void: no update is written.
// Bound by HBM: 25.6 M positions with a bfloat16 update 50 us (5.2 TB/s), 10^9 1.76 to 1.81 ms (5.6 TB/s; a copy of 4 GiB reaches 6.6).
// With nontemporal stores; ordinary ones, tiles of half or twice the size and an eighth of the vector per XCD were slower at 10^9.
// 200 003 positions take 6 us, of which the two searches and the launch are most.
constexpr int kMomentumRows = 4;                            // accesses of four positions per thread
constexpr int kMomentumTile = kBlock * kVec * kMomentumRows;

template <typename U, bool NESTEROV>
__global__ void __launch_bounds__(kBlock)
k_momentum(float* __restrict__ m, U* __restrict__ u, int64_t numel, const int32_t* __restrict__ idx,
           const float* __restrict__ vals, int64_t k, float scale, float mu)
{
    __shared__ __attribute__((aligned(16))) float g[kMomentumTile];
    __shared__ int64_t ends[2];
    const int64_t p0 = static_cast<int64_t>(blockIdx.x) * kMomentumTile;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    float4 x[kMomentumRows];
#pragma unroll
    for (int r = 0; r < kMomentumRows; ++r) {
        const int64_t p = p0 + (r * kBlock + static_cast<int>(threadIdx.x)) * kVec;
        x[r] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (p + 3 < numel)
            x[r] = load4(m + p);
        else if (p < numel)
            x[r] = load_guarded(m, p, 0, numel, false);
        *reinterpret_cast<float4*>(&g[(r * kBlock + threadIdx.x) * kVec]) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    if (wave < 2) {
        const int64_t end = wave_lower_bound(idx, k, p0 + wave * kMomentumTile);
        if (threadIdx.x % kLanes == 0) ends[wave] = end;
    }
    __syncthreads();
    for (int64_t t = ends[0] + threadIdx.x; t < ends[1]; t += kBlock) {
        const int64_t j = idx[t] - p0;
        if (j >= 0 && j < kMomentumTile) g[j] = scale * vals[t];   // (always, for ascending idx)
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kMomentumRows; ++r) {
        const int64_t p = p0 + (r * kBlock + static_cast<int>(threadIdx.x)) * kVec;
        if (p >= numel) continue;
        const float4 a = *reinterpret_cast<const float4*>(&g[(r * kBlock + threadIdx.x) * kVec]);
        const float4 n = make_float4(fmaf(mu, x[r].x, a.x), fmaf(mu, x[r].y, a.y), fmaf(mu, x[r].z, a.z), fmaf(mu, x[r].w, a.w));
        const bool full = p + 3 < numel;
        if (full)
            store4(m + p, n);
        else
            store_first(m + p, numel - p, n);
        if constexpr (!std::is_void<U>::value) {
            float4 w = n;
            if (NESTEROV) w = make_float4(fmaf(mu, n.x, a.x), fmaf(mu, n.y, a.y), fmaf(mu, n.z, a.z), fmaf(mu, n.w, a.w));
            if (full)
                store4(u + p, w);
            else
                store_first(u + p, numel - p, w);
        }
    }
}

// Weight update per tensor: theta = fma(-scale, update, decay * theta) on the rows of every tensor.
// The tensors of a launch travel with it (a launch's arguments are part of a captured graph, so nothing is copied and nothing
// is kept).  Rows that follow each other without a gap are one row.  Accesses of 16 bytes lie on multiples of four positions of
// the flat vector, so a row's first and last may be partial.
// Bound by HBM: 25.5 M weights in 54 matrices and two vectors with f32 updates 55 us (5.6 TB/s), 44 M in 96 matrices and a vector with bfloat16 updates 78 us
// (5.6 TB/s).
struct ApplyTensor {
    int64_t offset, stride, cols;
    uint32_t quads;                                         // accesses per row (0: more than fit, one row)
    float neg_scale;
    uint32_t rows;
};
constexpr int kApplyTensors = 90;                           // per launch: 3960 bytes of the 4096 that its arguments may have
constexpr int kApplyRows = 4;                               // accesses per thread
constexpr int kApplyQuads = kBlock * kApplyRows;            // and per block
constexpr int64_t kApplyBlocksMax = UINT32_MAX / kBlock;    // a launch has fewer than 2^32 threads

struct ApplyTable {
    uint32_t first[kApplyTensors];                          // block
    ApplyTensor t[kApplyTensors];
};

__host__ __device__ __forceinline__ int64_t row_quads(int64_t begin, int64_t cols)   // accesses that [begin, begin + cols) takes
{
    return (begin + cols - 1) / kVec - begin / kVec + 1;
}

template <typename U>
__global__ void __launch_bounds__(kBlock)
k_apply_tensors(float* __restrict__ theta, const U* __restrict__ update, float decay, int n, const ApplyTable table)
{
    const int at = find_block(table.first, n, blockIdx.x);
    const ApplyTensor t = table.t[at];
    const int64_t q0 = static_cast<int64_t>(blockIdx.x - table.first[at]) * kApplyQuads;
    const bool one = t.rows == 1;
    // (a row that begins elsewhere in its group of four may need one access less than `quads`: that one is empty)
    const int64_t row0 = one ? 0 : q0 / t.quads;
    const uint32_t rest = one ? 0 : static_cast<uint32_t>(q0 - row0 * t.quads);
    float4 w[kApplyRows], g[kApplyRows];
    int64_t at_[kApplyRows], begin_[kApplyRows];
#pragma unroll
    for (int r = 0; r < kApplyRows; ++r) {
        const uint32_t q = r * kBlock + threadIdx.x;
        const uint32_t down = one ? 0 : (rest + q) / t.quads;
        const int64_t row = row0 + down;
        const int64_t begin = t.offset + row * t.stride;
        const int64_t p = (begin & ~static_cast<int64_t>(kVec - 1)) + (one ? q0 + q : (rest + q) - down * t.quads) * static_cast<int64_t>(kVec);
        begin_[r] = begin;
        at_[r] = row < t.rows ? p : begin + t.cols;         // (past the end: nothing to do)
        leader_load<true>(theta, update, at_[r], begin, begin + t.cols, w[r], g[r]);
    }
#pragma unroll
    for (int r = 0; r < kApplyRows; ++r) {
        const int64_t end = begin_[r] + t.cols, p = at_[r];
        if (p >= end) continue;
        const float4 v = make_float4(fmaf(t.neg_scale, g[r].x, decay * w[r].x), fmaf(t.neg_scale, g[r].y, decay * w[r].y),
                                     fmaf(t.neg_scale, g[r].z, decay * w[r].z), fmaf(t.neg_scale, g[r].w, decay * w[r].w));
        store_guarded(theta, p, begin_[r], end, p >= begin_[r] && p + 3 < end, v);
    }
}

}  // namespace
