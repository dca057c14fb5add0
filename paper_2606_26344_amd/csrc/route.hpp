// Tokens sorted by expert and back, for gfx950.
//
// The sort is a stable counting sort in one launch: its results are whole numbers, so
// any order of the counting gives the same.  Rows are moved token by token: a token's
// row is read once and written to (or summed from) the k rows of its slots.
#pragma once

#include <type_traits>

#include "common.hpp"

namespace gmlp {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMaxExperts = 1024;
constexpr int kRouteThreads = 256;

struct SortParams {
    const void *ids;
    int32_t *offsets, *slots;
    int n;     // assignments
    int chunk; // of a block, a multiple of kSortThreads
    int experts;
    int bits; // that tell experts apart
};

template <class Id>
__device__ __forceinline__ int expert_of(const void *ids, int i, int experts)
{
    const Id v = static_cast<const Id *>(ids)[i];
    return v >= 0 && v < (Id)experts ? (int)v : -1;
}

// A block ranks its chunk of the assignments, its waves a sixteenth of that each, and
// counts all others: those before the chunk and those behind it.  So no block waits for
// another, at n / 1024 loads per thread in each.
template <class Id>
__global__ __launch_bounds__(kSortThreads) void route_sort_kernel(SortParams p)
{
    __shared__ uint32_t mine[kSortWaves][kMaxExperts]; // of a wave: counts, then its next slots
    __shared__ uint32_t before[kMaxExperts], behind[kMaxExperts];
    __shared__ uint32_t wave_sum[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = p.experts;
    for (int e = tid; e < E; e += kSortThreads) {
        before[e] = behind[e] = 0;
        for (int w = 0; w < kSortWaves; ++w)
            mine[w][e] = 0;
    }
    __syncthreads();
    const int lo = min(p.n, (int)blockIdx.x * p.chunk), hi = min(p.n, lo + p.chunk);
    for (int i = tid; i < lo; i += kSortThreads) {
        const int e = expert_of<Id>(p.ids, i, E);
        if (e >= 0)
            atomicAdd(&before[e], 1u);
    }
    for (int i = hi + tid; i < p.n; i += kSortThreads) {
        const int e = expert_of<Id>(p.ids, i, E);
        if (e >= 0)
            atomicAdd(&behind[e], 1u);
    }
    const int part = p.chunk / kSortWaves, first = lo + wave * part, last = min(hi, first + part);
    for (int i = first + lane; i < last; i += 64) {
        const int e = expert_of<Id>(p.ids, i, E);
        if (e >= 0)
            atomicAdd(&mine[wave][e], 1u);
    }
    __syncthreads();

    // Where each expert's rows begin (a thread per expert), and in them this block's
    // and its waves'.
    uint32_t total = 0, earlier = 0;
    if (tid < E) {
        earlier = before[tid];
        total = earlier + behind[tid];
        for (int w = 0; w < kSortWaves; ++w)
            total += mine[w][tid];
    }
    uint32_t sum = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(sum, d);
        sum += lane >= d ? up : 0;
    }
    if (lane == 63)
        wave_sum[wave] = sum;
    __syncthreads();
    uint32_t start = sum - total;
    for (int w = 0; w < wave; ++w)
        start += wave_sum[w];
    if (tid < E) {
        if (blockIdx.x == 0) {
            p.offsets[tid] = (int32_t)start;
            if (tid == E - 1)
                p.offsets[E] = (int32_t)(start + total);
        }
        uint32_t at = start + earlier;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = mine[w][tid];
            mine[w][tid] = at;
            at += c;
        }
    }
    __syncthreads();

    // Ranks within 64 assignments: the lanes of the same expert, from one vote per bit.
    for (int i0 = first; i0 < last; i0 += 64) {
        const int i = i0 + lane;
        const int e = i < last ? expert_of<Id>(p.ids, i, E) : -1;
        uint64_t same = __ballot(e >= 0);
        for (int b = 0; b < p.bits; ++b) {
            const uint64_t set = __ballot(e >> b & 1);
            same &= e >> b & 1 ? set : ~set;
        }
        const uint64_t below = same & ((uint64_t(1) << lane) - 1);
        const uint32_t at = e >= 0 ? mine[wave][e] : 0;
        wave_lds_fence();
        if (e >= 0 && below == 0) // the first of them moves the slot on for all
            mine[wave][e] = at + (uint32_t)__popcll(same);
        wave_lds_fence();
        if (i < last)
            p.slots[i] = e >= 0 ? (int32_t)(at + (uint32_t)__popcll(below)) : -1;
    }
}

struct RouteParams {
    const uint16_t *rows; // x of dispatch; ys
    const uint16_t *dy;   // of the backward pass
    uint16_t *out;        // xs, y or dys
    const int32_t *slots;
    const void *weights; // fp32 or bf16
    void *dweights;
    int tokens, choices, n; // n = tokens * choices
    int chunks;             // 16-byte chunks of a row
    int lanes_log;          // log2 of the threads of a row
};

// The slot of assignment i, or -1.
__device__ __forceinline__ int slot_of(const RouteParams &p, int i)
{
    const int s = p.slots[i];
    return (uint32_t)s < (uint32_t)p.n ? s : -1;
}

template <bool BF16>
__device__ __forceinline__ float weight_of(const RouteParams &p, int i)
{
    if constexpr (BF16)
        return bf16_lo(static_cast<const uint16_t *>(p.weights)[i]);
    else
        return static_cast<const float *>(p.weights)[i];
}

__device__ __forceinline__ const u32x4 *row_chunks(const uint16_t *base, int row, int chunks)
{
    return reinterpret_cast<const u32x4 *>(base) + (size_t)row * chunks;
}
__device__ __forceinline__ u32x4 *row_chunks(uint16_t *base, int row, int chunks)
{
    return reinterpret_cast<u32x4 *>(base) + (size_t)row * chunks;
}

// xs[slot] = x: 1 << lanes_log threads of a block move one token's row.
__global__ __launch_bounds__(kRouteThreads) void route_dispatch_kernel(RouteParams p)
{
    const int lanes = 1 << p.lanes_log;
    const int t = (int)blockIdx.x * (kRouteThreads >> p.lanes_log) + (threadIdx.x >> p.lanes_log);
    if (t >= p.tokens)
        return;
    const u32x4 *x = row_chunks(p.rows, t, p.chunks);
    for (int c = threadIdx.x & (lanes - 1); c < p.chunks; c += lanes) {
        const u32x4 v = x[c];
        for (int j = 0; j < p.choices; ++j) {
            const int s = slot_of(p, t * p.choices + j);
            if (s >= 0)
                row_chunks(p.out, s, p.chunks)[c] = v;
        }
    }
}

enum RouteWeights { ROUTE_ONES, ROUTE_FP32, ROUTE_BF16 };

// y = sum_j w_j ys[slot_j], eight columns per thread; up to J rows on their way at once.
template <int J, int WEIGHTS>
__global__ __launch_bounds__(kRouteThreads) void route_combine_kernel(RouteParams p)
{
    const int lanes = 1 << p.lanes_log;
    const int t = (int)blockIdx.x * (kRouteThreads >> p.lanes_log) + (threadIdx.x >> p.lanes_log);
    if (t >= p.tokens)
        return;
    for (int c = threadIdx.x & (lanes - 1); c < p.chunks; c += lanes) {
        float y[8] = {};
        for (int j0 = 0; j0 < p.choices; j0 += J) {
            u32x4 v[J];
            float w[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int i = t * p.choices + j0 + j;
                const int s = j0 + j < p.choices ? slot_of(p, i) : -1;
                v[j] = u32x4{};
                w[j] = 0.0f;
                if (s >= 0) {
                    v[j] = row_chunks(p.rows, s, p.chunks)[c];
                    w[j] = WEIGHTS == ROUTE_ONES ? 1.0f : weight_of<WEIGHTS == ROUTE_BF16>(p, i);
                }
            }
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    y[2 * q] += w[j] * bf16_lo(v[j][q]);
                    y[2 * q + 1] += w[j] * bf16_hi(v[j][q]);
                }
        }
        row_chunks(p.out, t, p.chunks)[c] =
            u32x4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
    }
}

// dys[slot_j] = w_j dy and dw_j = dy . ys[slot_j]: W waves of a block per token, a lane
// takes every 64 W-th chunk; the sums of its choices' products stay in registers, J
// choices at a time.
template <int J, int W, bool BF16>
__global__ __launch_bounds__(kRouteThreads) void route_combine_backward_kernel(RouteParams p)
{
    constexpr int TOKENS = kRouteThreads / 64 / W; // of a block
    __shared__ float sums[kRouteThreads / 64][J];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = wave % W;
    const int t = (int)blockIdx.x * TOKENS + wave / W;
    const bool in = t < p.tokens;
    for (int j0 = 0; j0 < p.choices; j0 += J) {
        int slot[J];
        float w[J], dot[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int i = t * p.choices + j0 + j;
            slot[j] = in && j0 + j < p.choices ? slot_of(p, i) : -1;
            w[j] = slot[j] >= 0 ? weight_of<BF16>(p, i) : 0.0f;
            dot[j] = 0.0f;
        }
        if (in)
            for (int c = part * 64 + lane; c < p.chunks; c += 64 * W) {
                const u32x4 d = row_chunks(p.dy, t, p.chunks)[c];
                u32x4 v[J];
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    v[j] = u32x4{};
                    if (slot[j] >= 0 && p.dweights)
                        v[j] = row_chunks(p.rows, slot[j], p.chunks)[c];
                }
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    u32x4 o;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float lo = bf16_lo(d[q]), hi = bf16_hi(d[q]);
                        if (slot[j] >= 0) { // 0 * NaN of a token without a row is no product
                            dot[j] += lo * bf16_lo(v[j][q]);
                            dot[j] += hi * bf16_hi(v[j][q]);
                        }
                        o[q] = pack_bf16x2(w[j] * lo, w[j] * hi);
                    }
                    if (slot[j] >= 0 && p.out)
                        row_chunks(p.out, slot[j], p.chunks)[c] = o;
                }
            }
        if (!p.dweights)
            continue;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int d = 1; d < 64; d <<= 1)
                dot[j] += __shfl_xor(dot[j], d);
        if constexpr (W > 1) {
            if (lane == 0)
#pragma unroll
                for (int j = 0; j < J; ++j)
                    sums[wave][j] = dot[j];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < J; ++j) {
                dot[j] = sums[wave - part][j];
#pragma unroll
                for (int q = 1; q < W; ++q)
                    dot[j] += sums[wave - part + q][j];
            }
            __syncthreads();
        }
        if (in && part == 0 && lane == 0)
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (j0 + j < p.choices) {
                    const int i = t * p.choices + j0 + j;
                    if constexpr (BF16)
                        static_cast<uint16_t *>(p.dweights)[i] = (uint16_t)pack_bf16x2(dot[j], 0.0f);
                    else
                        static_cast<float *>(p.dweights)[i] = dot[j];
                }
    }
}

} // namespace gmlp
