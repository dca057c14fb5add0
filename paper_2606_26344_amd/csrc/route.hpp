// Tokens sorted by expert and back, for gfx950.
//
// The sort is a stable counting sort: its results are whole numbers, so any order of the
// counting gives the same.  Rows are moved token by token: a token's
// row is read once and written to (or summed from) the k rows of its slots.  They are
// bound by the memory (us, TB/s): 4096 tokens of 4096 columns, dispatch to 2 rows each 16.5,
// 6.1; combine of 8 rows each 63.8, 4.7; its gradients 108.6, 5.3, where a copy takes 5.1.
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
    int n;      // assignments
    int chunk;  // of a block, a multiple of kSortThreads
    int blocks; // the last one takes what is behind the others' chunks too
    int experts;
    int bits; // that tell experts apart
};

template <class Id>
__device__ __forceinline__ int expert_of(const void *ids, int i, int experts)
{
    const Id v = static_cast<const Id *>(ids)[i];
    return v >= 0 && v < (Id)experts ? (int)v : -1;
}

// Counts the assignments begin + step 0, 1, .. below end, eight loads on their way at
// once.  counts: `stride` words to an expert.
template <class Id>
__device__ __forceinline__ void count_experts(const SortParams &p, uint32_t *counts, int stride, int begin, int end, int step)
{
    for (int i0 = begin; i0 < end; i0 += 8 * step) {
        int e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            e[j] = i0 + j * step < end ? expert_of<Id>(p.ids, i0 + j * step, p.experts) : -1;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (e[j] >= 0)
                atomicAdd(&counts[e[j] * stride], 1u);
    }
}

// The sum over the threads before this one.
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t (&wave_sum)[kSortWaves])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t sum = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(sum, d);
        sum += lane >= d ? up : 0;
    }
    if (lane == 63)
        wave_sum[wave] = sum;
    __syncthreads();
    sum -= v;
    for (int w = 0; w < wave; ++w)
        sum += wave_sum[w];
    return sum;
}

// A block's assignments: a sixteenth for each wave, whole rounds of 64.
struct SortRange {
    int lo, hi, first, last; // of the block, of this wave
};
__device__ __forceinline__ SortRange sort_range(const SortParams &p)
{
    SortRange r;
    r.lo = (int)blockIdx.x * p.chunk;
    r.hi = (int)blockIdx.x + 1 == p.blocks ? p.n : r.lo + p.chunk;
    const int part = (r.hi - r.lo + kSortThreads - 1) / kSortThreads * 64;
    r.first = min(r.hi, r.lo + (int)(threadIdx.x >> 6) * part);
    r.last = min(r.hi, r.first + part);
    return r;
}

// The slots of a wave's assignments, `next` its next slot of every expert.  Ranks within
// 64 of them: the lanes of the same expert, from one vote per bit.
template <class Id>
__device__ __forceinline__ void place_slots(const SortParams &p, const SortRange &r, uint32_t *next)
{
    const int lane = threadIdx.x & 63;
    for (int i0 = r.first; i0 < r.last; i0 += 64) {
        const int i = i0 + lane;
        const int e = i < r.last ? expert_of<Id>(p.ids, i, p.experts) : -1;
        uint64_t same = __ballot(e >= 0);
        for (int b = 0; b < p.bits; ++b) {
            const uint64_t set = __ballot(e >> b & 1);
            same &= e >> b & 1 ? set : ~set;
        }
        const uint64_t below = same & ((uint64_t(1) << lane) - 1);
        const uint32_t at = e >= 0 ? next[e] : 0;
        wave_lds_fence();
        if (e >= 0 && below == 0) // the first of them moves the slot on for all
            next[e] = at + (uint32_t)__popcll(same);
        wave_lds_fence();
        if (i < r.last)
            p.slots[i] = e >= 0 ? (int32_t)(at + (uint32_t)__popcll(below)) : -1;
    }
}

// Up to kSortOneLaunch assignments: a block ranks its chunk, its waves a sixteenth of
// that each, and counts all others, those before the chunk and those behind it.  So no
// block waits for another, but each reads everything, at 50 GB/s for each CU: us, one
// launch against three, 8 experts and 8192 assignments 5.6 and 15.2, 64 and 32768 9.7 and
// 10.1, 64 and 65536 15.5 and 10.1, 128 and 524288 95 and 14.5.
template <class Id>
__global__ __launch_bounds__(kSortThreads) void route_sort_kernel(SortParams p)
{
    __shared__ uint32_t mine[kSortWaves][kMaxExperts]; // of a wave: counts, then its next slots
    // Four counters each, since lanes that add to one counter take turns (65536 assignments
    // to one expert 24 us, with one counter 60).
    __shared__ uint32_t before[kMaxExperts][4], behind[kMaxExperts][4];
    __shared__ uint32_t wave_sum[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = p.experts;
    for (int e = tid; e < E; e += kSortThreads) {
        for (int c = 0; c < 4; ++c)
            before[e][c] = behind[e][c] = 0;
        for (int w = 0; w < kSortWaves; ++w)
            mine[w][e] = 0;
    }
    __syncthreads();
    const SortRange r = sort_range(p);
    count_experts<Id>(p, &before[0][lane & 3], 4, tid, r.lo, kSortThreads);
    count_experts<Id>(p, &behind[0][lane & 3], 4, r.hi + tid, p.n, kSortThreads);
    count_experts<Id>(p, mine[wave], 1, r.first + lane, r.last, 64);
    __syncthreads();

    // Where each expert's rows begin (a thread per expert), and in them this block's
    // and its waves'.
    uint32_t total = 0, earlier = 0;
    if (tid < E) {
        for (int c = 0; c < 4; ++c) {
            earlier += before[tid][c];
            total += behind[tid][c];
        }
        total += earlier;
        for (int w = 0; w < kSortWaves; ++w)
            total += mine[w][tid];
    }
    const uint32_t start = sum_before(total, wave_sum);
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
    place_slots<Id>(p, r, mine[wave]);
}

// More assignments, in three launches: each block's counts, then where its rows of each
// expert begin, are kept in its own part of the slots (a chunk is no less than the
// experts), until the last launch has read them.
constexpr int kSortOneLaunch = 1 << 15;

template <class Id>
__global__ __launch_bounds__(kSortThreads) void route_count_kernel(SortParams p)
{
    __shared__ uint32_t counts[kMaxExperts][4];
    const int tid = threadIdx.x;
    for (int e = tid; e < p.experts; e += kSortThreads)
        for (int c = 0; c < 4; ++c)
            counts[e][c] = 0;
    __syncthreads();
    const SortRange r = sort_range(p);
    count_experts<Id>(p, &counts[0][tid & 3], 4, r.lo + tid, r.hi, kSortThreads);
    __syncthreads();
    for (int e = tid; e < p.experts; e += kSortThreads)
        p.slots[r.lo + e] = (int32_t)(counts[e][0] + counts[e][1] + counts[e][2] + counts[e][3]);
}

// One block: 1 << bits threads walk the experts' counts of a run of blocks.
__global__ __launch_bounds__(kSortThreads) void route_scan_kernel(SortParams p)
{
    __shared__ uint32_t part[kSortThreads]; // counts of an expert in a run of blocks, then their sums
    __shared__ uint32_t wave_sum[kSortWaves];
    const int tid = threadIdx.x, E = p.experts;
    const int e = tid & ((1 << p.bits) - 1), run = tid >> p.bits, runs = min(kSortThreads >> p.bits, p.blocks);
    const int per = (p.blocks + runs - 1) / runs, first = min(p.blocks, run * per), last = min(p.blocks, first + per);
    uint32_t sum = 0;
    if (e < E)
        for (int b0 = first; b0 < last; b0 += 8)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                sum += b0 + j < last ? (uint32_t)p.slots[(size_t)(b0 + j) * p.chunk + e] : 0;
    part[tid] = sum;
    __syncthreads();
    uint32_t total = 0;
    if (tid < E)
        for (int r = 0; r < runs; ++r) {
            const uint32_t c = part[(r << p.bits) + tid];
            part[(r << p.bits) + tid] = total;
            total += c;
        }
    const uint32_t start = sum_before(total, wave_sum);
    if (tid < E) {
        p.offsets[tid] = (int32_t)start;
        if (tid == E - 1)
            p.offsets[E] = (int32_t)(start + total);
        for (int r = 0; r < runs; ++r)
            part[(r << p.bits) + tid] += start;
    }
    __syncthreads();
    uint32_t at = part[tid];
    if (e < E)
        for (int b0 = first; b0 < last; b0 += 8) {
            uint32_t c[8]; // eight blocks' on their way at once
#pragma unroll
            for (int j = 0; j < 8; ++j)
                c[j] = b0 + j < last ? (uint32_t)p.slots[(size_t)(b0 + j) * p.chunk + e] : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (b0 + j < last)
                    p.slots[(size_t)(b0 + j) * p.chunk + e] = (int32_t)at;
                at += c[j];
            }
        }
}

template <class Id>
__global__ __launch_bounds__(kSortThreads) void route_place_kernel(SortParams p)
{
    __shared__ uint32_t mine[kSortWaves][kMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = p.experts;
    for (int e = tid; e < E; e += kSortThreads)
        for (int w = 0; w < kSortWaves; ++w)
            mine[w][e] = 0;
    __syncthreads();
    const SortRange r = sort_range(p);
    count_experts<Id>(p, mine[wave], 1, r.first + lane, r.last, 64);
    __syncthreads();
    for (int e = tid; e < E; e += kSortThreads) {
        uint32_t at = (uint32_t)p.slots[r.lo + e];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = mine[w][e];
            mine[w][e] = at;
            at += c;
        }
    }
    __syncthreads(); // every thread has read the starts, which slots take the place of
    place_slots<Id>(p, r, mine[wave]);
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
// Sorted rows are read once, and pass the L2 where they are more than it holds.
template <bool ONCE>
__device__ __forceinline__ u32x4 load_row(const u32x4 *p)
{
    return ONCE ? __builtin_nontemporal_load(p) : *p;
}
// They are written for another kernel: dispatch of 4096 tokens to 8 rows each 66 us, through
// the L2 80.
__device__ __forceinline__ void store_row(u32x4 *p, const u32x4 &v) { __builtin_nontemporal_store(v, p); }

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
                store_row(row_chunks(p.out, s, p.chunks) + c, v);
        }
    }
}

enum RouteWeights { ROUTE_ONES, ROUTE_FP32, ROUTE_BF16 };

// y = sum_j w_j ys[slot_j], eight columns per thread; up to J rows on their way at once.
template <int J, int WEIGHTS, bool ONCE>
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
                    v[j] = load_row<ONCE>(row_chunks(p.rows, s, p.chunks) + c);
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
template <int J, int W, bool BF16, bool ONCE>
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
                        v[j] = load_row<ONCE>(row_chunks(p.rows, slot[j], p.chunks) + c);
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
                        store_row(row_chunks(p.out, slot[j], p.chunks) + c, o);
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
