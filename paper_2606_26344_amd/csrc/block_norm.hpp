// Norms between two blocks (include/gmlp_block_norm.h) for gfx950.
//
// A group of threads takes a row at a time and holds it in registers, one
// 16-byte chunk per thread for widths up to 8192, so that every tensor is read
// and written once: forward two sums over the row (of squares of Y, then of the
// new residual row), backward two more that the chain rule of each norm needs.
// Bound by memory: 8 bytes per element forward, 12 backward, with a bf16 residual
// stream.  A block holds several row groups, and the next rows' loads are issued
// before the sums of the present ones.
//
// Blocks are persistent: they keep the gains in registers across their rows, and
// backward also the sums over the rows of the gains' gradients, which a block
// adds over its groups and writes once as fp32 partial sums for
// norm_columns_kernel to add in the order of the blocks.
// Measured, 4096 rows of 4096 in bf16: forward 24 to 27 us (134 MB, 5.0 to 5.6 TB/s),
// backward 41 to 44 and 5 for the columns (201 MB, 4.1 to 4.4 TB/s in all).  Above 8192
// columns a thread holds two chunks, which leave no registers for the next row or the
// gains: 4096 x 16384 forward 125 us (4.3 TB/s), backward 394 (2.0 TB/s).
#pragma once

#include "common.hpp"

namespace gmlp {

struct NormParams {
    const uint16_t *y;       // [T, D] or nullptr
    const void *res;         // forward: the residual stream; backward: R
    const uint16_t *w_pre, *w_post, *gate;
    size_t gate_stride;      // 0: one gate row for all
    void *r_out;             // forward
    uint16_t *xn;
    const uint16_t *dxn;     // backward
    const void *dr;
    uint16_t *dy;
    void *dres;
    uint16_t *dgate;         // [T, D]: written row by row
    float *partial;          // [2][blocks][D], see kNormSums
    int T, D, post, sums;    // sums: bit k: plane k of partial is wanted
    int row_threads, row_groups; // threads of a row (whole waves), rows of a block
    float res_scale, eps;
};

constexpr int kNormMaxThreads = 1024;

// Sums of N values over the threads of a row, in a fixed order, the same in all of
// them.  Calls alternate between two halves of `part` by `turn`, so that one
// barrier per call is enough; rows of one wave need none.
template <int N>
__device__ __forceinline__ void norm_row_sum(float (&v)[N], float *part, int &turn, int row_waves)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += __shfl_xor(v[i], off);
    if (row_waves == 1)
        return;
    const int wave = threadIdx.x >> 6;
    float *at = part + turn * (kNormMaxThreads / 64 * 4);
    turn ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i)
            at[wave * 4 + i] = v[i];
    __syncthreads();
    at += wave / row_waves * row_waves * 4;
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = at[i];
    for (int w = 1; w < row_waves; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += at[w * 4 + i];
}

// Eight neighbouring values of a row.
__device__ __forceinline__ void norm_unpack(const u32x4 &w, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = bf16_lo(w[e]);
        v[2 * e + 1] = bf16_hi(w[e]);
    }
}
__device__ __forceinline__ u32x4 norm_pack(const float (&v)[8])
{
    return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

// 16 bytes at byte `off` of a row (scalar base); kOutOfRange reads zeros and
// stores nothing.
__device__ __forceinline__ u32x4 norm_load(const void *row, uint32_t off, int more = 0)
{
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(row), off, more, 0));
}
__device__ __forceinline__ void norm_store(void *row, uint32_t off, const u32x4 &v, int more = 0)
{
    __builtin_amdgcn_raw_buffer_store_b128(v, make_rsrc(row), off, more, 0);
}

// The raw bits of eight values of the residual stream; `off` counts bytes of bf16.
template <bool F32>
struct NormRes {
    u32x4 w[F32 ? 2 : 1];
    __device__ __forceinline__ static uint32_t bytes(uint32_t off)
    {
        return F32 && off != kOutOfRange ? 2 * off : off;
    }
    __device__ __forceinline__ void load(const void *base, size_t row, uint32_t off)
    {
        if constexpr (F32) {
            w[0] = norm_load((const float *)base + row, bytes(off));
            w[1] = norm_load((const float *)base + row, bytes(off), 16);
        } else {
            w[0] = norm_load((const uint16_t *)base + row, off);
        }
    }
    __device__ __forceinline__ void zero()
    {
        w[0] = u32x4{};
        if constexpr (F32)
            w[1] = u32x4{};
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = __builtin_bit_cast(f32x4, w[e >> 2])[e & 3];
        } else {
            norm_unpack(w[0], v);
        }
    }
    __device__ __forceinline__ static void store(void *base, size_t row, uint32_t off, const float (&v)[8])
    {
        if constexpr (F32) {
            norm_store((float *)base + row, bytes(off), __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}));
            norm_store((float *)base + row, bytes(off), __builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]}), 16);
        } else {
            norm_store((uint16_t *)base + row, off, norm_pack(v));
        }
    }
};

// The two sums over the rows that the gradients of the gains and of a channel gate
// need: sum dXn xhat, which is dw_pre, and sum S yhat (sum dZ yhat with a gate per
// element), which times the channel gate is dw_post and times w_post the gate's
// gradient (without a norm after the block yhat = Y, w_post = 1).
constexpr int kNormSums = 2;

constexpr uint32_t kOneBf16x2 = 0x3f803f80u;

// A gain's chunk, or ones.
__device__ __forceinline__ u32x4 norm_gain(const uint16_t *w, uint32_t off)
{
    return w ? norm_load(w, off) : u32x4{kOneBf16x2, kOneBf16x2, kOneBf16x2, kOneBf16x2};
}

// The gains and the channel gate of a thread's chunks: in registers with one chunk,
// read again for every row (from the L2) with more.
template <int CHUNKS>
struct NormGains {
    u32x4 w_pre[CHUNKS], w_post[CHUNKS], gate[CHUNKS];
    __device__ __forceinline__ void load(const NormParams &p, int j, uint32_t off)
    {
        w_pre[j] = norm_gain(p.w_pre, off);
        w_post[j] = norm_gain(p.w_post, off);
        gate[j] = norm_gain(p.gate_stride ? nullptr : p.gate, off);
    }
};

// Chunk j of thread t of a row is at byte 16 (j row_threads + t); chunks past the row
// read zeros, which add nothing to the sums, and are not stored.  Row groups past
// the last row repeat it and store nothing (they take part in the barriers).
template <int CHUNKS, bool F32>
struct NormRow {
    u32x4 y[CHUNKS], gate[CHUNKS];
    NormRes<F32> r[CHUNKS];
    __device__ __forceinline__ void load(const NormParams &p, int t, const uint32_t (&off)[CHUNKS],
                                         const NormGains<CHUNKS> &gains)
    {
        const size_t row = (size_t)min(t, p.T - 1) * p.D;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            r[j].load(p.res, row, off[j]);
            y[j] = p.y ? norm_load(p.y + row, off[j]) : u32x4{};
            gate[j] = p.gate_stride ? norm_load(p.gate + row, off[j]) : gains.gate[j];
        }
    }
};

template <int CHUNKS, bool F32>
__global__ __launch_bounds__(kNormMaxThreads) void norm_forward_kernel(NormParams p)
{
    __shared__ float part[2 * kNormMaxThreads / 64 * 4];
    int turn = 0;
    const int D = p.D, row_waves = p.row_threads >> 6;
    // Whole waves make a row, so its index and its address are scalars.
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / p.row_threads);
    const int tid = threadIdx.x - group * p.row_threads;
    const float inv_d = 1.0f / (float)D;
    uint32_t off[CHUNKS];
    NormGains<CHUNKS> gains;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        off[j] = 8 * (j * p.row_threads + tid) < D ? 16u * (uint32_t)(j * p.row_threads + tid) : kOutOfRange;
        gains.load(p, j, off[j]);
    }
    const int step = gridDim.x * p.row_groups;
    NormRow<CHUNKS, F32> next;
    if constexpr (CHUNKS == 1)
        next.load(p, blockIdx.x * p.row_groups + group, off, gains);
    for (int t0 = blockIdx.x * p.row_groups; t0 < p.T; t0 += step) {
        const int t = t0 + group;
        const size_t row = (size_t)t * D;
        const bool live = t < p.T;
        if constexpr (CHUNKS > 1) {
            asm volatile("" ::: "memory"); // the gains are not kept in registers across rows
            for (int j = 0; j < CHUNKS; ++j)
                gains.load(p, j, off[j]);
            next.load(p, t, off, gains);
        }
        const NormRow<CHUNKS, F32> a = next;
        if (CHUNKS == 1 && t0 + step < p.T)
            next.load(p, t + step, off, gains);
        float ry = 1.0f;
        if (p.post) {
            float s[1] = {0.0f};
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                float y[8];
                norm_unpack(a.y[j], y);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    s[0] += y[e] * y[e];
            }
            norm_row_sum(s, part, turn, row_waves);
            ry = 1.0f / __builtin_sqrtf(s[0] * inv_d + p.eps);
        }
        float r[CHUNKS][8], s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float y[8], g[8], w[8];
            norm_unpack(a.y[j], y);
            norm_unpack(a.gate[j], g);
            norm_unpack(gains.w_post[j], w);
            a.r[j].get(r[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = p.post ? y[e] * ry * w[e] : y[e];
                r[j][e] = p.y ? p.res_scale * r[j][e] + g[e] * z : p.res_scale * r[j][e];
                s[0] += r[j][e] * r[j][e];
            }
            if (live && p.r_out)
                NormRes<F32>::store(p.r_out, row, off[j], r[j]);
        }
        norm_row_sum(s, part, turn, row_waves);
        const float rr = 1.0f / __builtin_sqrtf(s[0] * inv_d + p.eps);
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float w[8];
            norm_unpack(gains.w_pre[j], w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w[e] = r[j][e] * rr * w[e];
            if (live)
                norm_store(p.xn + row, off[j], norm_pack(w));
        }
    }
}

template <int CHUNKS, bool F32>
__global__ __launch_bounds__(kNormMaxThreads) void norm_backward_kernel(NormParams p)
{
    __shared__ float part[2 * kNormMaxThreads / 64 * 4];
    __shared__ float columns[kNormMaxThreads * 8]; // the groups' sums of one gradient
    int turn = 0;
    const int D = p.D, row_waves = p.row_threads >> 6;
    // Whole waves make a row, so its index and its address are scalars.
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / p.row_threads);
    const int tid = threadIdx.x - group * p.row_threads;
    const float inv_d = 1.0f / (float)D;
    uint32_t off[CHUNKS];
    NormGains<CHUNKS> gains;
    float s_pre[CHUNKS][8], s_mid[CHUNKS][8];
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        off[j] = 8 * (j * p.row_threads + tid) < D ? 16u * (uint32_t)(j * p.row_threads + tid) : kOutOfRange;
        gains.load(p, j, off[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            s_pre[j][e] = s_mid[j][e] = 0.0f;
    }
    struct Row {
        NormRow<CHUNKS, F32> a;
        u32x4 dxn[CHUNKS];
        NormRes<F32> dr[CHUNKS];
    };
    auto load = [&](Row &v, int t) __attribute__((always_inline)) {
        const size_t row = (size_t)min(t, p.T - 1) * D;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            v.dxn[j] = norm_load(p.dxn + row, off[j]);
            if (p.dr)
                v.dr[j].load(p.dr, row, off[j]);
            else
                v.dr[j].zero();
        }
        v.a.load(p, t, off, gains);
    };
    const int step = gridDim.x * p.row_groups;
    Row next;
    if constexpr (CHUNKS == 1)
        load(next, blockIdx.x * p.row_groups + group);
    for (int t0 = blockIdx.x * p.row_groups; t0 < p.T; t0 += step) {
        const int t = t0 + group;
        const size_t row = (size_t)t * D;
        const bool live = t < p.T;
        if constexpr (CHUNKS > 1) {
            asm volatile("" ::: "memory"); // the gains are not kept in registers across rows
            for (int j = 0; j < CHUNKS; ++j)
                gains.load(p, j, off[j]);
            load(next, t);
        }
        const Row v = next;
        if (CHUNKS == 1 && t0 + step < p.T)
            load(next, t + step);
        // Sums of R^2, a R and Y^2.
        float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float r[8], x[8], w[8], y[8];
            v.a.r[j].get(r);
            norm_unpack(v.dxn[j], x);
            norm_unpack(gains.w_pre[j], w);
            norm_unpack(v.a.y[j], y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[0] += r[e] * r[e];
                s[1] += x[e] * w[e] * r[e];
                s[2] += y[e] * y[e];
            }
        }
        norm_row_sum(s, part, turn, row_waves);
        const float rr = 1.0f / __builtin_sqrtf(s[0] * inv_d + p.eps);
        const float ry = p.post ? 1.0f / __builtin_sqrtf(s[2] * inv_d + p.eps) : 1.0f;
        const float c = s[1] * rr * inv_d; // mean(a xhat)
        // S, all of R's gradient, and the sum of b Y.
        float total[CHUNKS][8], sb[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float r[8], x[8], w[8], y[8], g[8], wp[8], out[8];
            v.a.r[j].get(r);
            norm_unpack(v.dxn[j], x);
            norm_unpack(gains.w_pre[j], w);
            norm_unpack(v.a.y[j], y);
            norm_unpack(v.a.gate[j], g);
            norm_unpack(gains.w_post[j], wp);
            v.dr[j].get(total[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xhat = r[e] * rr, yhat = y[e] * ry;
                total[j][e] += rr * (x[e] * w[e] - xhat * c);
                const float dz = total[j][e] * g[e];
                sb[0] += dz * wp[e] * y[e];
                if (live) {
                    s_pre[j][e] += x[e] * xhat;
                    s_mid[j][e] += (p.gate_stride ? dz : total[j][e]) * yhat;
                }
                out[e] = p.res_scale * total[j][e];
            }
            if (live && p.dres)
                NormRes<F32>::store(p.dres, row, off[j], out);
            if (live && p.dgate) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    out[e] = total[j][e] * (p.post ? y[e] * ry * wp[e] : y[e]);
                norm_store(p.dgate + row, off[j], norm_pack(out));
            }
        }
        float cb = 0.0f;
        if (p.post) {
            norm_row_sum(sb, part, turn, row_waves);
            cb = sb[0] * ry * inv_d; // mean(b yhat)
        }
        if (p.dy) {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                float y[8], g[8], wp[8], out[8];
                norm_unpack(v.a.y[j], y);
                norm_unpack(v.a.gate[j], g);
                norm_unpack(gains.w_post[j], wp);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float dz = total[j][e] * g[e];
                    out[e] = p.post ? ry * (dz * wp[e] - y[e] * ry * cb) : dz;
                }
                if (live)
                    norm_store(p.dy + row, off[j], norm_pack(out));
            }
        }
    }
    // The groups' sums, in their order, then one partial row per block.
    const size_t plane = (size_t)gridDim.x * D;
#pragma unroll
    for (int k = 0; k < kNormSums; ++k) {
        if (!(p.sums >> k & 1))
            continue;
        float *out = p.partial + k * plane + (size_t)blockIdx.x * D;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float(&v)[8] = k == 0 ? s_pre[j] : s_mid[j];
            if (p.row_groups > 1) {
                __syncthreads(); // the sums of the turn before have been read
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    columns[e * kNormMaxThreads + threadIdx.x] = v[e];
                __syncthreads();
                if (group == 0)
                    for (int g = 1; g < p.row_groups; ++g)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            v[e] += columns[e * kNormMaxThreads + g * p.row_threads + tid];
            }
            if (group == 0)
                NormRes<true>::store(out, 0, off[j], v);
        }
    }
}

// Plane blockIdx.y of the partial sums, added over the blocks: 32 columns per
// block, 16 groups of partial rows, each with 8 loads in flight; the groups' sums
// in order.  Plane 1, times the channel gate (w_post), is dw_post (dgate); of no rows
// (no blocks) all are zeros, whatever the gate is.
struct NormColumns {
    const float *partial;
    const uint16_t *w_post, *gate; // nullptr: ones
    uint16_t *dw_pre, *dw_post, *dgate;
    int blocks, D;
};
constexpr int kNormColumns = 32, kNormGroups = 16;
__global__ __launch_bounds__(kNormColumns *kNormGroups) void norm_columns_kernel(NormColumns p)
{
    __shared__ float sum[kNormGroups][kNormColumns];
    const int k = blockIdx.y;
    if (k == 0 ? !p.dw_pre : !p.dw_post && !p.dgate) // the same for the whole block
        return;
    const int col = threadIdx.x % kNormColumns, group = threadIdx.x / kNormColumns;
    const int d = blockIdx.x * kNormColumns + col;
    float s = 0.0f;
    if (d < p.D) {
        const float *at = p.partial + (size_t)k * p.blocks * p.D + d;
#pragma unroll 8
        for (int b = group; b < p.blocks; b += kNormGroups)
            s += at[(size_t)b * p.D];
    }
    sum[group][col] = s;
    __syncthreads();
    if (group != 0 || d >= p.D)
        return;
#pragma unroll
    for (int g = 1; g < kNormGroups; ++g)
        s += sum[g][col];
    const auto bf16 = [](float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); };
    if (k == 0) {
        p.dw_pre[d] = bf16(s);
        return;
    }
    if (p.dw_post)
        p.dw_post[d] = bf16(p.gate && p.blocks ? s * bf16_lo(p.gate[d]) : s);
    if (p.dgate)
        p.dgate[d] = bf16(p.w_post && p.blocks ? s * bf16_lo(p.w_post[d]) : s);
}

} // namespace gmlp
