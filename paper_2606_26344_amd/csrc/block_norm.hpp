// Norms between two blocks (include/gmlp_block_norm.h) for gfx950.
//
// One block of threads takes a row at a time and holds it in registers, so that
// every tensor is read and written once: forward two sums over the row (of
// squares of Y, then of the new residual row), backward two more that the chain
// rule of each norm needs.  Bound by memory: 8 bytes per element forward, 12
// backward, with a bf16 residual stream.
//
// Blocks are persistent: a block takes rows blockIdx, blockIdx + gridDim, ...,
// keeps the gains in registers across them, and backward also the sums over
// its rows of the gains' gradients, which it writes once as fp32 partial sums
// for norm_columns_kernel to add in the order of the blocks.
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
    float *partial;          // [3][blocks][D]: dw_pre, dw_post, dgate (channel)
    int T, D, post, sums;    // sums: bit 0 dw_pre, 1 dw_post, 2 dgate of a channel gate
    float res_scale, eps;
};

// Sums of N values over the block, in a fixed order, the same in every thread.
// Calls alternate between two halves of `part` by `turn`, so that one barrier
// per call is enough.
template <int THREADS, int N>
__device__ __forceinline__ void norm_block_sum(float (&v)[N], float *part, int &turn)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += __shfl_xor(v[i], off);
    if constexpr (THREADS > 64) {
        constexpr int WAVES = THREADS / 64;
        float *at = part + turn * (WAVES * 4);
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                at[(threadIdx.x >> 6) * 4 + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = at[i];
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
                s += at[w * 4 + i];
            v[i] = s;
        }
    }
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

// The raw bits of eight values of the residual stream.
template <bool F32>
struct NormRes {
    u32x4 w[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void *base, size_t at)
    {
        if constexpr (F32) {
            const u32x4 *p = (const u32x4 *)((const float *)base + at);
            w[0] = p[0];
            w[1] = p[1];
        } else {
            w[0] = *(const u32x4 *)((const uint16_t *)base + at);
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
    __device__ __forceinline__ static void store(void *base, size_t at, const float (&v)[8])
    {
        if constexpr (F32) {
            f32x4 *p = (f32x4 *)((float *)base + at);
            p[0] = f32x4{v[0], v[1], v[2], v[3]};
            p[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
            *(u32x4 *)((uint16_t *)base + at) = norm_pack(v);
        }
    }
};

constexpr uint32_t kOneBf16x2 = 0x3f803f80u;

// A gain's chunk, or ones.
__device__ __forceinline__ u32x4 norm_gain(const uint16_t *w, int at)
{
    return w ? *(const u32x4 *)(w + at) : u32x4{kOneBf16x2, kOneBf16x2, kOneBf16x2, kOneBf16x2};
}

// Chunk j of thread t covers elements 8 (j THREADS + t) ..; chunks past the row
// hold zeros with gains of one, which add nothing to the sums, and are not stored.
template <int THREADS, int CHUNKS, bool F32>
__global__ __launch_bounds__(THREADS) void norm_forward_kernel(NormParams p)
{
    __shared__ float part[2 * 4 * (THREADS / 64)];
    int turn = 0;
    const int tid = threadIdx.x, D = p.D;
    const float inv_d = 1.0f / (float)D;
    int at[CHUNKS];
    bool in[CHUNKS];
    u32x4 wpre[CHUNKS], wpost[CHUNKS], gch[CHUNKS];
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        at[j] = 8 * (j * THREADS + tid);
        in[j] = at[j] < D;
        wpre[j] = norm_gain(in[j] ? p.w_pre : nullptr, at[j]);
        wpost[j] = norm_gain(in[j] ? p.w_post : nullptr, at[j]);
        gch[j] = norm_gain(in[j] && !p.gate_stride ? p.gate : nullptr, at[j]);
    }
    for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
        const size_t row = (size_t)t * D;
        u32x4 yw[CHUNKS], gw[CHUNKS];
        NormRes<F32> rw[CHUNKS];
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            yw[j] = u32x4{};
            rw[j].zero();
            gw[j] = gch[j];
            if (in[j]) {
                rw[j].load(p.res, row + at[j]);
                if (p.y)
                    yw[j] = *(const u32x4 *)(p.y + row + at[j]);
                if (p.gate_stride)
                    gw[j] = *(const u32x4 *)(p.gate + row + at[j]);
            }
        }
        float ry = 1.0f;
        if (p.post) {
            float s[1] = {0.0f};
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                float y[8];
                norm_unpack(yw[j], y);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    s[0] += y[e] * y[e];
            }
            norm_block_sum<THREADS>(s, part, turn);
            ry = 1.0f / __builtin_sqrtf(s[0] * inv_d + p.eps);
        }
        float r[CHUNKS][8], s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float y[8], g[8], w[8];
            norm_unpack(yw[j], y);
            norm_unpack(gw[j], g);
            norm_unpack(wpost[j], w);
            rw[j].get(r[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = p.post ? y[e] * ry * w[e] : y[e];
                r[j][e] = p.y ? p.res_scale * r[j][e] + g[e] * z : p.res_scale * r[j][e];
                s[0] += r[j][e] * r[j][e];
            }
            if (in[j] && p.r_out)
                NormRes<F32>::store(p.r_out, row + at[j], r[j]);
        }
        norm_block_sum<THREADS>(s, part, turn);
        const float rr = 1.0f / __builtin_sqrtf(s[0] * inv_d + p.eps);
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float w[8];
            norm_unpack(wpre[j], w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w[e] = r[j][e] * rr * w[e];
            if (in[j])
                *(u32x4 *)(p.xn + row + at[j]) = norm_pack(w);
        }
    }
}

template <int THREADS, int CHUNKS, bool F32>
__global__ __launch_bounds__(THREADS) void norm_backward_kernel(NormParams p)
{
    __shared__ float part[2 * 4 * (THREADS / 64)];
    int turn = 0;
    const int tid = threadIdx.x, D = p.D;
    const float inv_d = 1.0f / (float)D;
    int at[CHUNKS];
    bool in[CHUNKS];
    u32x4 wpre[CHUNKS], wpost[CHUNKS], gch[CHUNKS];
    float s_pre[CHUNKS][8], s_post[CHUNKS][8], s_gate[CHUNKS][8];
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        at[j] = 8 * (j * THREADS + tid);
        in[j] = at[j] < D;
        wpre[j] = norm_gain(in[j] ? p.w_pre : nullptr, at[j]);
        wpost[j] = norm_gain(in[j] ? p.w_post : nullptr, at[j]);
        gch[j] = norm_gain(in[j] && !p.gate_stride ? p.gate : nullptr, at[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            s_pre[j][e] = s_post[j][e] = s_gate[j][e] = 0.0f;
    }
    for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
        const size_t row = (size_t)t * D;
        u32x4 yw[CHUNKS], gw[CHUNKS], xw[CHUNKS];
        NormRes<F32> rw[CHUNKS], dw[CHUNKS];
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            yw[j] = xw[j] = u32x4{};
            rw[j].zero();
            dw[j].zero();
            gw[j] = gch[j];
            if (in[j]) {
                xw[j] = *(const u32x4 *)(p.dxn + row + at[j]);
                rw[j].load(p.res, row + at[j]);
                if (p.dr)
                    dw[j].load(p.dr, row + at[j]);
                if (p.y)
                    yw[j] = *(const u32x4 *)(p.y + row + at[j]);
                if (p.gate_stride)
                    gw[j] = *(const u32x4 *)(p.gate + row + at[j]);
            }
        }
        // Sums of R^2, a R and Y^2.
        float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float r[8], x[8], w[8], y[8];
            rw[j].get(r);
            norm_unpack(xw[j], x);
            norm_unpack(wpre[j], w);
            norm_unpack(yw[j], y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[0] += r[e] * r[e];
                s[1] += x[e] * w[e] * r[e];
                s[2] += y[e] * y[e];
            }
        }
        norm_block_sum<THREADS>(s, part, turn);
        const float rr = 1.0f / __builtin_sqrtf(s[0] * inv_d + p.eps);
        const float ry = p.post ? 1.0f / __builtin_sqrtf(s[2] * inv_d + p.eps) : 1.0f;
        const float c = s[1] * rr * inv_d; // mean(a xhat)
        // S, all of R's gradient, and the sum of b Y.
        float total[CHUNKS][8], sb[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            float r[8], x[8], w[8], y[8], g[8], wp[8], out[8];
            rw[j].get(r);
            norm_unpack(xw[j], x);
            norm_unpack(wpre[j], w);
            norm_unpack(yw[j], y);
            norm_unpack(gw[j], g);
            norm_unpack(wpost[j], wp);
            dw[j].get(total[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xhat = r[e] * rr;
                total[j][e] += rr * (x[e] * w[e] - xhat * c);
                s_pre[j][e] += x[e] * xhat;
                out[e] = p.res_scale * total[j][e];
                const float yhat = y[e] * ry;
                const float dz = total[j][e] * g[e];
                s_post[j][e] += dz * yhat;
                s_gate[j][e] += total[j][e] * (p.post ? yhat * wp[e] : y[e]);
                sb[0] += dz * wp[e] * y[e];
            }
            if (in[j] && p.dres)
                NormRes<F32>::store(p.dres, row + at[j], out);
            if (in[j] && p.dgate) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    out[e] = total[j][e] * (p.post ? y[e] * ry * wp[e] : y[e]);
                *(u32x4 *)(p.dgate + row + at[j]) = norm_pack(out);
            }
        }
        float cb = 0.0f;
        if (p.post) {
            norm_block_sum<THREADS>(sb, part, turn);
            cb = sb[0] * ry * inv_d; // mean(b yhat)
        }
        if (p.dy) {
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                float y[8], g[8], wp[8], out[8];
                norm_unpack(yw[j], y);
                norm_unpack(gw[j], g);
                norm_unpack(wpost[j], wp);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float dz = total[j][e] * g[e];
                    out[e] = p.post ? ry * (dz * wp[e] - y[e] * ry * cb) : dz;
                }
                if (in[j])
                    *(u32x4 *)(p.dy + row + at[j]) = norm_pack(out);
            }
        }
    }
    if (p.sums) {
        const size_t plane = (size_t)gridDim.x * D;
        float *out = p.partial + (size_t)blockIdx.x * D;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j)
            if (in[j])
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (p.sums >> k & 1) {
                        const float(&v)[8] = k == 0 ? s_pre[j] : k == 1 ? s_post[j] : s_gate[j];
                        f32x4 *o = (f32x4 *)(out + k * plane + at[j]);
                        o[0] = f32x4{v[0], v[1], v[2], v[3]};
                        o[1] = f32x4{v[4], v[5], v[6], v[7]};
                    }
    }
}

// out[k][d] = bf16(sum over the blocks of partial[k][b][d]) for the wanted k
// (blockIdx.y-th of them): 32 columns per block, 8 groups of partial rows, the
// groups' sums in order.
constexpr int kNormColumns = 32, kNormGroups = 8;
__global__ __launch_bounds__(kNormColumns *kNormGroups) void norm_columns_kernel(const float *partial, uint16_t *o0,
                                                                                 uint16_t *o1, uint16_t *o2, int blocks,
                                                                                 int D)
{
    __shared__ float sum[kNormGroups][kNormColumns];
    const int k = blockIdx.y;
    uint16_t *out = k == 0 ? o0 : k == 1 ? o1 : o2;
    if (!out) // the same for the whole block
        return;
    const int col = threadIdx.x % kNormColumns, group = threadIdx.x / kNormColumns;
    const int d = blockIdx.x * kNormColumns + col;
    float s = 0.0f;
    if (d < D)
        for (int b = group; b < blocks; b += kNormGroups)
            s += partial[((size_t)k * blocks + b) * D + d];
    sum[group][col] = s;
    __syncthreads();
    if (group == 0 && d < D) {
#pragma unroll
        for (int g = 1; g < kNormGroups; ++g)
            s += sum[g][col];
        out[d] = __builtin_bit_cast(uint16_t, (__bf16)s);
    }
}

} // namespace gmlp
