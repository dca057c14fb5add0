// Dropout with a mask from a counter-based generator, for gfx950.
//
// Element i of a tensor is kept where 16 bits of Philox4x32-10 of the counter i / 8 are
// at least a threshold (include/gmlp_dropout.h), so forward and backward pass are one
// elementwise pass that makes the mask on the way; nothing but the tensors is read or
// written.
//
// A thread takes the eight elements of one counter, 16 bytes of bf16, so that a call of
// the generator serves them all.  Ten rounds of two 32 x 32 -> 64-bit products (quarter
// rate) and eight other instructions are about 600 cycles of a wave's 512 elements; with
// 32 bits for each element they would be twice that and bound the pass instead of the
// memory.  Measured: 4096 x 4096 into an fp32 residual stream 31.8 us, 5.3 TB/s (a copy
// on that board 5.1); past the L2 the stores are slower (32.0 against 28.6 us on inputs in
// the last-level cache).
#pragma once

#include <type_traits>

#include "common.hpp"

namespace gmlp {

struct DropoutParams {
    const void *x, *res;
    void *out;
    int64_t groups; // of eight elements
    uint64_t offset;
    const uint64_t *position; // nullptr: 0
    uint32_t key0, key1;
    uint32_t threshold; // 0 .. 65536
    float factor;
};

constexpr int kDropoutThreads = 256;

// Philox4x32-10 of the counter (c, 0).
__device__ __forceinline__ u32x4 philox(uint64_t c, uint32_t k0, uint32_t k1)
{
    u32x4 x{(uint32_t)c, (uint32_t)(c >> 32), 0u, 0u};
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)x[0] * 0xD2511F53u, b = (uint64_t)x[2] * 0xCD9E8D57u;
        x = u32x4{(uint32_t)(b >> 32) ^ x[1] ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ x[3] ^ k1, (uint32_t)a};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return x;
}

// Eight neighbouring elements: 16 bytes of bf16, or 32 of fp32.
template <int BYTES>
struct Eight {
    u32x4 v[BYTES / 2];
    __device__ __forceinline__ void load(const void *p, int64_t group)
    {
#pragma unroll
        for (int i = 0; i < BYTES / 2; ++i)
            v[i] = static_cast<const u32x4 *>(p)[group * (BYTES / 2) + i];
    }
    __device__ __forceinline__ void store(void *p, int64_t group) const
    {
#pragma unroll
        for (int i = 0; i < BYTES / 2; ++i)
            static_cast<u32x4 *>(p)[group * (BYTES / 2) + i] = v[i];
    }
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (BYTES == 2)
            return e % 2 ? bf16_hi(v[0][e / 2]) : bf16_lo(v[0][e / 2]);
        else
            return __builtin_bit_cast(float, (uint32_t)v[e / 4][e % 4]);
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        if constexpr (BYTES == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[0][i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e / 4][e % 4] = __builtin_bit_cast(uint32_t, x[e]);
        }
    }
};

// IN, RES, OUT: bytes of an element (RES 0: no residual).
template <int IN, int RES, int OUT>
__global__ __launch_bounds__(kDropoutThreads) void dropout_kernel(DropoutParams p)
{
    const uint64_t start = p.offset + (p.position ? *p.position : 0);
    for (int64_t g = (int64_t)blockIdx.x * kDropoutThreads + threadIdx.x; g < p.groups;
         g += (int64_t)gridDim.x * kDropoutThreads) {
        Eight<IN> x;
        Eight<RES ? RES : 2> res;
        x.load(p.x, g);
        if constexpr (RES != 0)
            res.load(p.res, g);
        const u32x4 w = philox(start + (uint64_t)g, p.key0, p.key1);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t bits = e % 2 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu;
            y[e] = bits >= p.threshold ? x.get(e) * p.factor : 0.0f;
            if constexpr (RES != 0)
                y[e] += res.get(e);
        }
        Eight<OUT> out;
        out.set(y);
        out.store(p.out, g);
    }
}

} // namespace gmlp
