// Launch helpers of the GEMM kernels: their parameters and launches, and the
// counters of a workspace that has not been prepared.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>

#include "gemm_mfma.hpp"
#include "hip_status.hpp"
#include "plan.hpp"

namespace gmlp {
namespace {

inline GemmParams gemm_params(const Step &s, const void *w0, const void *w1, const void *act, void *out, uint8_t *ws,
                       const Layout &l, const Variant &v, const float *rrms, const float *rowdiv)
{
    GemmParams p;
    p.w0 = static_cast<const uint16_t *>(w0);
    p.w1 = static_cast<const uint16_t *>(w1);
    p.act = static_cast<const uint16_t *>(act);
    p.out = static_cast<uint16_t *>(out);
    p.partial = reinterpret_cast<float *>(ws + l.partial_off);
    p.counters = reinterpret_cast<uint32_t *>(ws + l.counters_off);
    p.M = s.M;
    p.N = s.N;
    p.K = s.K;
    p.k_split = s.k_split;
    p.splits = s.splits;
    p.tiles_m = s.tiles_m;
    p.tiles_n = s.tiles_n;
    p.group_m = s.group_m;
    p.tile_base = s.tile_base;
    p.tile_count = s.tile_count;
    p.head_blocks = 0;
    p.activation = v.act;
    p.beta = v.beta;
    p.rrms = rrms;
    p.rowdiv = rowdiv;
    p.out_g = p.out_u = nullptr;
    return p;
}

template <class S, int EPI, bool SPLIT, bool STREAM_W = false>
int launch_gemm(const Step &s, const void *w0, const void *w1, const void *act, void *out,
                uint8_t *ws, const Layout &l, const Variant &v, const float *rrms, const float *rowdiv,
                hipStream_t stream, int head_blocks = 0)
{
    GemmParams p = gemm_params(s, w0, w1, act, out, ws, l, v, rrms, rowdiv);
    if (head_blocks && (!SPLIT || head_blocks % 8 != 0))
        return fail(GMLP_ERR_INVALID_ARG, "internal: %d whole-tile head blocks", head_blocks);
    p.head_blocks = head_blocks;
    if (!SPLIT && s.splits != 1)
        return fail(GMLP_ERR_INVALID_ARG, "internal: split-K plan for a kernel without split-K");
    if (s.partial_bytes > (size_t)kNumRecords)
        return fail(GMLP_ERR_UNSUPPORTED, "split-K partial sums of %zu bytes exceed the 2 GiB buffer range",
                    s.partial_bytes);
    hipLaunchKernelGGL((gemm_mfma_kernel<S, EPI, SPLIT, STREAM_W>), dim3(head_blocks + s.blocks), dim3(S::NTHREADS), 0,
                       stream, p);
    return hip_check(hipGetLastError(), "MFMA GEMM launch");
}

// Zero n 32-bit words.  A kernel rather than a memset, so that a captured
// call holds kernels only.
__global__ void zero_words_kernel(uint32_t *p, uint32_t n)
{
    for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x)
        p[i] = 0u;
}

inline int clear_words(uint32_t *p, int words, hipStream_t st)
{
    if (words <= 0)
        return GMLP_OK;
    hipLaunchKernelGGL(zero_words_kernel, dim3((unsigned)std::min(64, (words + 255) / 256)), dim3(256), 0, st, p,
                       (uint32_t)words);
    return hip_check(hipGetLastError(), "counter clear launch");
}

// A call on a workspace that was not initialised (GMLP_FRESH_WORKSPACE)
// clears the arrival counters its steps use, if any: at most 64 KB of the
// 128 KB counter block, which the kernels of these paths touch nothing else
// of, and no launch at all where no step splits K.
inline int clear_counters(bool fresh, int words, uint8_t *ws, const Layout &l, hipStream_t st)
{
    return fresh ? clear_words(reinterpret_cast<uint32_t *>(ws + l.counters_off), words, st) : GMLP_OK;
}

// Takes GMLP_FRESH_WORKSPACE out of `path`.  The fused paths' ready words
// and give-up count need a prepared workspace, so with them the flag stays in
// and the path is refused as unknown.
constexpr int kFreshAuto = GMLP_PATH_AUTO | GMLP_FRESH_WORKSPACE;
inline bool take_fresh(int *path)
{
    const int base = *path & ~GMLP_FRESH_WORKSPACE;
    if (base == *path || (base != GMLP_PATH_AUTO && base != GMLP_PATH_GEMV && base != GMLP_PATH_MFMA))
        return false;
    *path = base;
    return true;
}

} // namespace
} // namespace gmlp
