// The C ABI of include/gmlp_dropout.h: validation and launches (dropout.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "gmlp_dropout.h"
#include "dropout.hpp"
#include "hip_status.hpp"
#include "spans.hpp"

using namespace gmlp;

namespace {

int check_dropout(int64_t T, int64_t D, double p, const void *position, int flags)
{
    if (T < 0 || D <= 0)
        return fail(GMLP_ERR_INVALID_ARG, "invalid shape T=%lld D=%lld (need T >= 0, D > 0)", (long long)T, (long long)D);
    if (D % 8)
        return fail(GMLP_ERR_UNSUPPORTED, "D=%lld must be a multiple of 8", (long long)D);
    if (D > kMaxDim || T > kMaxTokens || T * D > kMaxElements)
        return fail(GMLP_ERR_UNSUPPORTED, "shape T=%lld D=%lld exceeds the supported range (D <= %lld, T <= %lld, at most "
                    "%lld elements)", (long long)T, (long long)D, (long long)kMaxDim, (long long)kMaxTokens,
                    (long long)kMaxElements);
    if (!(p >= 0.0 && p <= 1.0))
        return fail(GMLP_ERR_INVALID_ARG, "p must be in 0 .. 1");
    if (reinterpret_cast<uintptr_t>(position) % 8)
        return fail(GMLP_ERR_UNSUPPORTED, "position (%p) is not 8-byte aligned", position);
    if (flags & ~GMLP_DROPOUT_FP32)
        return fail(GMLP_ERR_INVALID_ARG, "unknown flags %d", flags);
    return GMLP_OK;
}

DropoutParams dropout_params(const void *x, const void *res, void *out, int64_t T, int64_t D, double p, uint64_t seed,
                             uint64_t offset, const void *position)
{
    DropoutParams d{};
    d.x = x;
    d.res = res;
    d.out = out;
    d.groups = T * D / 8;
    d.offset = offset;
    d.position = static_cast<const uint64_t *>(position);
    d.key0 = (uint32_t)seed;
    d.key1 = (uint32_t)(seed >> 32);
    d.threshold = (uint32_t)std::rint(65536.0 * p);
    d.factor = d.threshold < 65536 ? (float)(65536.0 / (65536 - d.threshold)) : 0.0f;
    return d;
}

template <int IN, int RES, int OUT>
int launch_dropout(const DropoutParams &p, void *stream)
{
    const int64_t blocks = std::min<int64_t>(cdiv(p.groups, kDropoutThreads), 1 << 20);
    hipLaunchKernelGGL((dropout_kernel<IN, RES, OUT>), dim3((unsigned)blocks), dim3(kDropoutThreads), 0,
                       static_cast<hipStream_t>(stream), p);
    const int rc = hip_check(hipGetLastError(), "dropout launch");
    return rc ? rc : ok();
}

} // namespace

extern "C" {

int gmlp_dropout(const void *X, const void *res, void *out, int64_t T, int64_t D, double p, uint64_t seed, uint64_t offset,
                 const void *position, int flags, void *stream)
{
    int rc;
    const bool rows = T > 0, fp32 = flags & GMLP_DROPOUT_FP32;
    if ((rc = check_dropout(T, D, p, position, flags)) || (rc = check_ptr(X, "X", rows)) || (rc = check_ptr(res, "res", rows && fp32)) ||
        (rc = check_ptr(out, "out", rows)))
        return rc;
    if (!rows)
        return ok();
    const size_t e = (size_t)T * D, b = fp32 ? 4 : 2;
    const Extent in[] = {{X, 2 * e, "X"}, {res, b * e, "res"}, {position, 8, "position"}};
    const Extent outs[] = {{out, b * e, "out", {X, res}}};
    if ((rc = check_extents(in, 3, outs, 1)))
        return rc;
    const DropoutParams d = dropout_params(X, res, out, T, D, p, seed, offset, position);
    return !res ? launch_dropout<2, 0, 2>(d, stream) : fp32 ? launch_dropout<2, 4, 4>(d, stream) : launch_dropout<2, 2, 2>(d, stream);
}

int gmlp_dropout_backward(const void *dout, void *dX, int64_t T, int64_t D, double p, uint64_t seed, uint64_t offset,
                          const void *position, int flags, void *stream)
{
    int rc;
    const bool rows = T > 0, fp32 = flags & GMLP_DROPOUT_FP32;
    if ((rc = check_dropout(T, D, p, position, flags)) || (rc = check_ptr(dout, "dout", rows)) || (rc = check_ptr(dX, "dX", rows)))
        return rc;
    if (!rows)
        return ok();
    const size_t e = (size_t)T * D;
    const Extent in[] = {{dout, (fp32 ? 4 : 2) * e, "dout"}, {position, 8, "position"}};
    const Extent outs[] = {{dX, 2 * e, "dX", {dout, nullptr}}};
    if ((rc = check_extents(in, 2, outs, 1)))
        return rc;
    const DropoutParams d = dropout_params(dout, nullptr, dX, T, D, p, seed, offset, position);
    return fp32 ? launch_dropout<4, 0, 2>(d, stream) : launch_dropout<2, 0, 2>(d, stream);
}

} // extern "C"
