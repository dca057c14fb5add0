// HIP errors as status codes of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include "plan.hpp"

namespace gmlp {
namespace {

inline int hip_check(hipError_t e, const char *what)
{
    if (e != hipSuccess)
        return fail(GMLP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return GMLP_OK;
}

} // namespace
} // namespace gmlp
