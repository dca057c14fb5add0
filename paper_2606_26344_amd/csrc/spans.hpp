// Checks of which memory the outputs of a call may share.
#pragma once

#include "plan.hpp"

namespace gmlp {
namespace {

struct Extent {
    const void *p;
    size_t bytes;
    const char *name;
    // An output: up to two inputs that it may be (the same memory, element by element).
    const void *same[2] = {nullptr, nullptr};
};

// Every output apart from every input that it may not be, the other outputs and the
// workspace.
inline int check_extents(const Extent *in, int n_in, const Extent *out, int n_out, const void *ws = nullptr,
                         size_t ws_bytes = 0)
{
    for (int i = 0; i < n_out; ++i) {
        const Extent &o = out[i];
        if (!o.p)
            continue;
        for (int j = 0; j < n_in; ++j) {
            const bool same = in[j].p == o.p && in[j].bytes == o.bytes && (o.same[0] == o.p || o.same[1] == o.p);
            if (in[j].p && !same && overlaps(o.p, o.bytes, in[j].p, in[j].bytes))
                return fail(GMLP_ERR_INVALID_ARG, "%s overlaps %s", o.name, in[j].name);
        }
        for (int j = 0; j < i; ++j)
            if (out[j].p && overlaps(o.p, o.bytes, out[j].p, out[j].bytes))
                return fail(GMLP_ERR_INVALID_ARG, "%s overlaps %s", o.name, out[j].name);
        if (ws && overlaps(o.p, o.bytes, ws, ws_bytes))
            return fail(GMLP_ERR_INVALID_ARG, "%s overlaps the workspace", o.name);
    }
    return GMLP_OK;
}

} // namespace
} // namespace gmlp
