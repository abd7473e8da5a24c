// abi.h -- what every C entry point shares: the status of a failed CUDA call, the launch context of the
// current device, and the checks of pointers, sizes and overlaps.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "internal.h"
#include "resbm.h"

namespace resbm {

// RESBM_ERR_CUDA, with `e` kept for resbm_last_cuda_error() of this host thread
resbm_status cuda_fail(cudaError_t e);
// the current device and its SM count, for work on `stream`
resbm_status make_ctx(void *stream, Ctx *c);

inline resbm_status finish(cudaError_t e) { return e == cudaSuccess ? RESBM_OK : cuda_fail(e); }

inline bool mul_ok(int64_t a, int64_t b) { return a >= 0 && b >= 0 && (a == 0 || b <= INT64_MAX / a); }

// A tensor argument: required non-null when it has elements, aligned to its element size.
inline bool ptr_ok(const void *p, size_t align, bool required)
{
    if (!p) return !required;
    return (reinterpret_cast<uintptr_t>(p) % align) == 0;
}

struct Range {
    uintptr_t lo, hi;
};
inline Range rng(const void *p, int64_t n, size_t es)
{
    uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return Range{a, a + (uintptr_t)n * es};
}
inline bool overlaps(Range a, Range b)
{
    if (!a.lo || !b.lo || a.lo == a.hi || b.lo == b.hi) return false;
    return a.lo < b.hi && b.lo < a.hi;
}
template <size_t N> bool any_overlap(const Range (&outs)[N], const Range *ins, size_t nin)
{
    for (size_t i = 0; i < N; ++i) {
        for (size_t j = 0; j < nin; ++j)
            if (overlaps(outs[i], ins[j])) return true;
        for (size_t j = i + 1; j < N; ++j)
            if (overlaps(outs[i], outs[j])) return true;
    }
    return false;
}

}  // namespace resbm
