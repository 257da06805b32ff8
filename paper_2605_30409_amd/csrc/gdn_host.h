// Host-side helpers of the C ABI's implementations: alignment and overlap of arguments, launches.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "gdn.h"

namespace {

bool misaligned(const void *p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

struct Range {
    uintptr_t lo, hi;
    Range(const void *p, size_t bytes) : lo((uintptr_t)p), hi((uintptr_t)p + (p ? bytes : 0)) {}
    bool overlaps(const Range &o) const { return lo < o.hi && o.lo < hi; }
    bool same(const Range &o) const { return lo == o.lo && hi == o.hi; }
};

// Launch one kernel whose only argument is a parameter struct; returns the
// launch's own status (the thread's pending HIP error is neither read nor cleared).
template <class P>
int launch(void (*fn)(P), dim3 grid, dim3 block, size_t lds, hipStream_t s, const P &p) {
    P copy = p;
    void *args[] = {&copy};
    return hipLaunchKernel((const void *)fn, grid, block, args, lds, s) == hipSuccess ? GDN_OK : GDN_ERR_HIP;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace
