// Argument checks that the entry points of the imputer's operators share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>
#include <vector>

#include "../../include/same.h"
#include "errors.hpp"

namespace same {

constexpr size_t kAlign = 256;  // of workspaces and their parts

inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p) % a == 0; }

struct Extent {
    uintptr_t lo = 0, hi = 0;
};

inline Extent extent(const void *p, int64_t bytes) { return {(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes}; }
inline bool overlap(const Extent &a, const Extent &b) {
    return a.lo < a.hi && b.lo < b.hi && a.lo < b.hi && b.lo < a.hi;
}

// Writable buffers must not overlap each other or what is read.
inline int check_apart(const std::vector<Extent> &writes, const std::vector<Extent> &reads) {
    for (size_t i = 0; i < writes.size(); ++i) {
        for (size_t j = i + 1; j < writes.size(); ++j)
            if (overlap(writes[i], writes[j])) return record_error(SAME_EINVAL, "two outputs overlap");
        for (const Extent &r : reads)
            if (overlap(writes[i], r)) return record_error(SAME_EINVAL, "an output overlaps an input");
    }
    return SAME_OK;
}

inline int check_hip(hipError_t e, const char *what) {
    if (e == hipSuccess) return SAME_OK;
    return record_error(SAME_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace same
