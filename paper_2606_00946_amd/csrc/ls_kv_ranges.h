// Where the arrays of a call's caches lie.  Host code, no HIP.
#pragma once

#include <algorithm>
#include <cstdint>

namespace ls {

// Bytes [lo, hi) of memory.
struct KvRange {
    uint64_t lo, hi;
};
inline KvRange kv_range(const void* p, int64_t bytes) { return {(uint64_t)(uintptr_t)p, (uint64_t)(uintptr_t)p + (uint64_t)bytes}; }

// Whether two of n ranges have a byte in common; sorts them.
inline bool kv_ranges_meet(KvRange* r, int64_t n) {
    std::sort(r, r + n, [](const KvRange& a, const KvRange& b) { return a.lo < b.lo; });
    for (int64_t i = 1; i < n; ++i)
        if (r[i].lo < r[i - 1].hi) return true;
    return false;
}

}  // namespace ls
