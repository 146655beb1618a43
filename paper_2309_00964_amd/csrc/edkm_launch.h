// The size of a launch (host logic without HIP).
#pragma once
#include <cstdint>

namespace edkm {

// Workgroups that one launch of a one-dimensional grid may have: the runtime counts a
// dimension's threads in 32 bits.  A multiple of eight, so that every part of a larger grid
// starts on the first XCD.
inline uint32_t most_groups(uint32_t threads) { return 0xFFFFFFFFu / threads & ~7u; }

// Calls go(first workgroup, workgroups) for the parts of a grid, in order, until one fails.
template <class Status, class Go>
Status in_parts(uint64_t groups, uint32_t threads, Status ok, Go go) {
    const uint64_t most = most_groups(threads);
    for (uint64_t at = 0; at < groups; at += most) {
        const Status s = go((uint32_t)at, (uint32_t)(groups - at < most ? groups - at : most));
        if (s != ok) return s;
    }
    return ok;
}

}  // namespace edkm
