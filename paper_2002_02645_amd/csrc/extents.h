// Which runs of memory a call reads and writes, for the checks of its arguments.  Host code alone.
#pragma once
#include <algorithm>
#include <cstdint>

namespace fz {

struct Extent {
    uintptr_t begin, end;
    bool dst;
};
// whether a dst shares a byte with another extent (sorts them)
inline bool written_twice(Extent *e, int n)
{
    std::sort(e, e + n, [](const Extent &a, const Extent &b) { return a.begin < b.begin; });
    uintptr_t any_end = 0, dst_end = 0;   // how far the extents so far reach
    for (int i = 0; i < n; ++i) {
        if (e[i].begin < (e[i].dst ? any_end : dst_end)) return true;
        any_end = std::max(any_end, e[i].end);
        if (e[i].dst) dst_end = std::max(dst_end, e[i].end);
    }
    return false;
}

}  // namespace fz
