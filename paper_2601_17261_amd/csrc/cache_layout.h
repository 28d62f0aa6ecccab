// How a cache's keys or values lie in memory, and whether the two share any of it: what a call that writes both has to know.  (Host only)
#pragma once
#include <stdint.h>

namespace agzo {

// One of a cache's tensors: its axes of more than one index from the closest on, and what each covers (in values).  extent[0]: a head's values
struct CacheLayout { int64_t stride[3], size[3], extent[4]; int axes; };

enum class CacheFault { none, stride, overlap, large };

// axes: stride and size each.  bad: a stride that is none
inline CacheFault cache_layout(int64_t head_dim, const int64_t (&axes)[3][2], CacheLayout& out, int64_t& bad) {
    out = CacheLayout{};
    out.extent[0] = head_dim;
    for (const auto& x : axes) {
        if (x[1] <= 1) continue;
        bad = x[0];
        if (x[0] % 8 || x[0] < head_dim || x[0] >= (1LL << 40)) return CacheFault::stride;
        int i = out.axes++;
        for (; i > 0 && out.stride[i - 1] > x[0]; --i) { out.stride[i] = out.stride[i - 1]; out.size[i] = out.size[i - 1]; }
        out.stride[i] = x[0];
        out.size[i] = x[1];
    }
    for (int i = 0; i < out.axes; ++i) {
        if (out.stride[i] < out.extent[i]) return CacheFault::overlap;
        const __int128 more = (__int128)(out.size[i] - 1) * out.stride[i] + out.extent[i];
        if (more >= (__int128)1 << 60) return CacheFault::large;
        out.extent[i + 1] = (int64_t)more;
    }
    return CacheFault::none;
}

// Whether two tensors that lie alike share no memory, `between` values from the start of one to the start of the other: apart as a whole, or the blocks of one axis in
// the gaps that the other's leave there, of which the last one's on each axis outside it ends in front of the next block.  (False too where blocks lie in gaps further on)
inline bool layouts_apart(const CacheLayout& k, const CacheLayout& v, int64_t between) {
    if (k.axes != v.axes) return false;
    for (int i = 0; i < k.axes; ++i)
        if (k.stride[i] != v.stride[i] || k.size[i] != v.size[i]) return false;
    if (between >= k.extent[k.axes]) return true;
    for (int i = k.axes - 1; i >= 0 && between + k.extent[i] <= k.stride[i]; --i)
        if (k.extent[i] <= between) return true;
    return false;
}

}  // namespace agzo
