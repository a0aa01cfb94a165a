// How much work one launch takes: plain host arithmetic.
//
// A launch holds fewer than 2^32 threads along an axis; with more, the count wraps
// and part of the work is not done (a lookup of 2^24 + 3 rows of 256 threads each
// returned with hardly a row written) or the launch is refused.  Work that may be
// larger is therefore enqueued in parts.
#pragma once

#include <algorithm>
#include <cstdint>

namespace fc {

// A part's threads: enough that its launch costs nothing beside them.
constexpr int64_t LAUNCH_THREADS = (int64_t)1 << 28;

// f(first, count) for consecutive parts of `units` of `threads` threads each.
template <typename F> void by_launches(int64_t units, int64_t threads, F&& f) {
    const int64_t most = std::max<int64_t>(1, LAUNCH_THREADS / threads);
    for (int64_t first = 0; first < units; first += most) f(first, std::min(most, units - first));
}

}  // namespace fc
