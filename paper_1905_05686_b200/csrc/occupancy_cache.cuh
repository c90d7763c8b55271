// Blocks of a kernel that an SM takes at once, remembered (host code, no CUDA): the driver takes microseconds to answer, and
// calls whose kernels need it take a few themselves.
#pragma once
#include <cstddef>
#include <map>
#include <mutex>
#include <tuple>

namespace lrbi {

class OccupancyCache {
    // Kernels are told apart by their addresses: many have the same type.
    std::map<std::tuple<const void *, int, int, size_t>, int> known_;
    std::mutex mutex_;

public:
    // ask() -> the answer, or 0 where there is none: then 1 is taken, and asked for again the next time.
    template <class Ask>
    int get(const void *kernel, int device, int threads, size_t smem, Ask ask)
    {
        std::lock_guard<std::mutex> lock(mutex_);
        const auto key = std::make_tuple(kernel, device, threads, smem);
        const auto at = known_.find(key);
        if (at != known_.end()) return at->second;
        const int n = ask();
        if (n < 1) return 1;
        try {
            known_.emplace(key, n);
        } catch (...) {      // no room to remember it
        }
        return n;
    }
};

}  // namespace lrbi
