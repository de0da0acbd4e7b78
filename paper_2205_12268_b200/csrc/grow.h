// Limits that only grow (host code, no CUDA: a test compiles it by itself).
#pragma once

#include <atomic>
#include <mutex>

namespace wcc {

// A limit outside that set(n) sets to n, whatever it was, and the largest n that it is known to have been set to.  After raise(want) returns true the
// limit is at least `want` and never falls below it again: check, set and record are one step to other threads.  (Recorded apart, two threads can leave
// the smaller limit set and the larger one recorded.)  Once large enough, a call is one load.
class GrowingLimit {
public:
    template <typename Set>
    bool raise(int want, Set set)
    {
        if (known_.load(std::memory_order_acquire) >= want) return true;
        std::lock_guard<std::mutex> hold(lock_);
        if (known_.load(std::memory_order_relaxed) >= want) return true;
        if (!set(want)) return false;
        known_.store(want, std::memory_order_release);
        return true;
    }

private:
    std::atomic<int> known_{0};
    std::mutex lock_;
};

}  // namespace wcc
