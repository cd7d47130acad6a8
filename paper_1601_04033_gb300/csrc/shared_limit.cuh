// A kernel's limit on dynamic shared memory, raised once a device.  Calls on several
// host threads may come first together, so every one asks for the same, the most that
// the kernel can have: no order of theirs leaves the limit below what one was told.
#pragma once

#include <atomic>
#include <cstdint>

namespace fasgd {

struct SharedLimit {
    std::atomic<uint64_t> raised{0};         // by device (one past the 63rd: every time)

    // Before a launch with `need` bytes on `device`, whose kernel can have `most`:
    // raise(bytes) sets the limit; its error (0: none) is returned.
    template <class Raise>
    int ensure(int device, int64_t need, int64_t most, Raise raise) {
        if (need > most) return raise(need);             // refused, as the launch would be
        const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
        if (raised.load(std::memory_order_acquire) & bit) return 0;
        const int error = raise(most);
        if (error == 0) raised.fetch_or(bit, std::memory_order_release);
        return error;
    }
};

}  // namespace fasgd
