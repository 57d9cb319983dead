// A number that is asked of the driver once for each device and key.  Host code without CUDA.
#pragma once
#include <atomic>

namespace excp {

template <unsigned KEYS, unsigned DEVICES = 64>
class PerDevice {
public:
    // The number of (device, key): what `ask` said when it was asked first.  0 says that the question failed, and is asked again by the next
    // call, as is everything about a device past the last that there is room for.
    template <typename Ask>
    unsigned get(int device, unsigned key, Ask&& ask) {
        if (device < 0 || (unsigned)device >= DEVICES || key >= KEYS) return ask();
        std::atomic<unsigned>& known = known_[device][key];
        unsigned n = known.load(std::memory_order_relaxed);
        if (n == 0 && (n = ask()) != 0) known.store(n, std::memory_order_relaxed);
        return n;
    }

private:
    std::atomic<unsigned> known_[DEVICES][KEYS] = {};
};

}  // namespace excp
