// What a host thread has done once on a device and need not do again, such as a kernel's shared memory allowance.
#pragma once

#include <atomic>

namespace modse {

// A flag a device; host threads may ask and set at any time.  Devices beyond 63 have none: the question is always answered no.
class DeviceFlags {
public:
    bool has(int device) const { return in(device) && ((bits_.load(std::memory_order_acquire) >> device) & 1ull) != 0; }
    void set(int device)
    {
        if (in(device)) bits_.fetch_or(1ull << device, std::memory_order_release);
    }

private:
    static bool in(int device) { return device >= 0 && device < 64; }
    std::atomic<unsigned long long> bits_{0};
};

}  // namespace modse
