// What has to be done once on each device of a process, such as raising a kernel's
// limit of dynamic shared memory: that belongs to the kernel on one device.
#pragma once

#include <atomic>
#include <cstdint>

namespace sn {

class PerDevice {
    std::atomic<uint64_t> done_{0};  // devices 0 to 63; on others it is done at every call

public:
    // `act` on device `dev`, unless it succeeded there before; its status, 0 for success
    // (two threads at once may both do it: what is done here may be done twice)
    template <typename F>
    auto once(int dev, F act) -> decltype(act()) {
        const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t{1} << dev : 0;
        if (done_.load(std::memory_order_acquire) & bit) return {};
        const auto status = act();
        if (!static_cast<int>(status)) done_.fetch_or(bit, std::memory_order_release);
        return status;
    }
};

}  // namespace sn
