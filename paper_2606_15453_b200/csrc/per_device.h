// What a call has to find out about a device once: kept per device ordinal, filled by whichever host
// thread comes first.  A reader sees either nothing or the whole value (the flag is written behind the value
// and read ahead of it), a failed fill is tried again by the next call.
#pragma once
#include <atomic>
#include <mutex>

namespace stmoe_host {

constexpr int kMaxDevices = 64;

template <typename T> class PerDevice {
    std::atomic<bool> ready_[kMaxDevices] = {};
    T kept_[kMaxDevices] = {};
    std::mutex fill_;

public:
    // the value of device dev into *out; fill(T &) returns 0 or an error code, which get returns
    template <typename Fill> int get(int dev, T *out, Fill fill)
    {
        if (!ready_[dev].load(std::memory_order_acquire)) {
            std::lock_guard<std::mutex> hold(fill_);
            if (!ready_[dev].load(std::memory_order_relaxed)) {
                T t{};
                if (const int rc = fill(t)) return rc;
                kept_[dev] = t;
                ready_[dev].store(true, std::memory_order_release);
            }
        }
        *out = kept_[dev];
        return 0;
    }
};

}  // namespace stmoe_host
