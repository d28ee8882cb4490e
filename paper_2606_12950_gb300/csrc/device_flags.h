// device_flags.h -- which devices something has been done on once (not part of
// the ABI).  A kernel's attributes belong to it on one device: a process with
// pools on several sets them on each.
#pragma once

#include <atomic>
#include <cstdint>

namespace kvp {

class DeviceFlags {
public:
    bool has(int device) const { return flag(device) && (bits_.load() & flag(device)) != 0; }
    void set(int device) { bits_.fetch_or(flag(device)); }

private:
    static uint64_t flag(int device) { return device >= 0 && device < 64 ? 1ull << device : 0; }
    std::atomic<uint64_t> bits_{0};
};

}  // namespace kvp
