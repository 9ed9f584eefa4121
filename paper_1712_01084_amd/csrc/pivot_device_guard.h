// The device that a call works on, for as long as the guard lives.
#pragma once

#include <hip/hip_runtime.h>

namespace pivot {

struct DeviceGuard {
    int prev = -1;
    bool ok = true, changed = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) { (void)hipGetLastError(); ok = false; return; }
        if (prev == dev) return;
        if (hipSetDevice(dev) == hipSuccess) changed = true;
        else { (void)hipGetLastError(); ok = false; }
    }
    ~DeviceGuard() { if (changed) (void)hipSetDevice(prev); }
    DeviceGuard(const DeviceGuard&) = delete;
    DeviceGuard& operator=(const DeviceGuard&) = delete;
};

}  // namespace pivot
