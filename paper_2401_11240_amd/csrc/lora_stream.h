// Host side: the device of a launch's stream.
#pragma once
#include <hip/hip_runtime.h>

namespace lora {

// The device a stream belongs to current for the launch.
struct StreamDevice {
    int prev = -1;
    bool ok = false, moved = false;
    explicit StreamDevice(hipStream_t s) {
        int dev = -1;
        if (hipGetDevice(&prev) != hipSuccess) return;
        if (s) {
            if (hipStreamGetDevice(s, &dev) != hipSuccess) return;
        } else {
            dev = prev;
        }
        moved = dev != prev;
        ok = !moved || hipSetDevice(dev) == hipSuccess;
    }
    ~StreamDevice() {
        if (moved) (void)hipSetDevice(prev);
    }
};

}  // namespace lora
