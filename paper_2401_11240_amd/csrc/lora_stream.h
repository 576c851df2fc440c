// Host side: the device of a launch's stream.
#pragma once
#include <hip/hip_runtime.h>

namespace lora {

// The device a stream belongs to current for the launch.
struct StreamDevice {
    int prev = -1;
    bool ok = false;
    explicit StreamDevice(hipStream_t s) {
        int dev = -1;
        if (hipGetDevice(&prev) != hipSuccess) return;
        if (s) {
            if (hipStreamGetDevice(s, &dev) != hipSuccess) return;
        } else {
            dev = prev;
        }
        ok = dev == prev || hipSetDevice(dev) == hipSuccess;
    }
    ~StreamDevice() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

}  // namespace lora
