// Host-side helpers shared by the entry points of softsync_learn.h.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace softsync {

// Makes `device` current for the duration of a call and restores the caller's choice afterwards.
class DeviceSwitch {
public:
    explicit DeviceSwitch(int device)
    {
        if (device >= 0 && cudaGetDevice(&prev_) == cudaSuccess && prev_ != device)
            switched_ = cudaSetDevice(device) == cudaSuccess;
    }
    ~DeviceSwitch() { if (switched_) cudaSetDevice(prev_); }
    DeviceSwitch(const DeviceSwitch &) = delete;
    DeviceSwitch &operator=(const DeviceSwitch &) = delete;
private:
    int prev_ = -1;
    bool switched_ = false;
};

inline bool aligned_to(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace softsync
