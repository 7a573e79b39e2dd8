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

// dependent: the kernel may start while the one before it on the stream still runs, and waits for it itself before it touches memory.
template <typename... K, typename... A>
bool launch(void (*kernel)(K...), int64_t blocks, int threads, int shared, bool dependent, cudaStream_t st, const A &...args)
{
    if (blocks < 1 || blocks > 0x7fffffff) return false;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = static_cast<size_t>(shared);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = dependent ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<K>(args)...) == cudaSuccess;
}

inline bool aligned_to(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace softsync
