// Kernel launches that report their own status.  hipGetLastError() after a launch also returns what any
// earlier call of the thread left there, another library's too, and a handle would be refused for good
// because of it.
#pragma once

#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace a2t {

template <class T>
struct AsGiven {
    using type = T;
};

// Where a launch goes, with the events of a timed one, and its dynamic LDS.
struct LaunchOn {
    hipStream_t stream;
    hipEvent_t start, stop;
    uint32_t lds;
    LaunchOn(hipStream_t stream, hipEvent_t start = nullptr, hipEvent_t stop = nullptr, uint32_t lds = 0)
        : stream(stream), start(start), stop(stop), lds(lds) {}
};

template <class... P>
hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, const LaunchOn& on, const typename AsGiven<P>::type&... args) {
    void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};
    const void* const f = reinterpret_cast<const void*>(kernel);
    const hipError_t e = on.start ? hipExtLaunchKernel(f, grid, block, at, on.lds, on.stream, on.start, on.stop, 0)
                                  : hipLaunchKernel(f, grid, block, at, on.lds, on.stream);
    if (e != hipSuccess) (void)hipGetLastError();   // returned here, not left for the thread's next caller
    return e;
}

}  // namespace a2t
