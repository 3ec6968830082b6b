// Kernel launches that report their own status.  hipGetLastError() after a launch also returns what any
// earlier call of the thread left there, another library's too, and a handle would be refused for good
// because of it.
#pragma once

#include <hip/hip_runtime.h>

namespace a2t {

template <class T>
struct AsGiven {
    using type = T;
};

template <class... P>
hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t stream, const typename AsGiven<P>::type&... args) {
    void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, at, 0, stream);
    if (e != hipSuccess) (void)hipGetLastError();   // returned here, not left for the thread's next caller
    return e;
}

}  // namespace a2t
