// Kernel launches that return their own status.
#pragma once

#include <hip/hip_runtime.h>

namespace micro {

template <class T>
struct Same {
    using type = T;
};

// Launches `kernel`.  (hipGetLastError behind a launch would also return, and
// take away, an error that any earlier call on the thread left.)
template <class... P>
hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t stream, typename Same<P>::type... args) {
    void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, at, 0, stream);
}

}  // namespace micro
