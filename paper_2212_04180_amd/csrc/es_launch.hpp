// es_launch.hpp -- a kernel's launch with its own status.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

namespace esmi {

// hipGetLastError after a launch also gives what an earlier call of the program's
// has left, and the operators would report work as failed that is under way.
template <typename... P>
hipError_t launch(void (*kernel)(P...), unsigned grid, unsigned threads, size_t lds, hipStream_t s, std::common_type_t<P>... args)
{
    void* p[] = {static_cast<void*>(&args)...};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(grid), dim3(threads), p, lds, s);
    if (e != hipSuccess) (void)hipGetLastError();  // reported by this call, not by the next one too
    return e;
}

}  // namespace esmi
