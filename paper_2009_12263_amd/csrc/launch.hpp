// Launches of kernels with arguments of their own.  Whether one failed is what the launch itself says: the runtime's last error may be one that the
// program left behind before the call, and is the program's to read.
#pragma once
#include <hip/hip_runtime.h>

#include <tuple>
#include <utility>

#include "status.hpp"

namespace fg {

template <class... P, class... A>
hipError_t launch_kernel(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t stream, A &&...args) {
    static_assert(sizeof...(P) == sizeof...(A), "one argument for each parameter");
    std::tuple<P...> values(static_cast<P>(std::forward<A>(args))...);
    return std::apply([&](auto &...v) {
        void *at[] = {const_cast<void *>((const void *)&v)...};
        const hipError_t e = hipLaunchKernel((const void *)kernel, grid, block, at, 0, stream);
        if (e != hipSuccess) (void)hipGetLastError();           // (reported by status)
        return e;
    }, values);
}

// The launches of one call on a stream: once one has failed no other is made.
struct Launches {
    hipStream_t stream;
    hipError_t first = hipSuccess;
    explicit Launches(void *s) : stream((hipStream_t)s) {}
    template <class... P, class... A> void operator()(void (*kernel)(P...), dim3 grid, dim3 block, A &&...args) {
        if (first == hipSuccess) first = launch_kernel(kernel, grid, block, stream, std::forward<A>(args)...);
    }
    fg_status status(const char *what) const { return first == hipSuccess ? FG_OK : fail(FG_ERR_LAUNCH, "launch of %s failed: %s", what, hipGetErrorString(first)); }
};

}  // namespace fg
