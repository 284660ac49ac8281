// A kernel launch that answers for itself.
#pragma once

#include <tuple>

#include "kernel.hpp"

namespace opevo {

// What <<<>>> leaves to be asked for is the thread's last error, which may be another call's: a failure that some library met and let pass would be reported as this
// launch's.  Arguments are converted to the kernel's own parameters.
template <typename... P, typename... A>
int launch(const char *what, void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t stream, A... args)
{
    std::tuple<P...> values(args...);
    const hipError_t e = std::apply([&](P &...value) {
        void *at[] = {&value...};
        return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, at, 0, stream);
    }, values);
    if (e == hipSuccess) return OPEVO_OK;
    (void)hipGetLastError();            // reported here, and to nobody else
    return hip_fail(e, what);
}

}  // namespace opevo
