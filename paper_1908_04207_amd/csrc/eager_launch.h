// How every kernel of the library is launched.
#pragma once

#include <hip/hip_runtime.h>

namespace eager {
namespace {

// A kernel with arguments of the types that it declares: what is handed over is an array of addresses, from which
// the runtime copies as many bytes as the kernel takes.  (The runtime's own call: the configuration stack and the
// look at the last error behind a <<<>>> launch are 0.15 of 2.35 us, and a small round is bound by what it costs
// the host.)
template <typename... A>
hipError_t launch(void (*kernel)(A...), dim3 grid, dim3 block, unsigned lds, hipStream_t st, const A &...a)
{
    void *args[] = {const_cast<A *>(&a)...};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, args, lds, st);
    if (e != hipSuccess) (void)hipGetLastError();        // reported here, and nowhere again
    return e;
}

}  // namespace
}  // namespace eager
