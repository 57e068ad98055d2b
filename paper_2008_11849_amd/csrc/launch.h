// One kernel of an operator on the caller's stream.  Host code of the .hip files.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

#include "plan.h"

namespace sparsert {

// A launch has under 2^32 threads along x.
inline int check_launch(int64_t workgroups, int threads, std::string &err) {
    if (workgroups * threads < 1ll << 32) return SPARSERT_OK;
    err = "more workgroups than a launch can have";
    return SPARSERT_EUNSUPPORTED;
}

template <typename Args>
int launch_operator(const void *kernel, dim3 grid, int threads, Args &args, void *stream, std::string &err, int lds_bytes = 0) {
    // (104 bytes were measured at 96 bytes' 5.9 us of a call.)
    static_assert(sizeof(Args) <= kArgBytes + 8, "a longer argument block costs the host more per launch");
    void *list[] = {&args};
    const hipError_t e = hipLaunchKernel(kernel, grid, dim3(threads), list, (size_t)lds_bytes, static_cast<hipStream_t>(stream));
    if (e == hipSuccess) return SPARSERT_OK;
    err = std::string("hipLaunchKernel: ") + hipGetErrorString(e);
    return SPARSERT_EHIP;
}

}  // namespace sparsert
