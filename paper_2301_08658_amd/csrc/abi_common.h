// Internal: argument checks and launch timing of the C ABI, shared by its
// translation units (defined in abi.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "errors.h"

namespace atp {
namespace abi {

// A row-major device matrix / a device vector argument (as every call checks them).
atp_status check_matrix(const void* p, int64_t rows, int64_t ld, int64_t cols, const char* name);
atp_status check_vector(const void* p, const char* name);
// Runs launch(arg) on s, with timing events around it when profiling is on.
atp_status run_timed(const char* name, double flops, double bytes, hipStream_t s,
                     hipError_t (*launch)(void*), void* arg);
template <class F>
atp_status run_timed(const char* name, double flops, double bytes, hipStream_t s, F&& launch) {
    return run_timed(name, flops, bytes, s,
                     [](void* f) { return (*static_cast<std::remove_reference_t<F>*>(f))(); },
                     &launch);
}

}  // namespace abi
}  // namespace atp
