// Enqueueing a call's kernels, and the check of a device pointer: what every translation unit's entry points use.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <tuple>
#include <utility>

#include "tahq.h"

namespace tahq {

inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// The runtime counts a launch's lanes along a dimension in 32 bits
inline bool launchable(uint64_t workgroups, uint32_t lanes) { return workgroups * lanes < (uint64_t)1 << 32; }

// Kernel launches of one call: each launch returns its own status (the thread's sticky "last error", which may
// belong to the caller's earlier work, is neither read nor cleared), and after a failure nothing more is enqueued.
struct Enqueue {
    hipStream_t stream;
    hipError_t status = hipSuccess;

    template <typename... P, typename... A>
    void operator()(void (*kernel)(P...), dim3 grid, dim3 block, A... args)
    {
        static_assert(sizeof...(P) == sizeof...(A), "one argument per kernel parameter");
        if (status != hipSuccess) return;
        std::tuple<P...> values(static_cast<P>(args)...);
        status = launch(kernel, grid, block, values, std::index_sequence_for<P...>{});
    }
    tahq_status result() const { return status == hipSuccess ? TAHQ_OK : TAHQ_ERR_HIP; }

private:
    template <typename... P, size_t... I>
    hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, std::tuple<P...> &values, std::index_sequence<I...>)
    {
        void *ptrs[] = {static_cast<void *>(&std::get<I>(values))...};
        return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, ptrs, 0, stream);
    }
};

}  // namespace tahq
