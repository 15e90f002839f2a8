// What the entry points of every source file share on the host: argument checks, launches on the caller's stream, and the
// one-shot timing request of resq_time_next_kernel().
#pragma once
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resq.h"

namespace resq {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline int launch_status() { return hipGetLastError() == hipSuccess ? RESQ_OK : RESQ_ERR_HIP; }

// One-shot timing request of resq_time_next_kernel(): the next main kernel this
// thread launches is bracketed by the two events (exact kernel start and end).
inline thread_local hipEvent_t g_time_start = nullptr, g_time_stop = nullptr;

template <typename... KArgs, typename... Args>
inline void launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t lds, hipStream_t st, Args... args) {
    hipEvent_t e0 = g_time_start, e1 = g_time_stop;
    g_time_start = g_time_stop = nullptr;
    hipExtLaunchKernelGGL(kernel, grid, block, lds, st, e0, e1, 0, args...);
}

// a launch counts the threads along an axis in 32 bits
inline bool launch_fits(int64_t blocks, int64_t threads) { return blocks <= 0xFFFFFFFFll / threads; }

// a head's row of the compact K/V cache: d_head and the width r of its 8-bit group
inline bool kv_head_ok(int64_t d_head, int64_t r) {
    return d_head >= 8 && d_head <= 512 && d_head % 8 == 0 && r >= 0 && r <= d_head && r % 8 == 0;
}

}  // namespace resq
