// What the host sides share: HIP errors, launches and their timing (defined in iwp_api.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/iwp.h"

#pragma GCC visibility push(hidden)
namespace iwp {

int hip_fail(hipError_t e, const char* what);        // keeps the text for iwp_last_hip_error(); IWP_EHIP

struct TimedLaunch {       // records an event pair around the launch made while it is alive, if its kernel is being timed
    hipStream_t s;
    int slot = -1;
    TimedLaunch(const char* kernel, hipStream_t stream);
    ~TimedLaunch();
};

}  // namespace iwp
#pragma GCC visibility pop

#define IWP_HIP(call)                                         \
    do {                                                      \
        hipError_t e_ = (call);                               \
        if (e_ != hipSuccess) return hip_fail(e_, #call);     \
    } while (0)

// Launch `kernel<<<grid, BLOCK, lds, s>>>(args...)`, timed if asked for, and turn a
// launch failure into IWP_EHIP.  lds: bytes of LDS that no one uses, see few_at_a_time().
#define IWP_LAUNCH(name, kernel, grid, s, ...) IWP_LAUNCH_AS(name, kernel, grid, BLOCK, 0u, s, __VA_ARGS__)
#define IWP_LAUNCH_BLOCK(name, kernel, grid, block, s, ...) IWP_LAUNCH_AS(name, kernel, grid, block, 0u, s, __VA_ARGS__)
#define IWP_LAUNCH_FEW(name, kernel, grid, lds, s, ...) IWP_LAUNCH_AS(name, kernel, grid, BLOCK, lds, s, __VA_ARGS__)
#define IWP_LAUNCH_AS(name, kernel, grid, block, lds, s, ...)         \
    do {                                                              \
        {                                                             \
            TimedLaunch tl_(name, s);                                 \
            kernel<<<(grid), (block), (lds), (s)>>>(__VA_ARGS__);     \
        }                                                             \
        hipError_t e_ = hipGetLastError();                            \
        if (e_ != hipSuccess) return hip_fail(e_, name);              \
    } while (0)
