// What the sources of the C ABI share: the error state and the forms of a launch.
#pragma once
#include "../../include/hch.h"

#include <hip/hip_runtime.h>
#include <hip/hip_ext.h>

#include <string>

#include "profile.hpp"

// Every kernel launch of the library: carries the two timing events of the enclosing LaunchTimer,
// if there is one and timing is on; an ordinary launch otherwise.
#define HCH_LAUNCH(kernel, grid, block, lds, stream, ...)                                          \
    do {                                                                                           \
        hipEvent_t ev_a_ = hch::tls_start_event, ev_b_ = hch::tls_stop_event;                      \
        hch::tls_start_event = hch::tls_stop_event = nullptr;                                      \
        if (ev_a_) hipExtLaunchKernelGGL(kernel, grid, block, lds, stream, ev_a_, ev_b_, 0, __VA_ARGS__); \
        else hipLaunchKernelGGL(kernel, grid, block, lds, stream, __VA_ARGS__);                    \
    } while (0)

#define HCH_LAUNCH_CHECK(name)                                                             \
    do {                                                                                   \
        hipError_t e_ = hipGetLastError();                                                 \
        if (e_ != hipSuccess)                                                              \
            return fail(HCH_EHIP, std::string("launch ") + name + ": " + hipGetErrorString(e_)); \
    } while (0)

namespace hch {
inline thread_local std::string tls_error;     // what hch_last_error returns
}

static inline hch_status fail(hch_status st, const std::string &msg)
{
    hch::tls_error = msg;
    return st;
}
