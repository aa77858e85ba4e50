// host.hpp — what the host units of the C ABI (api.cpp, forward.cpp) share:
// the thread's last error message and the guards of the C entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdio>
#include <exception>
#include <new>
#include <stdexcept>

#include "../../include/mezo.h"

namespace mezo {

// The last failure's message on this thread (a fixed buffer: reporting an
// error allocates nothing).
inline thread_local char t_last_error[256];

inline void set_error(const char* what, const char* detail = nullptr)
{
    std::snprintf(t_last_error, sizeof(t_last_error), detail ? "%s: %s" : "%s", what, detail);
}

inline int hip_fail(hipError_t e, const char* where)
{
    set_error(where, hipGetErrorString(e));
    return MEZO_EHIP;
}

// Runs the body of a C entry point: no C++ exception crosses the C ABI. The
// only ones the bodies can raise are host allocation failures (record lists,
// tables) and, in principle, a failing mutex.
template <class F>
int guarded(const char* what, F&& body) noexcept
{
    try {
        return body();
    } catch (const std::bad_alloc&) {
        set_error(what, "host allocation failed");
    } catch (const std::length_error&) {
        set_error(what, "host allocation failed");
    } catch (const std::exception& e) {
        set_error(what, e.what());
        return MEZO_EINVAL;
    } catch (...) {
        set_error(what, "unexpected exception");
        return MEZO_EINVAL;
    }
    return MEZO_ENOMEM;
}

#define MEZO_HIP(call)                                  \
    do {                                                \
        hipError_t err_ = (call);                       \
        if (err_ != hipSuccess) return mezo::hip_fail(err_, #call); \
    } while (0)

}  // namespace mezo
