// What the host code of the library's translation units shares: the text of the last HIP error of a thread, and the
// checks around a launch.
#ifndef CONVNET_HOST_STATUS_H
#define CONVNET_HOST_STATUS_H

#include <hip/hip_runtime.h>

#include <stdint.h>
#include <stdio.h>

#include "plan.h"

namespace convnet {

inline thread_local char g_hip_error[256] = "";

inline int hip_fail(hipError_t e)
{
    snprintf(g_hip_error, sizeof(g_hip_error), "%s", hipGetErrorString(e));
    return kErrHip;
}

inline int check_launch()
{
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? kStatusOk : hip_fail(e);
}

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace convnet

#endif
