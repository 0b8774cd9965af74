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

// element type of the glue tensors: fp32 for kDtypeF32, bfloat16 for the two bf16 codes
inline int glue_elem_bytes(int dtype)
{
    if (dtype == kDtypeF32) return 4;
    if (dtype == kDtypeBf16 || dtype == kDtypeBf16OutBf16) return 2;
    return 0;
}

}  // namespace convnet

#endif
