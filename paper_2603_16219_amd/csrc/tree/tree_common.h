// What the kernels over trees have in common.  Included by each .hip file of this folder inside no namespace; nothing here has external linkage.
#pragma once

#include <hip/hip_runtime.h>

#include "../device_common.h"
#include "tree_plan.h"

namespace {

inline ss_status tree_launched() { return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_DEVICE; }
inline bool off_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline bool bad_workspace(const void* workspace, size_t bytes, size_t need) {
    return !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || bytes < need;
}

}  // namespace
