// What the kernels over trees have in common.  Included by each .hip file of this folder inside no namespace; nothing here has external linkage.
#pragma once

#include <hip/hip_runtime.h>

#include <initializer_list>

#include "../device_common.h"
#include "tree_plan.h"

namespace {

inline ss_status tree_launched() { return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_DEVICE; }
inline bool off_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline bool bad_workspace(const void* workspace, size_t bytes, size_t need) {
    return !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || bytes < need;
}

// Whether one of the outputs is an input or another output.
inline bool shared(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
    for (const void* const* o = outputs.begin(); o != outputs.end(); ++o) {
        for (const void* i : inputs)
            if (*o && *o == i) return true;
        for (const void* const* p = outputs.begin(); p != o; ++p)
            if (*o && *o == *p) return true;
    }
    return false;
}

}  // namespace
