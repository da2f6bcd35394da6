// What every launch on the host side needs (not installed).
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "qesgd_internal.h"

namespace qesgd {

inline int launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QESGD_OK;
    set_last_hip_error((int)e);
    return QESGD_ERR_HIP;
}

// f(the number of dtype as a constant)
template <class F>
void by_type(uint32_t dtype, F&& f) {
    switch (dtype) {
        case QESGD_F32: f(std::integral_constant<uint32_t, QESGD_F32>{}); break;
        case QESGD_BF16: f(std::integral_constant<uint32_t, QESGD_BF16>{}); break;
        default: f(std::integral_constant<uint32_t, QESGD_F16>{}); break;
    }
}

}  // namespace qesgd
