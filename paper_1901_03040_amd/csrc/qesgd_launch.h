// What every launch on the host side needs, and the element types in a kernel (not installed).
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

// Element number `at` of type DT becomes v, rounded to it.
template <uint32_t DT>
__device__ __forceinline__ void put(void* c, uint64_t at, float v) {
    if (DT == QESGD_F32) ((float*)c)[at] = v;
    else if (DT == QESGD_F16) ((_Float16*)c)[at] = (_Float16)v;
    else ((__bf16*)c)[at] = (__bf16)v;
}

// f(first, count) for all of `groups` workgroups of `threads`, as many at a time as one launch may number threads for: fewer than 2^32.
template <class F>
int by_launches(uint64_t groups, uint32_t threads, F&& f) {
    const uint64_t most = (1ull << 31) / threads;
    for (uint64_t first = 0; first < groups; first += most) {
        f((uint32_t)first, (uint32_t)(groups - first < most ? groups - first : most));
        if (const int rc = launched(); rc != QESGD_OK) return rc;
    }
    return QESGD_OK;
}

}  // namespace qesgd
