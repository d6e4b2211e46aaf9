// Shared by the files of the C ABI (api.hip defines it): error slot, launch profiling, argument checks.
#pragma once
#include "../../include/quartet.h"

#include <hip/hip_runtime.h>

namespace quartet {

// keeps the code for quartet_last_hip_error (per thread); QUARTET_EHIP
int hip_fail(hipError_t e);

// one launch (or the launches of one call) in quartet_profile_read's record, if that is on
struct ProfileScope {
    int slot = -1;
    hipStream_t st;
    ProfileScope(int kind, hipStream_t s);
    ~ProfileScope();
    ProfileScope(const ProfileScope&) = delete;
    ProfileScope& operator=(const ProfileScope&) = delete;
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_gemm_args(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales, int64_t m, int64_t n,
                    int64_t k, const void* d, int d_dtype, int64_t ldd);

}  // namespace quartet
