// e^x in fp32 out of the hardware's 2^x.
#pragma once

#include <hip/hip_runtime.h>

namespace darb {

// e^x, off by at most 1.5 units in the last place wherever it is a normal number (3 2^-24 of it: the
// hardware's 2^t by 2 of them, the last step by 1): 2^t with t = x log2 e, where t's rounding and what
// fp32 leaves of log2 e are put right in the result.  Uncorrected, it is off by |x| 2^-24 of itself.
__device__ __forceinline__ float exp_of(float x) {
    constexpr float kLog2E = 0x1.715476p+0f, kLog2ELow = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;
    const float t = x * kLog2E;
    const float e = __builtin_amdgcn_exp2f(t);
    const float r = fmaf(x, kLog2ELow, fmaf(x, kLog2E, -t)) * kLn2;
    return fabsf(t) < 128.0f ? fmaf(e, r, e) : e;           // not where t or e is infinite
}

}  // namespace darb
