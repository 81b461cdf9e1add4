// exp(x) in fp32 where its argument's size must not cost bits.  __expf rounds x log2(e), and log2(e) itself, before the exponential: |x| 2^-24 and
// |x| 2^-25 of the result.  What these leave out, e = x log2(e) - y, is put back as 2^y (1 + e ln 2), so that the result is within the
// exponential's own unit and a rounding.
#pragma once
#include <hip/hip_runtime.h>

namespace ee {

__device__ __forceinline__ float exp_of(float x) {
    constexpr float LOG2E = 0x1.715476p+0f, LOG2E_LEFT_LN2 = 1.3349759e-8f, LN2 = 0.69314718f;  // log2(e), what it lacks times ln 2, ln 2
    const float y = x * LOG2E, p = __builtin_amdgcn_exp2f(y);
    const float e_ln2 = fmaf(x, LOG2E_LEFT_LN2, fmaf(x, LOG2E, -y) * LN2);
    return fabsf(y) < 128.f ? fmaf(p, e_ln2, p) : p;  // (0 or infinite otherwise, and of a NaN a NaN)
}

}  // namespace ee
