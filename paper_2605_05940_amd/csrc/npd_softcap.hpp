// The soft cap of a head's logits.
#pragma once
#include "npd_device.hpp"

namespace npd {

// cap tanh(x / cap).  With w = 2 log2(e) x / cap: tanh = 1 - 2 / (1 + 2^w), whose rounding errors are absolute (2^-22), from |w| = 1 (tanh
// .33) on; below w P(w^2), P fitted there to 3.3e-8 relative.  Either is within 2^-20 of itself, so that a logit's accuracy does not
// depend on the cap: the first form alone is off by cap 2^-22, 0.09 at a cap of 1e6.  Measured (MI355X): the forward kernel of 6,554 x
// 262,144 x 1,152 4.72 ms with the first form alone, 5.04 with both; one of the two by a branch where all values of a wave allow it is 0.1 ms
// faster there and 5 % slower in small calls (333 x 50,003 x 1,000 logits 88.3 and 92.2 us).
struct SoftCap {
  float cap, k2;
  __device__ __forceinline__ explicit SoftCap(float c) : cap(c), k2(2.0f * kLog2e / c) {}
  __device__ __forceinline__ float tanh_of(float x) const {
    const float w = x * k2, t = w * w;
    const float far = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + exp2_fast(w));
    float p = __builtin_fmaf(t, -0x1.ed6cb4p-16f, 0x1.5c8edcp-11f);
    p = __builtin_fmaf(t, p, -0x1.c6ad7cp-7f);
    p = __builtin_fmaf(t, p, 0x1.62e43p-2f);
    return __builtin_fabsf(w) < 1.0f ? w * p : far;
  }
};

}  // namespace npd
