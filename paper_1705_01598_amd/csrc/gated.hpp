// The sigmoid of the gated activation.
#pragma once
#include <hip/hip_runtime.h>

namespace tperm {

// The sigmoid of g as p * last, and that of -g.  Below -87 it is no normal number in binary32, though its products with g and with
// larger numbers are, and the hardware's reciprocal, right to 2^-23 like its exp2, gives zero there.
struct Sigmoid {
    float p, last, other;
};
template <typename T> __device__ __forceinline__ Sigmoid sigmoid(float g) {
    constexpr float kHalf = 0x1.715476p-1f, kRest = 0x1.4ae0cp-27f;     // log2(e) / 2 and what that rounds off
    if constexpr (sizeof(T) == 4) {
        // With E = exp(-|g| / 2), r = 1 / (1 + E^2) and for negative g the last E when all else is in a product: no factor
        // leaves the normal numbers before the result does, which is right to 8.25 * 2^-23 whatever g is.
        const float a = __builtin_fminf(__builtin_fabsf(g), 256.0f), x = a * kHalf;       // an infinity would be subtracted from itself
        const float rest = __builtin_fmaf(a, kRest, __builtin_fmaf(a, kHalf, -x)), e0 = __builtin_amdgcn_exp2f(-x), e = __builtin_fmaf(e0, rest * -0.6931472f, e0);
        const float r = __builtin_amdgcn_rcpf(__builtin_fmaf(e, e, 1.0f)), low = g < 0.0f ? e : 1.0f, high = g < 0.0f ? 1.0f : e;
        return {r * low, low, r * high * high};
    } else {
        // The rounding of |g| * log2(e) / 2 adds |g| * 2^-24, and a sigmoid that is no normal number has fewer bits: results of
        // 16 bits show neither.  2^-32 / (2^-32 (1 + exp(-g))) in three operations less; of g and u in 8 bits 91 us
        // against 94 for 32768 rows of 2048 bfloat16 channels.
        const float t = __builtin_amdgcn_exp2f(g * -kHalf), p = __builtin_amdgcn_rcpf(__builtin_fmaf(t * 0x1p-32f, t, 0x1p-32f)) * 0x1p-32f;
        return {p, 1.0f, 1.0f - p};
    }
}

}  // namespace tperm
