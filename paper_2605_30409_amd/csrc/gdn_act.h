// Activations and their slopes, fp32.  With s(z) = 1 / (1 + e^-z), Phi and phi the normal distribution's:
//   silu       z s(z)                 slope s (1 + z (1 - s))
//   gelu       z Phi(z)               slope Phi + z phi
//   gelu_tanh  z s(2k), k = sqrt(2/pi) (z + 0.044715 z^3)
//                                     slope s(2k) + z s(2k) (1 - s(2k)) 2 k'
#pragma once

#include "gdn_device.h"

namespace gdn {

enum Act { kActNone = 0, kActSilu = 1, kActGelu = 2, kActGeluTanh = 3 };

// 1 / (1 + e^-z) by the hardware's reciprocal (within 1 ulp); an e^-z past fp32's range gives 0.
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * erfcf(-0.70710678f * z); }

// 2k = 2 sqrt(2/pi) (z + 0.044715 z^3), and 2k' at a z held where z^2 stays finite (1 - s is 0 from 12 on)
__device__ __forceinline__ float gelu_2k(float z) { return z * (1.5957691f + 0.071354816f * z * z); }
__device__ __forceinline__ float gelu_2k_slope(float z) {
    const float c = fminf(fmaxf(z, -64.f), 64.f);
    return 1.5957691f + 0.21406445f * c * c;
}

__device__ __forceinline__ float act_of(float z, int act) {
    switch (act) {
    case kActSilu: return z * logistic(z);
    case kActGelu: return z * normal_cdf(z);
    case kActGeluTanh: return z * logistic(gelu_2k(z));
    default: return z;
    }
}

// Value and slope at once.
__device__ __forceinline__ void act_and_slope(float z, int act, float &a, float &d) {
    if (act == kActSilu) {
        const float s = logistic(z);
        a = z * s;
        d = s + a * (1.f - s);
    } else if (act == kActGelu) {
        const float s = normal_cdf(z);
        a = z * s;
        d = s + z * (0.39894228f * __expf(-0.5f * z * z));
    } else if (act == kActGeluTanh) {
        const float s = logistic(gelu_2k(z));
        a = z * s;
        d = s + a * (1.f - s) * gelu_2k_slope(z);
    } else {
        a = z;
        d = 1.f;
    }
}

// n values in place; one branch for all of them.
template <int n> __device__ __forceinline__ void act_all(float *z, int act) {
    if (act == kActSilu) {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] = act_of(z[i], kActSilu);
    } else if (act == kActGelu) {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] = act_of(z[i], kActGelu);
    } else if (act == kActGeluTanh) {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] = act_of(z[i], kActGeluTanh);
    }
}

// n slopes in place.
template <int n> __device__ __forceinline__ void slope_all(float *z, int act) {
    float a;
    if (act == kActSilu) {
#pragma unroll
        for (int i = 0; i < n; ++i) act_and_slope(z[i], kActSilu, a, z[i]);
    } else if (act == kActGelu) {
#pragma unroll
        for (int i = 0; i < n; ++i) act_and_slope(z[i], kActGelu, a, z[i]);
    } else if (act == kActGeluTanh) {
#pragma unroll
        for (int i = 0; i < n; ++i) act_and_slope(z[i], kActGeluTanh, a, z[i]);
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] = 1.f;
    }
}

}  // namespace gdn
