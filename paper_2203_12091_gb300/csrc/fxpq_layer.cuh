#pragma once
// fxpq_layer.cuh -- activations of the 8-bit layers, their derivatives, and the form in which sums are kept for a gradient.
#include "fxpq_llm.cuh"

namespace fxpq {
namespace llm {

inline bool act_ok(int a) { return a >= FXPQ_ACT_NONE && a <= FXPQ_ACT_GELU_TANH; }

// 1 / (1 + e^-z).  (__expf and __fdividef: 2^-21 of the result where it is 2^-8 or more; past e^88 the quotient is 0.)
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
constexpr float GELU_A = 1.5957691216057308f, GELU_B = 0.044715f;  // 2 sqrt(2 / pi)
__device__ __forceinline__ float activate(float z, int act) {
    switch (act) {
        case FXPQ_ACT_RELU: return fmaxf(z, 0.0f);
        case FXPQ_ACT_SILU: return z * sigmoid(z);
        case FXPQ_ACT_GELU: return 0.5f * z * erfcf(-0.70710678118654752f * z);
        case FXPQ_ACT_GELU_TANH: return z * sigmoid(GELU_A * z * fmaf(GELU_B, z * z, 1.0f));
        default: return z;
    }
}
// act(z) and its derivative.  Where the derivative has reached its limits z is cut off, so that no inf meets a zero.
__device__ __forceinline__ float activate_slope(float z, int act, float& slope) {
    switch (act) {
        case FXPQ_ACT_RELU: slope = z > 0.0f ? 1.0f : 0.0f; return fmaxf(z, 0.0f);
        case FXPQ_ACT_SILU: {
            const float c = fminf(fmaxf(z, -100.0f), 100.0f), s = sigmoid(c);
            slope = s * fmaf(c, 1.0f - s, 1.0f);
            return z * s;
        }
        case FXPQ_ACT_GELU: {
            const float p = 0.5f * erfcf(-0.70710678118654752f * z), c = fminf(fmaxf(z, -20.0f), 20.0f);
            slope = fmaf(c * 0.3989422804014327f, __expf(-0.5f * c * c), p);
            return z * p;
        }
        case FXPQ_ACT_GELU_TANH: {
            const float c = fminf(fmaxf(z, -30.0f), 30.0f), p = sigmoid(GELU_A * c * fmaf(GELU_B, c * c, 1.0f));
            slope = p * fmaf(c * (1.0f - p), GELU_A * fmaf(3.0f * GELU_B, c * c, 1.0f), 1.0f);
            return z * p;
        }
        default: slope = 1.0f; return z;
    }
}

// Sums kept for a gradient in fp16 are times 2^-p: the largest, K * 127 * 128, fits, and an odd sum keeps 11 bits up to K = 2^16.
inline int sum_shift(int32_t K) {
    int p = 0;
    while (p < 40 && (double)K * (127.0 * 128.0) > 65504.0 * (double)(1LL << p)) ++p;
    return p;
}

}  // namespace llm
}  // namespace fxpq
