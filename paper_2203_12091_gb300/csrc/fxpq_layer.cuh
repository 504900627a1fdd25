#pragma once
// fxpq_layer.cuh -- activations of the 8-bit layers, their derivatives, and the form in which sums are kept for a gradient.
#include "fxpq_llm.cuh"

namespace fxpq {
namespace llm {

// The larger of z and low; NaN stays NaN (fmaxf drops it).
__device__ __forceinline__ float cut(float z, float low) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(z), "f"(low));
    return y;
}
// z between -limit and limit; NaN stays NaN.
__device__ __forceinline__ float within(float z, float limit) {
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(cut(z, -limit)), "f"(limit));
    return y;
}
inline bool act_ok(int a) { return a >= FXPQ_ACT_NONE && a <= FXPQ_ACT_GELU_TANH; }

// 1 / (1 + e^-z).  (__expf and __fdividef: 2^-21 of the result where it is 2^-8 or more; past e^88 the quotient is 0.)
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
constexpr float GELU_A = 1.5957691216057308f, GELU_B = 0.044715f;  // 2 sqrt(2 / pi)
// The normal distribution's tail Phi(-a) = e^(-a^2 / 2) t P(t), a >= 0, t = 1 / (1 + 0.45 a / sqrt 2): P a polynomial of degree 9 fitted to
// e^(x^2) erfc(x) / (2 t) at x = a / sqrt 2 by weighted least squares, to 7e-8 of itself for a up to 40; with fp32 steps 4e-7.  (erfcf took four times as
// long: 2000 x 4096 of 2048 with GELU 75 us, without 44.)  e: the exponential.
__device__ __forceinline__ float normal_tail(float a, float& e) {
    const float t = __fdividef(1.0f, fmaf(0.31819805f, a, 1.0f));
    float p = -2.069910988e-02f;
    p = fmaf(p, t, 9.535939991e-02f);
    p = fmaf(p, t, -1.503192931e-01f);
    p = fmaf(p, t, 7.122809440e-02f);
    p = fmaf(p, t, -1.119495742e-02f);
    p = fmaf(p, t, 5.998074636e-02f);
    p = fmaf(p, t, 8.762495220e-02f);
    p = fmaf(p, t, 1.141359434e-01f);
    p = fmaf(p, t, 1.269415766e-01f);
    p = fmaf(p, t, 1.269426644e-01f);
    e = __expf(-0.5f * a * a);
    return p * t * e;
}
__device__ __forceinline__ float gelu(float z) {
    float e;
    const float q = normal_tail(fabsf(z), e);
    return cut(z, -40.0f) * (z > 0.0f ? 1.0f - q : q);  // (far below, a tail of 0 meets no inf)
}
__device__ __forceinline__ float activate(float z, int act) {
    switch (act) {
        case FXPQ_ACT_RELU: return cut(z, 0.0f);
        case FXPQ_ACT_SILU: return z * sigmoid(z);
        case FXPQ_ACT_GELU: return gelu(z);
        case FXPQ_ACT_GELU_TANH: return z * sigmoid(GELU_A * z * fmaf(GELU_B, z * z, 1.0f));
        default: return z;
    }
}
// act(z) and its derivative.  Where the derivative has reached its limits z is cut off, so that no inf meets a zero; both are NaN where z is.
__device__ __forceinline__ float activate_slope(float z, int act, float& slope) {
    switch (act) {
        case FXPQ_ACT_RELU: slope = z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z; return cut(z, 0.0f);
        case FXPQ_ACT_SILU: {
            const float c = within(z, 100.0f), s = sigmoid(c);
            slope = s * fmaf(c, 1.0f - s, 1.0f);
            return z * s;
        }
        case FXPQ_ACT_GELU: {
            const float c = within(z, 40.0f);
            float e;
            const float q = normal_tail(fabsf(c), e), p = z > 0.0f ? 1.0f - q : q;
            slope = fmaf(c * 0.3989422804014327f, e, p);
            return cut(z, -40.0f) * p;
        }
        case FXPQ_ACT_GELU_TANH: {
            const float c = within(z, 30.0f), p = sigmoid(GELU_A * c * fmaf(GELU_B, c * c, 1.0f));
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

// Elements between rows of kept sums: whole 16 bytes.
__host__ __device__ inline long long pre_pitch(int32_t N) { return ((long long)N + 7) / 8 * 8; }

// The rows of a gradient, dz * sw, in two parts M rows apart (fxpq_layer_grad.cu).  PART: what the first part counts in.
constexpr float PART = 4096.0f;
struct GradRows {
    const void* dy;
    long long dy_stride;
    const void* pre;
    const float *sx, *sw, *bias;
    float pre_unit;
    int pre_f32, act, N, early;
    int vec;  // dy, kept sums, scales, biases in aligned accesses (bits 1, 2, 4, 8)
    __half* rows;
    long long pitch, M;
    float* scale;
    int* status;
};
fxpq_status grad_rows(const GradRows& rows, int y_type, int gated, cudaStream_t st);

}  // namespace llm
}  // namespace fxpq
