#pragma once
// fxpq_attend.cuh -- what the attention kernels over the paged 8-bit cache share.
//
// Scores and weights.  A query row is held in fp16 with a power of two of its own (its largest value in [2^15, 2^16)),
// codes become fp16 integers exactly, and their products sum in fp32.  With t = log2(e) * scale * (q . key) +
// log2(value scale of the key's block), a key's weight in the value sum is 2^t times its value's integer code, and in
// the normaliser 2^t / (value scale).  So the block's scales cost one fused multiply-add per score, and
// w = 2^(t - m + 7) is rounded to fp16 once.  m follows the running maximum only when t passes m + 8: sums are rescaled a
// few times per row instead of per tile.  w <= 2^15 is within fp16, and rounding to fp16's last step of 2^-24 costs at most
// 2^-31 of the row's largest weight: with w = 2^(t - m) it was 2^-24, and over 2^20 keys what small weights add was lost.  The
// normaliser sums the weights as they are before they are rounded, in fp32.
#include <cfloat>

#include "fxpq_llm.cuh"
#include "fxpq_ptx.cuh"

namespace fxpq {
namespace llm {

constexpr float NO_MAX = -3.0e38f;   // m of a row that has seen no key
constexpr float LAZY = 8.0f;         // t may pass m by this much
constexpr float LIFT = 7.0f, UNLIFT = 0.0078125f;  // weights are 2^LIFT larger than 2^(t - m); the results' division takes it back
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct AttendArgs {
    CUtensorMap tk, tv;  // codes as [n_pages * heads][page][dim] bytes
    Seqs s;
    const float *k_scale, *v_scale;
    const void* q;
    long long q_token, q_head;
    void* out;
    float* lse;
    float* part;  // partial results of units shared by several CTAs
    int n_pages, page, heads, q_heads, group, q_f16, q_vec, causal;
    int share_min, whole;  // see attend_stream_kernel
    int few, few_only;     // sequences of at most `few` rows per key head belong to the stream kernel, where both run
    float scale;
    int* status;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The power of two that brings a row's largest value into [2^15, 2^16) (rows of zeros or not finite: 1): no value of type fp16
// is scaled down, which would cost its last bit.  2^126 is the largest whose inverse is a normal number: below 2^-111 a
// row's largest value comes to lie lower, and at the other end bf16's 2^127 asks for 2^-112.
__device__ __forceinline__ int q_exponent(float amax) {
    const int e = (__float_as_int(amax) >> 23) - 127;
    return amax > 0.0f && amax <= FLT_MAX ? min(126, 15 - e) : 0;
}
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }

__device__ __forceinline__ void put_out(const AttendArgs& A, long long at, float a, float b) {  // two neighbours
    if (A.q_f16)
        *reinterpret_cast<__half2*>(static_cast<__half*>(A.out) + at) = __floats2half2_rn(a, b);
    else
        *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(A.out) + at) = __floats2bfloat162_rn(a, b);
}

// 8 consecutive query values as fp32.
__device__ __forceinline__ void load_q8(const AttendArgs& A, long long at, float (&v)[8]) {
    if (A.q_f16)
        load_f32<8>(static_cast<const __half*>(A.q) + at, A.q_vec, v);
    else
        load_f32<8>(static_cast<const __nv_bfloat16*>(A.q) + at, A.q_vec, v);
}

fxpq_status launch_attend_stream(AttendArgs& A, int dim, int nt, bool whole, cudaStream_t st);
size_t attend_stream_workspace(int dim, int nt);
int stream_nt(long long rows);
long long tile_blocks(int n_tokens, int n_seqs, int group, bool ragged);  // blocks of 256 rows for each key head
fxpq_status launch_attend_tile(AttendArgs& A, int dim, int shares, cudaStream_t st);
size_t attend_tile_workspace(int n_tokens, int q_heads, int dim, int shares);
// The same with the batch's codes expanded to fp16 before, into ws (attend_expand_workspace bytes).
fxpq_status launch_attend_tile_expanded(AttendArgs& A, const int8_t* k, const int8_t* v, int dim, void* ws, int shares, cudaStream_t st);
size_t attend_expand_workspace(int n_seqs, int heads, int dim, long long max_tokens);

}  // namespace llm
}  // namespace fxpq
