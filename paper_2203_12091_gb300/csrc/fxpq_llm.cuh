#pragma once
// fxpq_llm.cuh -- helpers shared by the 8-bit language-model kernels: element types, batches of sequences.
#include <cuda_bf16.h>

#include "fxpq_common.cuh"

namespace fxpq {
int num_sms();  // of the current device (fxpq_conv_tc.cu)

namespace llm {

inline bool ftype_ok(int t) { return t == FXPQ_FT_F32 || t == FXPQ_FT_F16 || t == FXPQ_FT_BF16; }
inline int ftype_bytes(int t) { return t == FXPQ_FT_F32 ? 4 : 2; }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// N consecutive elements as fp32; vec: the address is aligned to their size (at most 16 bytes per access).
template <int N, typename T>
__device__ __forceinline__ void load_f32(const T* __restrict__ p, bool vec, float (&v)[N]) {
    constexpr int B = N * (int)sizeof(T), A = B < 16 ? B : 16, E = A / (int)sizeof(T);
    if (vec) {
#pragma unroll
        for (int i = 0; i < N; i += E) {
            alignas(16) T t[E];
            if constexpr (A == 16)
                *reinterpret_cast<uint4*>(t) = *reinterpret_cast<const uint4*>(p + i);
            else
                *reinterpret_cast<uint2*>(t) = *reinterpret_cast<const uint2*>(p + i);
#pragma unroll
            for (int j = 0; j < E; ++j) v[i + j] = to_f32(t[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = to_f32(p[i]);
    }
}
template <int N, typename T>
__device__ __forceinline__ void store_f32(T* p, const float (&v)[N]) {  // aligned as above
    constexpr int B = N * (int)sizeof(T), A = B < 16 ? B : 16, E = A / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < N; i += E) {
        alignas(16) T t[E];
#pragma unroll
        for (int j = 0; j < E; ++j) t[j] = from_f32<T>(v[i + j]);
        if constexpr (A == 16)
            *reinterpret_cast<uint4*>(p + i) = *reinterpret_cast<const uint4*>(t);
        else
            *reinterpret_cast<uint2*>(p + i) = *reinterpret_cast<const uint2*>(t);
    }
}

__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
// Two codes (bytes 0, 1 or 2, 3 of x, sign bits flipped) as fp16: 0x6400 + u is 1024 + u, minus 1152.
__device__ __forceinline__ uint32_t code_pair(uint32_t x, uint32_t sel) {
    const uint32_t w = __byte_perm(x, 0x64646464u, sel);
    return h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&w), __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480))));
}
constexpr uint32_t LOW_PAIR = 0x4140, HIGH_PAIR = 0x4342;

// Four codes in a word, first one in the low byte.
__device__ __forceinline__ uint32_t pack_i8(int a, int b, int c, int d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// What the kernels see of a batch (fxpq_kv_batch).
struct Seqs {
    const int* pages;
    const int* lens;
    const int* starts;  // null: `each` new tokens per sequence
    long long pages_stride;
    int n_seqs, max_pages, n_tokens, each;
};
inline Seqs make_seqs(const fxpq_kv_batch& b) {
    return {b.d_pages, b.d_lens, b.d_starts, (long long)b.pages_stride, b.n_seqs, b.max_pages, b.n_tokens,
            b.d_starts || b.n_seqs == 0 ? 0 : b.n_tokens / b.n_seqs};
}
// Sequence b's new tokens are rows first .. first + count - 1 (kept within the list whatever d_starts holds).
__device__ __forceinline__ void new_rows(const Seqs& s, int b, int& first, int& count) {
    if (s.starts) {
        const int a = max(__ldg(s.starts + b), 0), e = min(__ldg(s.starts + b + 1), s.n_tokens);
        first = a;
        count = max(e - a, 0);
    } else {
        first = b * s.each;
        count = s.each;
    }
}

// Work units of ragged sequences without a scan.  Sequence b with n_b new tokens needs at most
// floor(mul n_b / unit) + pad units of `unit` rows (mul rows a token); the units from
// base(b) = floor(mul starts[b] / unit) + pad b on are its own, for floor(x + y) >= floor(x) + floor(y).  The grid
// covers base(n_seqs) units, of which those past a sequence's last have nothing to do.
__host__ __device__ __forceinline__ long long unit_base(long long start, int b, int mul, int unit, int pad) {
    return start * mul / unit + (long long)pad * b;
}
// The sequence of unit x, for a whole warp: a search in which the lanes probe 32 places at once.
__device__ __forceinline__ int find_seq(const Seqs& s, long long x, int mul, int unit, int pad) {
    int lo = 0, hi = s.n_seqs;
    const int lane = threadIdx.x & 31;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, i = lo + lane * step;
        const bool in = i < hi && unit_base(max(__ldg(s.starts + i), 0), i, mul, unit, pad) <= x;
        const int c = __popc(__ballot_sync(0xffffffffu, in));
        lo += (c > 0 ? c - 1 : 0) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// What codes of a row x under a norm need to know, f = x * weight: the largest |f| and |x|, the sum of x^2.  Where x or f is not finite
// f counts as 0 (x only if it is not finite itself).
struct RowStats {
    float top = 0.0f, far = 0.0f, sum = 0.0f;
    bool bad = false;
    static __device__ __forceinline__ float value(float x, float w) {
        const float f = __fmul_rn(x, w);
        return fabsf(f) <= 3.402823466e38f && fabsf(x) <= 3.402823466e38f ? f : 0.0f;
    }
    __device__ __forceinline__ void see(float x, float w, float per_unit) {
        const float f = __fmul_rn(x, w);
        const bool x_fine = fabsf(x) <= 3.402823466e38f, fine = x_fine && fabsf(f) <= 3.402823466e38f;
        bad |= !fine;
        top = fmaxf(top, fine ? fabsf(f) : 0.0f);
        if (!x_fine) x = 0.0f;
        far = fmaxf(far, fabsf(x));
        x *= per_unit;
        sum = fmaf(x, x, sum);
    }
    __device__ __forceinline__ void meet() {  // over a warp
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            far = fmaxf(far, __shfl_xor_sync(0xffffffffu, far, o));
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
    }
    // Squares of very large or small rows leave fp32: their sum is taken again in units of a power of two (of 2^-60 or more, so that
    // eps, at most 1, over its square stays within fp32).
    __device__ __forceinline__ float unit() const {
        return far > 1.0e15f || (far < 1.0e-15f && far > 0.0f) ? exp2f((float)max(ilogbf(far), -60)) : 1.0f;
    }
    __device__ __forceinline__ float inverse() const { return top >= 7.888609052210118e-31f ? __fmul_rn(__frcp_rn(top), 127.0f) : 0.0f; }
    // The row's scale, and what f is multiplied with for its code.  Rows whose largest |f| is below 2^-100 are zero
    // (inv is 1e-36 at least otherwise).
    __device__ __forceinline__ float scale(int K, float eps, float unit, float& inv) const {
        const float iu = 1.0f / unit, mean = fmaf(eps * iu, iu, sum / (float)K);
        inv = mean > 0.0f ? inverse() : 0.0f;
        return inv != 0.0f ? __fmul_rn(top, 1.0f / 127.0f) * iu * __frsqrt_rn(mean) : 0.0f;
    }
};

bool batch_ok(const fxpq_kv_batch* b);
bool cache_ok(const fxpq_kv_cache* c);

// Rows as fp16 in memory, half_pitch(K) apart, 256-byte aligned, zeros behind K: 8-bit codes of float rows (half_codes), and the product
// of such rows with 8-bit weights, y = (rows . w^T) * sx * sw + bias (null: ones, ones, zeros; fxpq_linear.cu).
// early: the product may be set up while the codes are formed (pdl_next).
struct RowNorm {
    const float* weight;  // null: no norm
    float eps;
    int vec, early;  // weight is 16-byte aligned
};
size_t half_pitch(int32_t K);
fxpq_status half_codes(const void* d_x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride, __half* codes, float* scale, const RowNorm& norm,
                       cudaStream_t st);
fxpq_status half_product(const __half* rows, const float* sx, const int8_t* d_w, int64_t w_stride, const float* sw, const float* bias, int64_t M,
                         int32_t N, int32_t K, int32_t y_type, void* d_y, int64_t y_stride, cudaStream_t st);

}  // namespace llm
}  // namespace fxpq
