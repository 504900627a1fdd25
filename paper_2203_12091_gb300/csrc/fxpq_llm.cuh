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

// What the codes of a row of f = x * weight (f = x without a norm) need to know: the largest |f|, as bits, and with a norm the sum of x^2.
// NORM's values take four instructions.  Where the bits are those of an inf or NaN, or the sum left the middle of fp32's range,
// the row is looked at again by careful_row.
template <bool NORM>
struct RowScan {
    uint32_t top = 0;
    float sum = 0.0f;
    __device__ __forceinline__ void see(float x, float w) {
        if constexpr (NORM) sum = fmaf(x, x, sum);
        top = max(top, __float_as_uint(NORM ? __fmul_rn(x, w) : x) & 0x7fffffffu);
    }
    __device__ __forceinline__ void meet() {  // over a warp
        top = __reduce_max_sync(0xffffffffu, top);
        if constexpr (NORM) {
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
    }
    __device__ __forceinline__ void join(uint32_t t, float s) { top = max(top, t), sum += s; }
    __device__ __forceinline__ bool odd() const { return top >= 0x7f800000u || (NORM && top && !(sum > 1.0e-25f && sum < 1.0e30f)); }
    // What f is multiplied with for its code.  Rows whose largest |f| is below 2^-100 are zero (inv is 1e-37 at least otherwise).
    static __device__ __forceinline__ float inverse(float top) { return top >= 7.888609052210118e-31f ? __fmul_rn(__frcp_rn(top), 127.0f) : 0.0f; }
    __device__ __forceinline__ float inverse() const { return inverse(__uint_as_float(top)); }
    __device__ __forceinline__ float scale(int K, float eps) const {
        if (inverse() == 0.0f) return 0.0f;
        const float s = __fmul_rn(__uint_as_float(top), 1.0f / 127.0f);
        return NORM ? s * __frsqrt_rn(sum / (float)K + eps) : s;
    }
};
// f as a code before rounding: what is not finite counts as 0.
__device__ __forceinline__ float scaled_code(float f, float inv) {
    const float c = __fmul_rn(f, inv);
    return fabsf(c) <= 128.0f ? c : 0.0f;
}
// The same numbers for any row, by one warp: values that are not finite do not count (x in the sum only if it is not finite itself), and the
// squares are taken in units of a power of two (2^-60 or more, so that eps, at most 1, over its square stays within fp32).
template <typename T>
__device__ __noinline__ void careful_row(const T* row, int K, const float* weight, float eps, float& inv, float& scale, int* status) {
    constexpr float FINITE = 3.402823466e38f;
    float top = 0.0f, far = 0.0f, sum = 0.0f;
    bool bad = false;
    const int lane = threadIdx.x & 31;
    for (int k = lane; k < K; k += 32) {
        const float x = to_f32(row[k]), f = weight ? __fmul_rn(x, __ldg(weight + k)) : x;
        const bool x_fine = fabsf(x) <= FINITE, fine = x_fine && fabsf(f) <= FINITE;
        bad |= !fine;
        if (fine) top = fmaxf(top, fabsf(f));
        if (x_fine) far = fmaxf(far, fabsf(x));
    }
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
    far = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(far)));
    inv = RowScan<true>::inverse(top);
    scale = inv != 0.0f ? __fmul_rn(top, 1.0f / 127.0f) : 0.0f;
    if (__any_sync(0xffffffffu, bad) && lane == 0) latch_status(status, FXPQ_ERR_NONFINITE);
    if (!weight || inv == 0.0f) return;
    const float iu = 1.0f / exp2f((float)max(far > 0.0f ? ilogbf(far) : 0, -60));
    for (int k = lane; k < K; k += 32) {
        const float x = to_f32(row[k]) * iu;
        if (fabsf(x) <= 2.0f) sum = fmaf(x, x, sum);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float mean = fmaf(eps * iu, iu, sum / (float)K);
    if (mean > 0.0f)
        scale *= iu * __frsqrt_rn(mean);
    else
        inv = scale = 0.0f;
}

bool batch_ok(const fxpq_kv_batch* b);
bool cache_ok(const fxpq_kv_cache* c);

// Float rows to 8-bit codes as fp16, half_pitch(K) apart, zeros behind K (fxpq_linear.cu), under a norm or not.
// early: the product may be set up from the first block's start on (1), or as the codes are written (2; pdl_next).
struct RowNorm {
    const float* weight;  // null: no norm
    float eps;
    int vec, early;  // weight is 16-byte aligned
};
size_t half_pitch(int32_t K);
fxpq_status half_codes(const void* d_x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride, __half* codes, float* scale, const RowNorm& norm,
                       cudaStream_t st);

}  // namespace llm
}  // namespace fxpq
