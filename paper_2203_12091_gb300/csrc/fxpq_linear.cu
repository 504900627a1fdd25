// fxpq_linear.cu -- rows quantized to 8 bits with a scale each, and the product of 8-bit rows with scales for
// each token and each output channel.
#include <atomic>
#include <cfloat>
#include <type_traits>

#include "fxpq_linear.cuh"

namespace fxpq {
namespace llm {
namespace {

// One block per row: the row stays in registers as it came (QT_KEEP steps of 8 values per thread; longer rows are read
// again, from L2) between the maximum and the codes.  Bytes bound it, so what counts is rows in flight: magnitudes are
// compared as bits, with infinities and NaN sorted out only where one is found, and codes are rounded by adding 1.5 * 2^23.
// Rows of more than 8192 values take 1024 threads: 64 rows of 25088 4.2 us with 256, 3.1 with 1024.
constexpr int QT_KEEP = 4;

template <typename T>
struct Raw8 {
    alignas(16) T v[8];
    __device__ __forceinline__ void load(const T* __restrict__ p, bool vec) {
        if (vec) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(v)[i] = reinterpret_cast<const uint4*>(p)[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p[i];
        }
    }
};

// C: int8 codes, or fp16 ones for the tensor-core kernels that take them so.
// NORM: codes of f = x * weight, which are those of f / rms; the root mean square goes into the scale.
template <typename T, typename C, int QT_THREADS, bool NORM>
__global__ void __launch_bounds__(QT_THREADS)
    quantize_tokens_kernel(const T* __restrict__ x, int K, long long x_stride, int vec, C* __restrict__ codes, long long c_stride, int c_vec,
                           float* __restrict__ scale, int* status, const __grid_constant__ RowNorm norm) {
    constexpr bool HALF = sizeof(C) == 2;
    pdl_wait();
    if (norm.early) pdl_next();
    const T* row = x + (long long)blockIdx.x * x_stride;
    C* out = codes + (long long)blockIdx.x * c_stride;
    const int t = threadIdx.x, groups = K / 8, tail = 8 * groups + t;  // whole groups of eight; the rest of the row one value at a time
    Raw8<T> keep[QT_KEEP];
    auto each = [&](auto&& f) {  // f(group, its values) for this thread's groups
#pragma unroll
        for (int s = 0; s < QT_KEEP; ++s)
            if (t + s * QT_THREADS < groups) f(t + s * QT_THREADS, keep[s]);
        for (int g = t + QT_KEEP * QT_THREADS; g < groups; g += QT_THREADS) {
            Raw8<T> v;
            v.load(row + 8 * g, vec);
            f(g, v);
        }
    };
#pragma unroll
    for (int s = 0; s < QT_KEEP; ++s)
        if (t + s * QT_THREADS < groups) keep[s].load(row + 8 * (t + s * QT_THREADS), vec);
    __shared__ uint32_t part[QT_THREADS / 32];
    if constexpr (NORM) {
        __shared__ float parts[3][QT_THREADS / 32];
        __shared__ float row_inv;
        float wt[8];
        auto weights = [&](int g) { load_f32<8>(norm.weight + 8 * g, norm.vec, wt); };
        RowStats st;
        each([&](int g, const Raw8<T>& v) {
            weights(g);
#pragma unroll
            for (int e = 0; e < 8; ++e) st.see(to_f32(v.v[e]), wt[e], 1.0f);
        });
        if (tail < K) st.see(to_f32(row[tail]), __ldg(norm.weight + tail), 1.0f);
        const bool bad = __syncthreads_or(st.bad);
        auto meet = [&]() {  // the block's statistics, in thread 0's warp
            st.meet();
            if ((t & 31) == 0) parts[0][t >> 5] = st.top, parts[1][t >> 5] = st.far, parts[2][t >> 5] = st.sum;
            __syncthreads();
            if (t < 32) {
                const bool in = t < QT_THREADS / 32;
                st.top = in ? parts[0][t] : 0.0f, st.far = in ? parts[1][t] : 0.0f, st.sum = in ? parts[2][t] : 0.0f;
                st.meet();
            }
        };
        meet();
        if (t == 0) parts[0][0] = st.unit();
        __syncthreads();
        const float unit = parts[0][0];
        if (unit != 1.0f) {  // (the block agrees)
            __syncthreads();
            st = RowStats();
            each([&](int g, const Raw8<T>& v) {
                weights(g);
#pragma unroll
                for (int e = 0; e < 8; ++e) st.see(to_f32(v.v[e]), wt[e], 1.0f / unit);
            });
            if (tail < K) st.see(to_f32(row[tail]), __ldg(norm.weight + tail), 1.0f / unit);
            meet();
        }
        if (t == 0) {
            float inv;
            scale[blockIdx.x] = st.scale(K, norm.eps, unit, inv);
            row_inv = inv;
            if (bad) latch_status(status, FXPQ_ERR_NONFINITE);
        }
        __syncthreads();
        const float inv = row_inv;
        each([&](int g, const Raw8<T>& v) {
            weights(g);
            float c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = __fmul_rn(RowStats::value(to_f32(v.v[e]), wt[e]), inv);
            *reinterpret_cast<uint4*>(out + 8 * g) =
                make_uint4(f32_codes_f16x2(c[0], c[1]), f32_codes_f16x2(c[2], c[3]), f32_codes_f16x2(c[4], c[5]), f32_codes_f16x2(c[6], c[7]));
        });
        if (tail < K) out[tail] = (C)(int)rintf(__fmul_rn(RowStats::value(to_f32(row[tail]), __ldg(norm.weight + tail)), inv));
        for (long long i = K + t; i < c_stride; i += QT_THREADS) out[i] = (C)0;
        return;
    }
    auto largest = [&](bool finite) {  // magnitudes as bits
        uint32_t top = 0;
        auto see = [&](float v) {
            const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
            top = max(top, finite && b >= 0x7f800000u ? 0u : b);
        };
        each([&](int, const Raw8<T>& v) {
#pragma unroll
            for (int e = 0; e < 8; ++e) see(to_f32(v.v[e]));
        });
        if (tail < K) see(to_f32(row[tail]));
        top = __reduce_max_sync(0xffffffffu, top);
        __syncthreads();
        if ((t & 31) == 0) part[t >> 5] = top;
        __syncthreads();
        top = 0;
#pragma unroll
        for (int w = 0; w < QT_THREADS / 32; ++w) top = max(top, part[w]);
        return top;
    };
    uint32_t bits = largest(false);
    const bool bad = bits >= 0x7f800000u;
    if (bad) {
        if (t == 0) latch_status(status, FXPQ_ERR_NONFINITE);
        bits = largest(true);
    }
    const float top = __uint_as_float(bits);
    const bool live = top >= 7.888609052210118e-31f;  // 2^-100
    const float inv = live ? __fmul_rn(__frcp_rn(top), 127.0f) : 0.0f;
    if (t == 0) scale[blockIdx.x] = live ? __fmul_rn(top, 1.0f / 127.0f) : 0.0f;
    // (a product is at most 127 (1 + 2^-22) and rounds to 127)
    auto scaled = [&](T v) {
        const float f = to_f32(v);
        return __fmul_rn(bad && !(fabsf(f) <= FLT_MAX) ? 0.0f : f, inv);
    };
    auto code = [&](T v) { return (int)(int8_t)__float_as_uint(scaled(v) + 12582912.0f); };
    each([&](int g, const Raw8<T>& v) {
        if constexpr (HALF) {  // (always aligned)
            *reinterpret_cast<uint4*>(out + 8 * g) =
                make_uint4(f32_codes_f16x2(scaled(v.v[0]), scaled(v.v[1])), f32_codes_f16x2(scaled(v.v[2]), scaled(v.v[3])),
                           f32_codes_f16x2(scaled(v.v[4]), scaled(v.v[5])), f32_codes_f16x2(scaled(v.v[6]), scaled(v.v[7])));
        } else {
            int c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = code(v.v[e]);
            if (c_vec)
                *reinterpret_cast<uint2*>(out + 8 * g) = make_uint2(pack_i8(c[0], c[1], c[2], c[3]), pack_i8(c[4], c[5], c[6], c[7]));
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) out[8 * g + e] = (C)c[e];
        }
    });
    if (tail < K) out[tail] = (C)code(row[tail]);
    for (long long i = K + t; i < c_stride; i += QT_THREADS) out[i] = (C)0;
}

// int8 rows to fp16 codes, 16 per thread.
__global__ void __launch_bounds__(256) expand_codes_kernel(const int8_t* __restrict__ x, long long x_stride, int chunks, __half* __restrict__ y,
                                                           long long y_stride) {
    pdl_wait();
    const long long m = blockIdx.y;
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= chunks) return;
    const uint4 v = *reinterpret_cast<const uint4*>(x + m * x_stride + 16 * c);
    const uint32_t w[4] = {v.x ^ 0x80808080u, v.y ^ 0x80808080u, v.z ^ 0x80808080u, v.w ^ 0x80808080u};
    uint4* dst = reinterpret_cast<uint4*>(y + m * y_stride + 16 * c);
    dst[0] = make_uint4(code_pair(w[0], LOW_PAIR), code_pair(w[0], HIGH_PAIR), code_pair(w[1], LOW_PAIR), code_pair(w[1], HIGH_PAIR));
    dst[1] = make_uint4(code_pair(w[2], LOW_PAIR), code_pair(w[2], HIGH_PAIR), code_pair(w[3], LOW_PAIR), code_pair(w[3], HIGH_PAIR));
}

}  // namespace
}  // namespace llm
}  // namespace fxpq

using namespace fxpq;
using namespace fxpq::llm;

namespace {
template <typename C>
fxpq_status quantize_rows(const void* d_x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride, C* d_codes, int64_t codes_stride,
                          float* d_scale, cudaStream_t st, const RowNorm& norm = {}) {
    const int e = ftype_bytes(x_type), vec = aligned(d_x, 16) && x_stride * e % 16 == 0;
    const int c_vec = aligned(d_codes, 8) && codes_stride % 8 == 0;
    const dim3 grid((unsigned)M);
    int* status = status_ptr();
    auto launch = [&](auto* x) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(x)>>;
        auto go = [&](auto threads, auto normed) {
            constexpr int THREADS = decltype(threads)::value;
            launch_pdl(quantize_tokens_kernel<T, C, THREADS, decltype(normed)::value>, grid, dim3(THREADS), 0, st, x, K, x_stride, vec, d_codes,
                       codes_stride, c_vec, d_scale, status, norm);
        };
        auto sized = [&](auto normed) {
            if (K <= 4096)
                go(std::integral_constant<int, 128>(), normed);
            else if (K > 8192)
                go(std::integral_constant<int, 1024>(), normed);
            else
                go(std::integral_constant<int, 256>(), normed);
        };
        if constexpr (sizeof(C) == 2)
            if (norm.weight) return sized(std::true_type());
        sized(std::false_type());
    };
    if (x_type == FXPQ_FT_F32)
        launch(static_cast<const float*>(d_x));
    else if (x_type == FXPQ_FT_F16)
        launch(static_cast<const __half*>(d_x));
    else
        launch(static_cast<const __nv_bfloat16*>(d_x));
    return after_launch("quantize_tokens");
}

bool rows_ok(const void* d_x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride) {
    return ftype_ok(x_type) && M >= 0 && K >= 0 && M <= INT32_MAX && (M == 0 || K == 0 || d_x) && (M <= 1 || x_stride >= K) &&
           aligned(d_x, ftype_bytes(x_type));
}
}  // namespace

extern "C" fxpq_status fxpq_quantize_tokens(const void* d_x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride, int8_t* d_codes,
                                            int64_t codes_stride, float* d_scale, void* stream) {
    if (!rows_ok(d_x, x_type, M, K, x_stride) || codes_stride < K || (M > 0 && !d_scale) || (M > 0 && codes_stride > 0 && !d_codes) || !aligned(d_scale, 4))
        return FXPQ_ERR_INVALID_ARG;
    if (M == 0) return FXPQ_OK;
    return quantize_rows(d_x, x_type, M, K, x_stride, d_codes, codes_stride, d_scale, as_stream(stream));
}

extern "C" size_t fxpq_linear_i8_workspace(int64_t M, int32_t N, int32_t K) {
    return M > 0 && many_tokens(M, N, K) ? ((size_t)M * codes_pitch(K) * sizeof(__half) + 255) / 256 * 256 : 0;
}

namespace {
fxpq_status check_linear(const int8_t* d_x, int64_t x_stride, const float* d_sx, const int8_t* d_w, int64_t w_stride, const float* d_sw,
                         const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type, const void* d_y, int64_t y_stride) {
    if (M < 0 || N < 0 || K < 0 || M > INT32_MAX || !ftype_ok(y_type)) return FXPQ_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return FXPQ_OK;
    if (!d_sx || !d_sw || !d_y || (K > 0 && (!d_x || !d_w)) || !aligned(d_x, 16) || !aligned(d_w, 16) || x_stride % 16 || w_stride % 16 ||
        x_stride < K || w_stride < K || y_stride < N || !aligned(d_y, ftype_bytes(y_type)) || !aligned(d_sx, 4) || !aligned(d_sw, 4) ||
        !aligned(d_bias, 4))
        return FXPQ_ERR_INVALID_ARG;
    return FXPQ_OK;
}

}  // namespace

extern "C" fxpq_status fxpq_linear_i8(const int8_t* d_x, int64_t x_stride, const float* d_sx, const int8_t* d_w, int64_t w_stride,
                                      const float* d_sw, const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type,
                                      void* d_y, int64_t y_stride, void* d_ws, size_t ws_bytes, void* stream) {
    const fxpq_status bad = check_linear(d_x, x_stride, d_sx, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride);
    if (bad != FXPQ_OK) return bad;
    if (M == 0 || N == 0) return FXPQ_OK;
    const size_t need = fxpq_linear_i8_workspace(M, N, K);
    if (need && (!d_ws || ws_bytes < need || !aligned(d_ws, 256))) return FXPQ_ERR_WORKSPACE;
    if (many_tokens(M, N, K)) {
        const size_t pitch = codes_pitch(K);
        if (pitch > (size_t)INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
        __half* half = static_cast<__half*>(d_ws);
        for (int64_t m = 0; m < M; m += 65535) {  // (the grid's second dimension)
            const int64_t rows = M - m < 65535 ? M - m : 65535;
            launch_pdl(expand_codes_kernel, dim3((unsigned)((pitch / 16 + 255) / 256), (unsigned)rows), dim3(256), 0, as_stream(stream),
                       d_x + m * x_stride, x_stride, (int)(pitch / 16), half + m * pitch, (long long)pitch);
            const fxpq_status rc = after_launch("expand_codes");
            if (rc != FXPQ_OK) return rc;
        }
        return product_many<PLAIN>(half, pitch, d_sx, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, as_stream(stream));
    }
    return product_few<PLAIN>(d_x, nullptr, x_stride, d_sx, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, as_stream(stream));
}

namespace {
// The workspace of fxpq_linear_tokens: the tokens' fp16 codes, then their scales.
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
size_t tokens_codes(int64_t M, int32_t K) { return up256((size_t)M * codes_pitch(K) * sizeof(__half)); }
}  // namespace

extern "C" size_t fxpq_linear_tokens_workspace(int64_t M, int32_t N, int32_t K) {
    if (M <= 0 || N < 0 || K < 0) return 0;
    return tokens_codes(M, K) + up256((size_t)M * sizeof(float));
}

extern "C" fxpq_status fxpq_linear_tokens(const void* d_x, int32_t x_type, int64_t x_stride, const int8_t* d_w, int64_t w_stride,
                                          const float* d_sw, const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type,
                                          void* d_y, int64_t y_stride, void* d_ws, size_t ws_bytes, void* stream) {
    if (M < 0 || N < 0 || K < 0 || !rows_ok(d_x, x_type, M, K, x_stride) || !ftype_ok(y_type)) return FXPQ_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return FXPQ_OK;
    if (!d_ws || ws_bytes < fxpq_linear_tokens_workspace(M, N, K) || !aligned(d_ws, 256)) return FXPQ_ERR_WORKSPACE;
    const size_t pitch = codes_pitch(K);
    __half* half = static_cast<__half*>(d_ws);
    float* scale = reinterpret_cast<float*>(static_cast<char*>(d_ws) + tokens_codes(M, K));
    cudaStream_t st = as_stream(stream);
    const fxpq_status bad = check_linear(static_cast<int8_t*>(d_ws), (int64_t)pitch, scale, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride);
    if (bad != FXPQ_OK) return bad;  // (before anything is launched)
    const fxpq_status rc = quantize_rows(d_x, x_type, M, K, x_stride, half, (int64_t)pitch, scale, st);
    if (rc != FXPQ_OK) return rc;
    if (many_tokens(M, N, K)) return product_many<PLAIN>(half, pitch, scale, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, st);
    return product_few<PLAIN>(nullptr, half, (int64_t)pitch, scale, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, st);
}

namespace fxpq {
namespace llm {
size_t half_pitch(int32_t K) { return codes_pitch(K); }
fxpq_status half_codes(const void* d_x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride, __half* codes, float* scale, const RowNorm& norm,
                       cudaStream_t st) {
    return quantize_rows(d_x, x_type, M, K, x_stride, codes, (int64_t)codes_pitch(K), scale, st, norm);
}
fxpq_status half_product(const __half* rows, const float* sx, const int8_t* d_w, int64_t w_stride, const float* sw, const float* bias, int64_t M,
                         int32_t N, int32_t K, int32_t y_type, void* d_y, int64_t y_stride, cudaStream_t st) {
    const size_t pitch = codes_pitch(K);
    if (many_tokens(M, N, K)) return product_many<PLAIN>(rows, pitch, sx, d_w, w_stride, sw, bias, M, N, K, y_type, d_y, y_stride, st);
    return product_few<PLAIN>(nullptr, rows, (int64_t)pitch, sx, d_w, w_stride, sw, bias, M, N, K, y_type, d_y, y_stride, st);
}
}  // namespace llm
}  // namespace fxpq
