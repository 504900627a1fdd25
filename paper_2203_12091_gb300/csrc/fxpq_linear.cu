// fxpq_linear.cu -- rows quantized to 8 bits with a scale each, and the product of 8-bit rows with scales for
// each token and each output channel.
#include <cfloat>

#include "fxpq_llm.cuh"

namespace fxpq {
namespace llm {
namespace {

// One block per row: the row stays in registers between the maximum and the codes (KEEP steps of 8 values per
// thread; longer rows are read again, from L2).
constexpr int QT_THREADS = 256, QT_KEEP = 4;

template <typename T>
__global__ void __launch_bounds__(QT_THREADS) quantize_tokens_kernel(const T* __restrict__ x, int K, long long x_stride, int vec,
                                                                     int8_t* __restrict__ codes, long long c_stride, int c_vec,
                                                                     float* __restrict__ scale, int* status) {
    pdl_wait();
    const T* row = x + (long long)blockIdx.x * x_stride;
    int8_t* out = codes + (long long)blockIdx.x * c_stride;
    const int t = threadIdx.x, groups = K / 8;  // whole groups of eight; the rest of the row one value at a time
    float keep[QT_KEEP][8], tail = 0.0f, top = 0.0f;
    bool bad = false;
    auto see = [&](float& v) {
        const float u = fabsf(v);
        if (!(u <= FLT_MAX)) {
            bad = true;
            v = 0.0f;
        } else
            top = fmaxf(top, u);
    };
#pragma unroll
    for (int s = 0; s < QT_KEEP; ++s) {
        const int g = t + s * QT_THREADS;
        if (g < groups) {
            load_f32<8>(row + 8 * g, vec, keep[s]);
#pragma unroll
            for (int e = 0; e < 8; ++e) see(keep[s][e]);
        }
    }
    for (int g = t + QT_KEEP * QT_THREADS; g < groups; g += QT_THREADS) {
        float v[8];
        load_f32<8>(row + 8 * g, vec, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) see(v[e]);
    }
    if (t < K - 8 * groups) {
        tail = to_f32(row[8 * groups + t]);
        see(tail);
    }
    __shared__ float part[QT_THREADS / 32];
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if ((t & 31) == 0) part[t >> 5] = top;
    __syncthreads();
    top = part[0];
#pragma unroll
    for (int w = 1; w < QT_THREADS / 32; ++w) top = fmaxf(top, part[w]);
    if (bad) latch_status(status, FXPQ_ERR_NONFINITE);
    const bool live = top >= 7.888609052210118e-31f;  // 2^-100
    const float inv = live ? __fmul_rn(__frcp_rn(top), 127.0f) : 0.0f;
    if (t == 0) scale[blockIdx.x] = live ? __fmul_rn(top, 1.0f / 127.0f) : 0.0f;
    auto code = [&](float v) { return max(-127, min(127, __float2int_rn(__fmul_rn(v, inv)))); };
    auto put = [&](int g, const float (&v)[8]) {
        int c[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = code(v[e]);
        if (c_vec)
            *reinterpret_cast<uint2*>(out + 8 * g) = make_uint2(pack_i8(c[0], c[1], c[2], c[3]), pack_i8(c[4], c[5], c[6], c[7]));
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) out[8 * g + e] = (int8_t)c[e];
    };
#pragma unroll
    for (int s = 0; s < QT_KEEP; ++s)
        if (t + s * QT_THREADS < groups) put(t + s * QT_THREADS, keep[s]);
    for (int g = t + QT_KEEP * QT_THREADS; g < groups; g += QT_THREADS) {
        float v[8];
        load_f32<8>(row + 8 * g, vec, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fabsf(v[e]) <= FLT_MAX ? v[e] : 0.0f;
        put(g, v);
    }
    if (t < K - 8 * groups) out[8 * groups + t] = (int8_t)code(tail);
    for (long long i = K + t; i < c_stride; i += QT_THREADS) out[i] = 0;
}

struct LinArgs {
    const int8_t *x, *w;
    const float *sx, *sw, *bias;
    void* y;
    long long xs, ws, ys, M;
    int N, K, y_type;
};

__device__ __forceinline__ void store_y(void* y, int type, long long at, float v) {
    if (type == FXPQ_FT_F32)
        static_cast<float*>(y)[at] = v;
    else if (type == FXPQ_FT_F16)
        static_cast<__half*>(y)[at] = __float2half_rn(v);
    else
        static_cast<__nv_bfloat16*>(y)[at] = __float2bfloat16_rn(v);
}

// 64 x 64 outputs per block of 256 threads, 64 codes of the reduction at a time in shared memory.
__global__ void __launch_bounds__(256) linear_i8_kernel(const LinArgs A) {
    pdl_wait();
    __shared__ int sx[64][17], sw[64][17];
    const long long m0 = (long long)blockIdx.y * 64;
    const int n0 = blockIdx.x * 64, t = threadIdx.x, tx = t & 15, ty = t >> 4;
    int acc[4][4] = {};
    for (int k0 = 0; k0 < A.K; k0 += 64) {
        for (int i = t; i < 64 * 16; i += 256) {
            const int r = i / 16, k = k0 + 4 * (i % 16);
            int a = 0, b = 0;
            if (k < A.K) {
                const int mask = A.K - k >= 4 ? -1 : (1 << (8 * (A.K - k))) - 1;
                if (m0 + r < A.M) a = *reinterpret_cast<const int*>(A.x + (m0 + r) * A.xs + k) & mask;
                if (n0 + r < A.N) b = *reinterpret_cast<const int*>(A.w + (long long)(n0 + r) * A.ws + k) & mask;
            }
            sx[r][i % 16] = a;
            sw[r][i % 16] = b;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 16; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(sx[ty + 16 * i][q], sw[tx + 16 * j][q], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const long long m = m0 + ty + 16 * i;
            const int n = n0 + tx + 16 * j;
            if (m < A.M && n < A.N)
                store_y(A.y, A.y_type, m * A.ys + n, (float)acc[i][j] * A.sx[m] * A.sw[n] + (A.bias ? A.bias[n] : 0.0f));
        }
}

}  // namespace
}  // namespace llm
}  // namespace fxpq

using namespace fxpq;
using namespace fxpq::llm;

extern "C" fxpq_status fxpq_quantize_tokens(const void* d_x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride, int8_t* d_codes,
                                            int64_t codes_stride, float* d_scale, void* stream) {
    if (!ftype_ok(x_type) || M < 0 || K < 0 || M > INT32_MAX || codes_stride < K || (M > 0 && !d_scale) ||
        (M > 0 && K > 0 && (!d_x || !d_codes)) || (M > 1 && x_stride < K) || !aligned(d_x, ftype_bytes(x_type)) || !aligned(d_scale, 4))
        return FXPQ_ERR_INVALID_ARG;
    if (M == 0) return FXPQ_OK;
    const int e = ftype_bytes(x_type), vec = aligned(d_x, 16) && x_stride * e % 16 == 0;
    const int c_vec = aligned(d_codes, 8) && codes_stride % 8 == 0;
    const dim3 grid((unsigned)M), block(QT_THREADS);
    cudaStream_t st = as_stream(stream);
    int* status = status_ptr();
    if (x_type == FXPQ_FT_F32)
        launch_pdl(quantize_tokens_kernel<float>, grid, block, 0, st, static_cast<const float*>(d_x), K, x_stride, vec, d_codes,
                   codes_stride, c_vec, d_scale, status);
    else if (x_type == FXPQ_FT_F16)
        launch_pdl(quantize_tokens_kernel<__half>, grid, block, 0, st, static_cast<const __half*>(d_x), K, x_stride, vec, d_codes,
                   codes_stride, c_vec, d_scale, status);
    else
        launch_pdl(quantize_tokens_kernel<__nv_bfloat16>, grid, block, 0, st, static_cast<const __nv_bfloat16*>(d_x), K, x_stride, vec,
                   d_codes, codes_stride, c_vec, d_scale, status);
    return after_launch("quantize_tokens");
}

extern "C" size_t fxpq_linear_i8_workspace(int64_t M, int32_t N, int32_t K) {
    (void)M, (void)N, (void)K;
    return 0;
}

extern "C" fxpq_status fxpq_linear_i8(const int8_t* d_x, int64_t x_stride, const float* d_sx, const int8_t* d_w, int64_t w_stride,
                                      const float* d_sw, const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type,
                                      void* d_y, int64_t y_stride, void* d_ws, size_t ws_bytes, void* stream) {
    if (M < 0 || N < 0 || K < 0 || M > INT32_MAX || !ftype_ok(y_type)) return FXPQ_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return FXPQ_OK;
    if (!d_sx || !d_sw || !d_y || (K > 0 && (!d_x || !d_w)) || !aligned(d_x, 16) || !aligned(d_w, 16) || x_stride % 16 || w_stride % 16 ||
        x_stride < K || w_stride < K || y_stride < N || !aligned(d_y, ftype_bytes(y_type)) || !aligned(d_sx, 4) || !aligned(d_sw, 4) ||
        !aligned(d_bias, 4))
        return FXPQ_ERR_INVALID_ARG;
    const size_t need = fxpq_linear_i8_workspace(M, N, K);
    if (need && (!d_ws || ws_bytes < need || !aligned(d_ws, 256))) return FXPQ_ERR_WORKSPACE;
    const LinArgs A = {d_x, d_w, d_sx, d_sw, d_bias, d_y, x_stride, w_stride, y_stride, M, N, K, y_type};
    launch_pdl(linear_i8_kernel, dim3((unsigned)((N + 63) / 64), (unsigned)((M + 63) / 64)), dim3(256), 0, as_stream(stream), A);
    return after_launch("linear_i8");
}
