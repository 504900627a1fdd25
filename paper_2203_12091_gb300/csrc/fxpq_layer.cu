// fxpq_layer.cu -- layers with 8-bit weights and what stands around their products: a norm before, activation, gate and residual
// after, and the gradient to their rows.
#include <cfloat>
#include <type_traits>

#include "fxpq_layer_few.cuh"

namespace fxpq {
namespace llm {
namespace {

// ------------------------------------------------------------------ rows of the gradient
struct GradRows {
    const void* dy;
    long long dy_stride;
    const void* pre;
    const float *sx, *sw, *bias;
    float pre_unit;
    int pre_f32, act, gated, N, early;
    __half* rows;
    long long pitch, M;
    float* scale;
    int* status;
};

// dz * sw of one row, as fp16 with a power of two of the row's own; SPLIT: in two parts, integers up to 2^11 (exact in
// fp16, as are their products' sums below 2^24), the lower ones M rows further on.
template <typename Y, bool SPLIT>
__global__ void __launch_bounds__(256) grad_rows_kernel(GradRows G) {
    pdl_wait();
    if (G.early) pdl_next();
    const long long m = blockIdx.x;
    const int t = threadIdx.x, N = G.N;
    const Y* dy = static_cast<const Y*>(G.dy) + m * G.dy_stride;
    const bool needs = G.gated || G.act != FXPQ_ACT_NONE;
    const float sx = needs ? __ldg(G.sx + m) : 0.0f;
    auto z = [&](int n) {
        const float a = G.pre_f32 ? static_cast<const float*>(G.pre)[m * N + n] : __half2float(static_cast<const __half*>(G.pre)[m * N + n]) * G.pre_unit;
        return fmaf(a * sx, __ldg(G.sw + n), G.bias ? __ldg(G.bias + n) : 0.0f);
    };
    auto pair = [&](int i, float& a, float& b) {  // channels 2 i, 2 i + 1
        const int n = 2 * i;
        float slope;
        if (G.gated) {
            const float f = activate_slope(z(n), G.act, slope), d = to_f32(dy[i]);
            a = d * z(n + 1) * slope, b = d * f;
        } else {
            a = to_f32(dy[n]), b = n + 1 < N ? to_f32(dy[n + 1]) : 0.0f;
            if (needs) {
                activate_slope(z(n), G.act, slope);
                a *= slope;
                if (n + 1 < N) {
                    activate_slope(z(n + 1), G.act, slope);
                    b *= slope;
                }
            }
        }
        a *= __ldg(G.sw + n);
        b = n + 1 < N ? b * __ldg(G.sw + n + 1) : 0.0f;
    };
    __shared__ uint32_t part[8];
    const int pairs = (N + 1) / 2;
    uint32_t top = 0;
    for (int i = t; i < pairs; i += 256) {
        float a, b;
        pair(i, a, b);
        top = max(top, max(__float_as_uint(a) & 0x7fffffffu, __float_as_uint(b) & 0x7fffffffu));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if ((t & 31) == 0) part[t >> 5] = top;
    __syncthreads();
    for (int w = 0; w < 8; ++w) top = max(top, part[w]);
    const bool bad = top >= 0x7f800000u;
    if (bad && t == 0) latch_status(G.status, FXPQ_ERR_NONFINITE);
    // top < 2^e; the row's largest value lies in [2^14, 2^15), or as an integer in [2^22, 2^23)
    const int e = max(top ? ilogbf(__uint_as_float(top)) + 1 : 0, -100);
    constexpr int UP = SPLIT ? 23 : 15;
    const float lift = bad || top == 0 ? 0.0f : ldexpf(1.0f, UP - e);
    if (t == 0) G.scale[m] = bad ? __int_as_float(0x7fffffff) : ldexpf(1.0f, e - UP);
    __half2* hi = reinterpret_cast<__half2*>(G.rows + m * G.pitch);
    __half2* lo = reinterpret_cast<__half2*>(G.rows + (G.M + m) * G.pitch);
    for (int i = t; i < G.pitch / 2; i += 256) {
        float a = 0.0f, b = 0.0f;
        if (i < pairs && lift != 0.0f) pair(i, a, b);
        a *= lift, b *= lift;
        if (SPLIT) {
            const float ha = rintf(a * (1.0f / 4096.0f)), hb = rintf(b * (1.0f / 4096.0f));
            hi[i] = __floats2half2_rn(ha, hb);
            lo[i] = __floats2half2_rn(rintf(fmaf(ha, -4096.0f, a)), rintf(fmaf(hb, -4096.0f, b)));
        } else {
            hi[i] = __floats2half2_rn(a, b);
        }
    }
}

// dx = (4096 high sums + low sums) * scale
__global__ void __launch_bounds__(256) join_parts_kernel(const float* __restrict__ sums, const float* __restrict__ scale, long long M, int K,
                                                         float* __restrict__ dx, long long dx_stride) {
    pdl_wait();
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < M * K; i += (long long)gridDim.x * 256) {
        const long long m = i / K;
        dx[m * dx_stride + (i - m * K)] = fmaf(sums[i], 4096.0f, sums[M * K + i]) * __ldg(scale + m);
    }
}

unsigned blocks_of(long long n) {
    const long long b = (n + 255) / 256, most = 64LL * num_sms();
    return (unsigned)(b < most ? b : most);
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Strides and alignment of rows of n values of `type`.
bool rows_fit(const void* p, int type, int64_t M, int64_t n, int64_t stride) {
    return p && aligned(p, ftype_bytes(type)) && (M <= 1 || stride >= n);
}

struct LayerSpace {
    size_t codes, end;
    explicit LayerSpace(const fxpq_layer& d) {
        codes = end = 0;
        if (float_rows_fit(d.M, d.K)) return;
        codes = up256((size_t)d.M * half_pitch(d.K) * 2);
        end = codes + up256((size_t)d.M * 4);
    }
};
bool sizes_ok(int64_t M, int32_t N, int32_t K) { return M >= 0 && N >= 0 && K >= 0 && M <= INT32_MAX; }

struct GradSpace {
    size_t rows, scale, sums, end;
    explicit GradSpace(const fxpq_layer_grad& d) {
        const int parts = d.dx_type == FXPQ_FT_F32 ? 2 : 1;
        rows = up256((size_t)parts * d.M * half_pitch(d.N) * 2);
        scale = rows + up256((size_t)d.M * 4);
        sums = scale;
        end = sums + (parts == 2 ? up256((size_t)parts * d.M * d.K * 4) : 0);
    }
};

// y of rows as fp16: what a layer's forward pass and its gradient have in common.
struct Product {
    const __half* rows;
    const float* scale;
    const int8_t* w;
    int64_t w_stride;
    const float *sw, *bias;
    int64_t M;
    int32_t N, K, y_type;
    void* y;
    int64_t y_stride;
};
template <int EPI>
fxpq_status product(const Product& p, const Epi& e, cudaStream_t st) {
    const int64_t pitch = (int64_t)half_pitch(p.K);
    if (many_tokens(p.M, p.N, p.K))
        return product_many<EPI>(p.rows, (size_t)pitch, p.scale, p.w, p.w_stride, p.sw, p.bias, p.M, p.N, p.K, p.y_type, p.y, p.y_stride, st, e);
    return few_product<EPI>(p.rows, pitch, p.scale, p.w, p.w_stride, p.sw, p.bias, p.M, p.N, p.K, p.y_type, p.y, p.y_stride, st, e, nullptr, true);
}

template <typename F>
void by_type(int type, F&& f) {
    if (type == FXPQ_FT_F32)
        f(float());
    else if (type == FXPQ_FT_F16)
        f(__half());
    else
        f(__nv_bfloat16());
}

}  // namespace
}  // namespace llm
}  // namespace fxpq

using namespace fxpq;
using namespace fxpq::llm;

extern "C" size_t fxpq_layer_workspace(const fxpq_layer* d) {
    if (!d || !sizes_ok(d->M, d->N, d->K) || d->M == 0 || d->N == 0) return 0;
    return LayerSpace(*d).end;
}

extern "C" fxpq_status fxpq_layer_forward(const fxpq_layer* layer, void* d_ws, size_t ws_bytes, void* stream) {
    if (!layer) return FXPQ_ERR_INVALID_ARG;
    const fxpq_layer& d = *layer;
    if (!sizes_ok(d.M, d.N, d.K) || !ftype_ok(d.x_type) || !ftype_ok(d.y_type) || !act_ok(d.activation) || d.gated < 0 || d.gated > 1 ||
        !(d.eps >= 0.0f && d.eps <= 1.0f) || (d.pre_type != FXPQ_FT_F16 && d.pre_type != FXPQ_FT_F32))
        return FXPQ_ERR_INVALID_ARG;
    if (d.gated && (d.N % 2 || d.activation == FXPQ_ACT_NONE || d.d_residual)) return FXPQ_ERR_INVALID_ARG;
    if (d.M == 0 || d.N == 0) return FXPQ_OK;
    const int wide = d.gated ? d.N / 2 : d.N;
    if ((d.K > 0 && (!rows_fit(d.d_x, d.x_type, d.M, d.K, d.x_stride) || !d.d_w || !aligned(d.d_w, 16) || d.w_stride % 16 || d.w_stride < d.K)) ||
        !d.d_sw || !aligned(d.d_sw, 4) || !aligned(d.d_bias, 4) || !aligned(d.d_norm, 4) || !aligned(d.d_sx, 4) ||
        !rows_fit(d.d_y, d.y_type, d.M, wide, d.y_stride) || (d.d_residual && !rows_fit(d.d_residual, d.y_type, d.M, d.N, d.residual_stride)) ||
        !aligned(d.d_pre, ftype_bytes(d.pre_type)))
        return FXPQ_ERR_INVALID_ARG;
    const LayerSpace at(d);
    if (at.end && (!d_ws || ws_bytes < at.end || !aligned(d_ws, 256))) return FXPQ_ERR_WORKSPACE;
    cudaStream_t st = as_stream(stream);
    const RowNorm norm = {d.d_norm, d.eps, aligned(d.d_norm, 16), !many_tokens(d.M, d.N, d.K)};
    const Epi e = {d.d_residual, d.residual_stride, d.d_pre, 1.0f / (float)(1LL << sum_shift(d.K)), d.pre_type == FXPQ_FT_F32, d.activation};
    if (at.end == 0) {
        const int vec = aligned(d.d_x, 16) && d.x_stride * ftype_bytes(d.x_type) % 16 == 0;
        const FloatRows rows = {d.d_x, d.x_stride, d.x_type, vec, d.K, d.d_sx, norm};
        const auto few = d.gated ? few_product<GATED> : few_product<LAYER>;
        return few(nullptr, 0, nullptr, d.d_w, d.w_stride, d.d_sw, d.d_bias, d.M, d.N, d.K, d.y_type, d.d_y, d.y_stride, st, e, &rows, false);
    }
    char* ws = static_cast<char*>(d_ws);
    __half* codes = reinterpret_cast<__half*>(ws);
    float* scale = d.d_sx ? d.d_sx : reinterpret_cast<float*>(ws + at.codes);
    const fxpq_status rc = half_codes(d.d_x, d.x_type, d.M, d.K, d.x_stride, codes, scale, norm, st);
    if (rc != FXPQ_OK) return rc;
    const Product p = {codes, scale, d.d_w, d.w_stride, d.d_sw, d.d_bias, d.M, d.N, d.K, d.y_type, d.d_y, d.y_stride};
    return d.gated ? product<GATED>(p, e, st) : product<LAYER>(p, e, st);
}

extern "C" size_t fxpq_layer_gradient_workspace(const fxpq_layer_grad* d) {
    if (!d || !sizes_ok(d->M, d->N, d->K) || d->M == 0 || d->K == 0 || d->M > INT32_MAX / 2) return 0;
    return GradSpace(*d).end;
}

extern "C" fxpq_status fxpq_layer_gradient(const fxpq_layer_grad* grad, void* d_ws, size_t ws_bytes, void* stream) {
    if (!grad) return FXPQ_ERR_INVALID_ARG;
    const fxpq_layer_grad& d = *grad;
    if (!sizes_ok(d.M, d.N, d.K) || d.M > INT32_MAX / 2 || !ftype_ok(d.y_type) || !ftype_ok(d.dx_type) || !act_ok(d.activation) || d.gated < 0 ||
        d.gated > 1 || (d.pre_type != FXPQ_FT_F16 && d.pre_type != FXPQ_FT_F32))
        return FXPQ_ERR_INVALID_ARG;
    if (d.gated && (d.N % 2 || d.activation == FXPQ_ACT_NONE)) return FXPQ_ERR_INVALID_ARG;
    if (d.M == 0 || d.K == 0) return FXPQ_OK;
    const int wide = d.gated ? d.N / 2 : d.N;
    if (!rows_fit(d.d_dx, d.dx_type, d.M, d.K, d.dx_stride) ||
        (d.N > 0 && (!rows_fit(d.d_dy, d.y_type, d.M, wide, d.dy_stride) || !d.d_sw || !aligned(d.d_sw, 4) || !aligned(d.d_bias, 4) || !d.d_wt ||
                     !aligned(d.d_wt, 16) || d.wt_stride % 16 || d.wt_stride < d.N)))
        return FXPQ_ERR_INVALID_ARG;
    if (d.N > 0 && d.activation != FXPQ_ACT_NONE && (!d.d_pre || !d.d_sx || !aligned(d.d_pre, ftype_bytes(d.pre_type)) || !aligned(d.d_sx, 4)))
        return FXPQ_ERR_INVALID_ARG;
    const GradSpace at(d);
    if (!d_ws || ws_bytes < at.end || !aligned(d_ws, 256)) return FXPQ_ERR_WORKSPACE;
    char* ws = static_cast<char*>(d_ws);
    cudaStream_t st = as_stream(stream);
    __half* rows = reinterpret_cast<__half*>(ws);
    float* scale = reinterpret_cast<float*>(ws + at.rows);
    float* sums = reinterpret_cast<float*>(ws + at.sums);
    const bool split = d.dx_type == FXPQ_FT_F32;
    GradRows G = {d.d_dy, d.dy_stride, d.d_pre, d.d_sx, d.d_sw, d.d_bias, (float)(1LL << sum_shift(d.K)), d.pre_type == FXPQ_FT_F32,
                  d.activation, d.gated, d.N, !many_tokens(split ? 2 * d.M : d.M, d.K, d.N), rows, (long long)half_pitch(d.N), (long long)d.M, scale, status_ptr()};
    by_type(d.y_type, [&](auto t) {
        using Y = decltype(t);
        if (split)
            launch_pdl(grad_rows_kernel<Y, true>, dim3((unsigned)d.M), dim3(256), 0, st, G);
        else
            launch_pdl(grad_rows_kernel<Y, false>, dim3((unsigned)d.M), dim3(256), 0, st, G);
    });
    fxpq_status rc = after_launch("layer_grad_rows");
    if (rc != FXPQ_OK) return rc;
    if (!split) return product<LAYER>({rows, scale, d.d_wt, d.wt_stride, nullptr, nullptr, d.M, d.K, d.N, d.dx_type, d.d_dx, d.dx_stride}, {}, st);
    rc = product<LAYER>({rows, nullptr, d.d_wt, d.wt_stride, nullptr, nullptr, 2 * d.M, d.K, d.N, FXPQ_FT_F32, sums, d.K}, {}, st);
    if (rc != FXPQ_OK) return rc;
    launch_pdl(join_parts_kernel, dim3(blocks_of(d.M * d.K)), dim3(256), 0, st, static_cast<const float*>(sums), static_cast<const float*>(scale), (long long)d.M,
               (int)d.K, static_cast<float*>(d.d_dx), (long long)d.dx_stride);
    return after_launch("layer_join_parts");
}
