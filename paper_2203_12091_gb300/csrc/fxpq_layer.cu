// fxpq_layer.cu -- layers with 8-bit weights and what stands around their products: a norm before, activation, gate and residual
// after, and the gradient to their rows.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "fxpq_layer_few.cuh"

namespace fxpq {
namespace llm {
namespace {

// dx = (PART first sums + second sums) * scale, a block a row (and 1024 of its values).
__global__ void __launch_bounds__(256) join_parts_kernel(const float* __restrict__ sums, const float* __restrict__ scale, long long M, int K, void* dx,
                                                         int type, long long dx_stride) {
    pdl_wait();
    const long long m = blockIdx.x;
    const float s = __ldg(scale + m);
    const float *hi = sums + m * K, *lo = hi + M * K;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = blockIdx.y * 1024 + i * 256 + threadIdx.x;
        if (k < K) store_y(dx, type, m * dx_stride + k, fmaf(hi[k], PART, lo[k]) * s);
    }
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Strides and alignment of rows of n values of `type`.
bool rows_fit(const void* p, int type, int64_t M, int64_t n, int64_t stride) {
    return p && aligned(p, ftype_bytes(type)) && (M <= 1 || stride >= n);
}

// How a product of rows as fp16 is done, by its sizes: few rows to a tile, or pairs of CTAs, a tile's reduction in `shares` and its sums
// through memory where that takes less time.
struct Plan {
    bool few;
    ManyPlan many;
    size_t bytes;  // of the sums
};
// Microseconds, measured on products of 300 to 8192 rows (512 x 512 of 25088 in 8 shares 34 us, in one 92, few rows to a tile 38; 1500 x 1024
// of 8192 in three 38, in one 51, few rows 41; 2000 x 4097 of 2048, GELU and residual, the sums through memory 60, stored by the pairs 88).
// epilogue: what the pairs take to finish and store a tile of 256 tokens, under the next tile's products or not.
Plan find_plan(int64_t M, int32_t N, int32_t K, double epilogue) {
    Plan best = {true, {0, 0, 1, nullptr}, 0};
    const double pairs = many_pairs(), blocks = (K + LS_KB - 1) / LS_KB, tn = (N + 255) / 256;
    const double few_tiles = (double)((N + 127) / 128) * ((M + 127) / 128);
    int few_shares = 1;
    while (few_shares < 8 && few_tiles * few_shares <= pairs && blocks >= 16 * few_shares) few_shares *= 2;
    double least = std::ceil(few_tiles * few_shares / (2 * pairs)) * (7.0 + std::ceil(blocks / few_shares) * 0.5);
    if ((N + 127) / 128 > 65535 || (M + 127) / 128 > 65535) least = 1e30;  // (its grid)
    for (int nt = 128; nt <= 256; nt += 128) {
        const int64_t tiles = (int64_t)tn * ((M + nt - 1) / nt), full = tiles / (int64_t)pairs * (int64_t)pairs;
        if (tiles > INT32_MAX / 16) continue;
        const double narrow = nt / 256.0, block = nt == 256 ? 0.54 : 0.36, round = std::max(blocks * block, epilogue * narrow) + 1.5;
        for (int whole = 0; whole < 3; ++whole)  // no tile, the full rounds' or all
            for (int shares = 1; shares <= 12 && 4 * shares <= blocks + 3; ++shares) {
                if (whole == 1 && (full == 0 || full == tiles || shares == 1)) continue;
                if (whole == 2 && shares > 1) continue;
                const int64_t own = whole == 2 ? tiles : whole == 1 ? full : 0, split = tiles - own;
                const double sums = (double)split * nt * 1024.0 * shares;  // (bytes)
                if (sums > 1073741824.0) continue;
                double time = 6.0 + std::ceil(own / pairs) * round;
                if (split) time += std::ceil(split * shares / pairs) * (std::ceil(blocks / shares) * block + 3.0) + 4.0 + sums / 2.6e6;
                if (!split) time += epilogue * narrow;
                if (time < least) least = time, best = {false, {nt, (int)own, shares, nullptr}, (size_t)sums};
            }
    }
    return best;
}
// (A call asks twice, for the workspace and for the run, and its like follow: the last ones are kept, 3 us otherwise.)
Plan plan_of(int64_t M, int32_t N, int32_t K, double epilogue) {
    if (M <= 64 || N < 128 || K < 128) return {true, {0, 0, 1, nullptr}, 0};
    struct Entry {
        int64_t M;
        int32_t N, K;
        double epilogue;
        Plan plan;
    };
    static thread_local Entry last[16];
    Entry& e = last[((uint32_t)M * 31u + (uint32_t)N * 7u + (uint32_t)K) % 16];
    if (e.M != M || e.N != N || e.K != K || e.epilogue != epilogue) e = {M, N, K, epilogue, find_plan(M, N, K, epilogue)};
    return e.plan;
}
// Outputs of 16 bits in pairs are stored fast; others, and above all their residuals, value by value.
double epilogue_time(int32_t N, int32_t y_type, int gated, bool residual) {
    return y_type != FXPQ_FT_F32 && N % (gated ? 4 : 2) == 0 ? 4.0 : residual ? 22.0 : 9.0;
}

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
fxpq_status product(const Product& p, const Epi& e, Plan plan, float* part, cudaStream_t st) {
    const int64_t pitch = (int64_t)half_pitch(p.K);
    if constexpr (EPI != PARTS)
        if (plan.few) return few_product<EPI>(p.rows, pitch, p.scale, p.w, p.w_stride, p.sw, p.bias, p.M, p.N, p.K, p.y_type, p.y, p.y_stride, st, e, nullptr, true);
    plan.many.part = plan.bytes ? part : nullptr;
    ManyArgs args;
    const fxpq_status rc = product_many<EPI>(p.rows, (size_t)pitch, p.scale, p.w, p.w_stride, p.sw, p.bias, p.M, p.N, p.K, p.y_type, p.y, p.y_stride, st, e,
                                             &plan.many, &args);
    if (rc != FXPQ_OK || !plan.bytes) return rc;
    args.e.vec = fours<EPI>(e, p.y_type, p.y, p.y_stride);
    launch_pdl(finish_kernel<EPI>, dim3(2 * (unsigned)(args.n_tiles - args.whole), plan.many.nt / (EPI == PARTS ? 64 : 32)), dim3(256), 0, st, args, plan.many.nt);
    return after_launch("finish");
}
struct LayerSpace {
    Plan plan;
    size_t codes, sums, end;
    explicit LayerSpace(const fxpq_layer& d) {
        codes = sums = end = 0;
        if (float_rows_fit(d.M, d.K)) return;
        plan = plan_of(d.M, d.N, d.K, epilogue_time(d.N, d.y_type, d.gated, d.d_residual));
        codes = up256((size_t)d.M * half_pitch(d.K) * 2);
        sums = codes + up256((size_t)d.M * 4);
        end = sums + up256(plan.bytes);
    }
};
bool sizes_ok(int64_t M, int32_t N, int32_t K) { return M >= 0 && N >= 0 && K >= 0 && M <= INT32_MAX; }

struct GradSpace {
    Plan plan;
    size_t rows, parts, sums, end;
    explicit GradSpace(const fxpq_layer_grad& d) {
        // Two parts of every row; the product of few rows leaves their sums to join_parts_kernel, pairs of CTAs join them (half as many to store a tile).
        plan = plan_of(2 * d.M, d.K, d.N, epilogue_time(d.K, d.dx_type, 0, false) / 2);
        rows = up256((size_t)2 * d.M * half_pitch(d.N) * 2);
        parts = rows + up256((size_t)d.M * 4);
        sums = parts + (plan.few ? up256((size_t)2 * d.M * d.K * 4) : 0);
        end = sums + up256(plan.bytes);
    }
};

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
    // The product of few rows is let in while the quantizer runs, for rows past 8192 as its blocks (of 512 threads and more) end: placed around
    // them earlier, clusters of 8 took a second round (17 x 4096 of 16384 26.8 us, so 18.5; without 19.2).
    const RowNorm norm = {d.d_norm, d.eps, aligned(d.d_norm, 16), !at.end || !at.plan.few ? 0 : d.K > 8192 ? 2 : 1};
    const Epi e = {d.d_residual, d.residual_stride, d.d_pre, 1.0f / (float)(1LL << sum_shift(d.K)), d.pre_type == FXPQ_FT_F32, d.activation, pre_pitch(d.N)};
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
    float* part = reinterpret_cast<float*>(ws + at.sums);
    return d.gated ? product<GATED>(p, e, at.plan, part, st) : product<LAYER>(p, e, at.plan, part, st);
}

extern "C" size_t fxpq_layer_gradient_workspace(const fxpq_layer_grad* d) {
    if (!d || !sizes_ok(d->M, d->N, d->K) || d->M == 0 || d->K == 0 || d->M > INT32_MAX / 2) return 0;
    return GradSpace(*d).end;
}

extern "C" fxpq_status fxpq_layer_gradient(const fxpq_layer_grad* grad, void* d_ws, size_t ws_bytes, void* stream) {
    if (!grad) return FXPQ_ERR_INVALID_ARG;
    const fxpq_layer_grad& d = *grad;
    if (!sizes_ok(d.M, d.N, d.K) || d.M > INT32_MAX / 2 || d.K > 65535 * 1024 || !ftype_ok(d.y_type) || !ftype_ok(d.dx_type) || !act_ok(d.activation) || d.gated < 0 ||
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
    // (sums rounded to 16 bits may lie on the other side of the step than the forward pass's z: gradients where y is 0)
    if (d.N > 0 && d.activation == FXPQ_ACT_RELU && d.pre_type == FXPQ_FT_F16) return FXPQ_ERR_INVALID_ARG;
    const GradSpace at(d);
    if (!d_ws || ws_bytes < at.end || !aligned(d_ws, 256)) return FXPQ_ERR_WORKSPACE;
    char* ws = static_cast<char*>(d_ws);
    cudaStream_t st = as_stream(stream);
    __half* rows = reinterpret_cast<__half*>(ws);
    float* scale = reinterpret_cast<float*>(ws + at.rows);
    float *sums = reinterpret_cast<float*>(ws + at.parts), *part = reinterpret_cast<float*>(ws + at.sums);
    const int dyb = ftype_bytes(d.y_type), some = d.gated ? 4 * dyb : 16;
    const int vec = (aligned(d.d_dy, some < 16 ? some : 16) && d.dy_stride * dyb % (some < 16 ? some : 16) == 0 ? 1 : 0) |
                    (aligned(d.d_pre, 16) ? 2 : 0) | (aligned(d.d_sw, 16) ? 4 : 0) | (aligned(d.d_bias, 16) ? 8 : 0);
    const int act = d.N > 0 ? d.activation : FXPQ_ACT_NONE;  // (rows of nothing read nothing)
    const GradRows G = {d.d_dy, d.dy_stride, d.d_pre, d.d_sx, d.d_sw, d.d_bias, (float)(1LL << sum_shift(d.K)), d.pre_type == FXPQ_FT_F32,
                        act, d.N, at.plan.few, vec, rows, (long long)half_pitch(d.N), (long long)d.M, scale,
                        status_ptr()};
    fxpq_status rc = grad_rows(G, d.y_type, d.N > 0 && d.gated, st);
    if (rc != FXPQ_OK) return rc;
    if (!at.plan.few) return product<PARTS>({rows, scale, d.d_wt, d.wt_stride, nullptr, nullptr, d.M, d.K, d.N, d.dx_type, d.d_dx, d.dx_stride}, {}, at.plan, part, st);
    const int64_t pitch = (int64_t)half_pitch(d.N), at_once = 2 * d.M <= 65535 * 128 ? 2 * d.M : d.M;  // (its grid)
    for (int64_t m = 0; m < 2 * d.M; m += at_once) {
        rc = few_product<LAYER>(rows + m * pitch, pitch, nullptr, d.d_wt, d.wt_stride, nullptr, nullptr, at_once, d.K, d.N, FXPQ_FT_F32, sums + m * d.K, d.K, st, {},
                                nullptr, m == 0);
        if (rc != FXPQ_OK) return rc;
    }
    launch_pdl(join_parts_kernel, dim3((unsigned)d.M, (unsigned)((d.K + 1023) / 1024)), dim3(256), 0, st, static_cast<const float*>(sums),
               static_cast<const float*>(scale), (long long)d.M, (int)d.K, d.d_dx, (int)d.dx_type, (long long)d.dx_stride);
    return after_launch("layer_join_parts");
}
