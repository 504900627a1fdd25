// fxpq_layer_grad.cu -- the rows dz * sw of a layer's gradient, which a product with the transposed weights turns into dx.
#include <type_traits>

#include "fxpq_layer.cuh"

namespace fxpq {
namespace llm {
namespace {

__device__ __forceinline__ float one_any(const void* p, int type, long long at) {
    return type == FXPQ_FT_F32 ? static_cast<const float*>(p)[at]
                               : type == FXPQ_FT_F16 ? to_f32(static_cast<const __half*>(p)[at]) : to_f32(static_cast<const __nv_bfloat16*>(p)[at]);
}

// N values as they lie in memory (vec: aligned, 8 to 32 bytes), and as fp32.
template <int N, int BYTES>
struct Words {
    uint32_t w[N * BYTES / 4];
    __device__ __forceinline__ void load(const void* p, long long at, bool vec = true) {
        const char* q = static_cast<const char*>(p) + at * BYTES;
        if (!vec) {
#pragma unroll
            for (int i = 0; i < N * BYTES / 4; ++i) {
                if constexpr (BYTES == 4)
                    w[i] = reinterpret_cast<const uint32_t*>(q)[i];
                else
                    w[i] = __byte_perm(reinterpret_cast<const unsigned short*>(q)[2 * i], reinterpret_cast<const unsigned short*>(q)[2 * i + 1], 0x5410);
            }
            return;
        }
        if constexpr (N * BYTES == 8) {
            const uint2 v = *reinterpret_cast<const uint2*>(q);
            w[0] = v.x, w[1] = v.y;
        } else {
#pragma unroll
            for (int i = 0; i < N * BYTES / 16; ++i) {
                const uint4 v = reinterpret_cast<const uint4*>(q)[i];
                w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ void values(bool f16, float (&v)[N]) const {
#pragma unroll
        for (int i = 0; i < N * BYTES / 4; ++i) {
            if constexpr (BYTES == 4) {
                v[i] = __uint_as_float(w[i]);
            } else {
                const float2 f = f16 ? __half22float2(*reinterpret_cast<const __half2*>(&w[i])) : __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
                v[2 * i] = f.x, v[2 * i + 1] = f.y;
            }
        }
    }
};

// One block a row, as two rows of fp16 with a power of two of the row's own: v up to 2^23, h = v / 2^12 rounded to an integer (up to 2^11: exact in
// fp16, as are its products' sums below 2^24), and what h leaves of v (up to 2^11, to 2^-12 of itself), M rows further on.  So a value
// loses 2^-23 of the row's largest at most, or 2^-12 of its own size where that is less.  (In one part of 11 bits gradients of 16 bits came
// out 3e-4 to 1e-3 from those of 32-bit products, in their last places.)
// Bytes bound it (dy and the sums in, both parts out): 8192 rows of 2 x 5632 830 MB, 125 us, 6.6 TB/s.  Rows stay in registers between their maximum
// and the rounding, GR_KEEP groups of eight channels a thread, which are also on their way together; what does not fit, the last
// group of some, and all of constants or sums that are not aligned, is formed again.  (A group at a time, kept in shared memory, the rows took
// twice as long.)  ALL: every group is kept; with the code for the others, and what it holds of registers, those rows took 158 us.
constexpr int GR_KEEP = 3;
template <bool GATE, int ACT, int DY, int PRE, int GR_THREADS, bool ALL>
__global__ void __launch_bounds__(GR_THREADS, 1024 / GR_THREADS) grad_rows_kernel(const __grid_constant__ GradRows G, int y_type) {
    pdl_wait();
    constexpr bool NEEDS = GATE || ACT != FXPQ_ACT_NONE;
    constexpr int D = GATE ? 4 : 8;  // values of dy to eight channels
    const long long m = blockIdx.x;
    const int t = threadIdx.x, N = G.N, groups = (N + 7) / 8, pre_type = PRE == 4 ? FXPQ_FT_F32 : FXPQ_FT_F16;
    const float sx = NEEDS ? __ldg(G.sx + m) : 0.0f;
    const long long pitch = pre_pitch(N);
    auto compute = [&](const float (&d)[D], float (&a)[8], const float (&w)[8], const float (&b)[8], float (&v)[8]) {
        if constexpr (NEEDS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float sum = PRE == 4 ? a[e] : a[e] * G.pre_unit;  // (a power of two; its product with sx instead can pass fp32 where z does not)
                a[e] = fmaf(sum * sx, w[e], G.bias ? b[e] : 0.0f);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e += GATE ? 2 : 1) {
            if constexpr (GATE) {
                float slope;
                const float f = activate_slope(a[e], ACT, slope);
                v[e] = d[e / 2] * a[e + 1] * slope * w[e], v[e + 1] = d[e / 2] * f * w[e + 1];
            } else if constexpr (NEEDS) {
                float slope;
                activate_slope(a[e], ACT, slope);
                v[e] = d[e] * slope * w[e];
            } else {
                v[e] = d[e] * w[e];
            }
        }
    };
    auto form = [&](int g, float (&v)[8]) {  // value by value
        const int n = 8 * g, left = min(N - n, 8);
        float d[D], a[8], w[8], b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool in = e < left;
            if (e < D) d[e] = (GATE ? 2 * e : e) < left ? one_any(G.dy, y_type, m * G.dy_stride + g * D + e) : 0.0f;
            w[e] = in ? __ldg(G.sw + n + e) : 0.0f;
            a[e] = NEEDS && in ? one_any(G.pre, pre_type, m * pitch + n + e) : 0.0f;
            b[e] = NEEDS && G.bias && in ? __ldg(G.bias + n + e) : 0.0f;
        }
        compute(d, a, w, b, v);
    };
    uint32_t top = 0;
    auto see = [&](const float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    };
    const int whole = ALL ? groups : (G.vec | 1 | (NEEDS ? 0 : 2) | (G.bias ? 0 : 8)) == 15 ? N / 8 : 0;  // groups whose constants and sums come in aligned accesses
    const auto of_words = [&](int g, const Words<D, DY>& d, const Words<8, PRE>& a, float (&v)[8]) {
        float df[D], af[8], w[8], b[8];
        load_f32<8>(G.sw + 8 * g, true, w);
        if (NEEDS && G.bias) load_f32<8>(G.bias + 8 * g, true, b);
        d.values(y_type == FXPQ_FT_F16, df);
        a.values(true, af);
        compute(df, af, w, b, v);
    };
    const auto again = [&](int g, float (&v)[8]) {  // a group that is not kept
        if (g >= whole) return form(g, v);
        Words<D, DY> d;
        Words<8, PRE> a;
        d.load(G.dy, m * G.dy_stride + g * D, G.vec & 1);
        if constexpr (NEEDS) a.load(G.pre, m * pitch + 8 * g);
        of_words(g, d, a, v);
    };
    float keep[GR_KEEP][8];
    {
        Words<D, DY> d[GR_KEEP];
        Words<8, PRE> a[GR_KEEP];
#pragma unroll
        for (int s = 0; s < GR_KEEP; ++s) {
            const int g = t + s * GR_THREADS;
            if (g >= whole) continue;
            d[s].load(G.dy, m * G.dy_stride + g * D, G.vec & 1);
            if constexpr (NEEDS) a[s].load(G.pre, m * pitch + 8 * g);
        }
#pragma unroll
        for (int s = 0; s < GR_KEEP; ++s) {
            const int g = t + s * GR_THREADS;
            if (g >= whole) continue;
            of_words(g, d[s], a[s], keep[s]);
            see(keep[s]);
        }
    }
    const int first = ALL ? groups : min(whole, GR_KEEP * GR_THREADS);  // of those that are not kept
    if constexpr (!ALL) {
#pragma unroll 1
        for (int g = first + t; g < groups; g += GR_THREADS) {
            float v[8];
            again(g, v);
            see(v);
        }
    }
    __shared__ uint32_t part[GR_THREADS / 32];
    top = __reduce_max_sync(0xffffffffu, top);
    if ((t & 31) == 0) part[t >> 5] = top;
    __syncthreads();
    top = 0;
#pragma unroll
    for (int w = 0; w < GR_THREADS / 32; ++w) top = max(top, part[w]);
    if (G.early) pdl_next();
    const bool bad = top >= 0x7f800000u;
    // top < 2^e; the row's largest value lies in [2^22, 2^23)
    const int e = max(top ? ilogbf(__uint_as_float(top)) + 1 : 0, -100), up = 23;
    const float lift = ldexpf(1.0f, up - e);
    if (t == 0) {
        G.scale[m] = bad ? __int_as_float(0x7fffffff) : ldexpf(1.0f, e - up);
        if (bad) latch_status(G.status, FXPQ_ERR_NONFINITE);
    }
    uint4* hi = reinterpret_cast<uint4*>(G.rows + m * G.pitch);
    uint4* lo = reinterpret_cast<uint4*>(G.rows + (G.M + m) * G.pitch);
    auto put = [&](int g, const float (&v)[8]) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = bad ? 0.0f : v[2 * i] * lift, b = bad ? 0.0f : v[2 * i + 1] * lift;
            const float ha = rintf(a * (1.0f / PART)), hb = rintf(b * (1.0f / PART));
            h[i] = h2_bits(__floats2half2_rn(ha, hb));
            l[i] = h2_bits(__floats2half2_rn(fmaf(ha, -PART, a), fmaf(hb, -PART, b)));
        }
        hi[g] = make_uint4(h[0], h[1], h[2], h[3]);
        lo[g] = make_uint4(l[0], l[1], l[2], l[3]);
    };
#pragma unroll
    for (int s = 0; s < GR_KEEP; ++s)
        if (t + s * GR_THREADS < whole) put(t + s * GR_THREADS, keep[s]);
    if constexpr (!ALL) {
#pragma unroll 1
        for (int g = first + t; g < groups; g += GR_THREADS) {
            float v[8];
            again(g, v);
            put(g, v);
        }
    }
    if (t == 0 && (groups & 1)) {  // rows are padded to 16
        hi[groups] = make_uint4(0, 0, 0, 0);
        lo[groups] = make_uint4(0, 0, 0, 0);
    }
}

}  // namespace

fxpq_status grad_rows(const GradRows& G, int y_type, int gated, cudaStream_t st) {
    auto go = [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        const auto sized = [&](auto gate) {
            constexpr bool GATE = decltype(gate)::value;
            const auto run = [&](auto dy, auto pre) {
                constexpr int DY = decltype(dy)::value, PRE = decltype(pre)::value;
                constexpr bool NEEDS = GATE || ACT != FXPQ_ACT_NONE;
                const bool fits = DY == 2 && G.N % 8 == 0 && G.N <= 8 * GR_KEEP * 1024 &&
                                  (G.vec | 1 | (NEEDS ? 0 : 2) | (G.bias ? 0 : 8)) == 15;
                const auto go = [&](auto threads) {
                    constexpr int THREADS = decltype(threads)::value;
                    const auto with = [&](auto kernel) { launch_pdl(kernel, dim3((unsigned)G.M), dim3(THREADS), 0, st, G, y_type); };
                    if constexpr (DY == 2)
                        if (fits) return with(grad_rows_kernel<GATE, ACT, DY, PRE, THREADS, true>);
                    if constexpr (THREADS <= 512) with(grad_rows_kernel<GATE, ACT, DY, PRE, THREADS, false>);
                };
                // As many threads as the row's groups need, so that more rows are under way (3990 rows of 549 channels in fp32: 12 us), or all
                // there are where that keeps the row (7999 rows of 22400: 293 us, with 512 and the rest formed again a tenth more).
                if (G.N <= 8 * GR_KEEP * 128)
                    go(std::integral_constant<int, 128>());
                else if (G.N <= 8 * GR_KEEP * 256)
                    go(std::integral_constant<int, 256>());
                else if (G.N <= 8 * GR_KEEP * 512 || !fits)
                    go(std::integral_constant<int, 512>());
                else
                    go(std::integral_constant<int, 1024>());
            };
            using Two = std::integral_constant<int, 2>;
            using Four = std::integral_constant<int, 4>;
            const auto kept = [&](auto dy) {
                if constexpr (GATE || ACT != FXPQ_ACT_NONE)  // (else none are read)
                    if (G.pre_f32) return run(dy, Four());
                run(dy, Two());
            };
            y_type == FXPQ_FT_F32 ? kept(Four()) : kept(Two());
        };
        if (!gated) return sized(std::false_type());
        if constexpr (ACT != FXPQ_ACT_NONE) sized(std::true_type());
    };
    switch (G.act) {
        case FXPQ_ACT_RELU: go(std::integral_constant<int, FXPQ_ACT_RELU>()); break;
        case FXPQ_ACT_SILU: go(std::integral_constant<int, FXPQ_ACT_SILU>()); break;
        case FXPQ_ACT_GELU: go(std::integral_constant<int, FXPQ_ACT_GELU>()); break;
        case FXPQ_ACT_GELU_TANH: go(std::integral_constant<int, FXPQ_ACT_GELU_TANH>()); break;
        default: go(std::integral_constant<int, FXPQ_ACT_NONE>());
    }
    return after_launch("layer_grad_rows");
}

}  // namespace llm
}  // namespace fxpq
