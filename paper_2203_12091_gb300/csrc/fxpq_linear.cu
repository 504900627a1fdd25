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
    if (norm.early == 1) pdl_next();
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
        __shared__ float sums[QT_THREADS / 32], row_inv;
        float wt[8];
        auto weights = [&](int g) { load_f32<8>(norm.weight + 8 * g, norm.vec, wt); };
        RowScan<true> scan;
        each([&](int g, const Raw8<T>& v) {
            weights(g);
#pragma unroll
            for (int e = 0; e < 8; ++e) scan.see(to_f32(v.v[e]), wt[e]);
        });
        if (tail < K) scan.see(to_f32(row[tail]), __ldg(norm.weight + tail));
        scan.meet();
        if ((t & 31) == 0) part[t >> 5] = scan.top, sums[t >> 5] = scan.sum;
        __syncthreads();
        if (t < 32) {
            scan = RowScan<true>();
            if (t < QT_THREADS / 32) scan.join(part[t], sums[t]);
            scan.meet();
            float inv = scan.inverse(), sx;
            if (scan.odd())
                careful_row(row, K, norm.weight, norm.eps, inv, sx, status);
            else
                sx = scan.scale(K, norm.eps);
            if (t == 0) row_inv = inv, scale[blockIdx.x] = sx;
        }
        __syncthreads();
        if (norm.early == 2) pdl_next();
        const float inv = row_inv;
        each([&](int g, const Raw8<T>& v) {
            weights(g);
            float c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = scaled_code(__fmul_rn(to_f32(v.v[e]), wt[e]), inv);
            *reinterpret_cast<uint4*>(out + 8 * g) =
                make_uint4(f32_codes_f16x2(c[0], c[1]), f32_codes_f16x2(c[2], c[3]), f32_codes_f16x2(c[4], c[5]), f32_codes_f16x2(c[6], c[7]));
        });
        if (tail < K) out[tail] = (C)(int)rintf(scaled_code(__fmul_rn(to_f32(row[tail]), __ldg(norm.weight + tail)), inv));
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
    if (norm.early == 2) pdl_next();
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

struct LinArgs {
    // weights' codes as [N][K] bytes in boxes of 128 codes x 128 rows (tw), or x the rows that the last tile has (tw2: a box is
    // slow where it lies outside the tensor); tokens' as [M][K] bytes in boxes of 128 x `rows`, or as fp16 in 64 x `rows`
    CUtensorMap tw, tw2, tx;
    const float *sx, *sw, *bias;
    void* y;
    long long ys, M;
    int N, y_type, n_kb;
    int rows, cols;  // tokens of a tile, and rounded up to 16, at most 128 (the columns past `rows` hold whatever the stage does)
    int w_rows;      // channels of the last tile
    int y_four;      // four outputs of a row in one aligned access
    int stages;
    int* status;
};

// ------------------------------------------------------------------ few tokens
// y^T = w x^T on tcgen05 (kind::f16: the 8-bit kind does not exist on sm_103a; codes are exact in fp16, their products in fp32): 128
// output channels on the accumulator's lanes, up to 128 tokens on its columns.  The weights are the traffic.  They
// arrive as codes (TMA, 128 x 128 bytes a block) and go through registers into tensor memory as the fp16 A operand,
// so that their shared-memory traffic stays at two bytes a code.  The tokens' rows come as fp16 codes (HALF: written so by the
// quantizer) or as bytes that are expanded in shared memory.
//   warp 0   copies;   warp 1   tensor memory, products;   warps 4-7, 8-11   converters (blocks in turn), then the epilogue.
// The reduction is shared by the CTAs of a cluster, whose fp32 sums meet through distributed shared memory: one launch, a
// fixed order.  Up to 64 tokens two CTAs fit an SM.
constexpr int LS_THREADS = 384;

__host__ __device__ inline int ls_smem(int cols, int stages, bool half) {  // stages, with bytes two expanded token stages
    const int ring = half ? stages * (LS_A + cols * LS_KB * 2) : stages * (LS_A + cols * LS_KB) + 2 * cols * LS_KB * 2, sums = cols * 128 * 4;
    return 1024 + (ring > sums ? ring : sums);
}

template <bool HALF>
__global__ void __launch_bounds__(LS_THREADS) linear_few_kernel(const __grid_constant__ LinArgs P) {
    using namespace tc;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    __shared__ __align__(8) uint64_t bars[8 + 2 + 2 + 1 + 8];
    __shared__ int abort_flag;
    __shared__ uint32_t tmem_slot;
    volatile int* abort = &abort_flag;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, ST = P.stages, cols = P.cols;
    const uint32_t raw_full = smem_u32(bars), raw_empty = raw_full + 8 * 8, conv_full = raw_empty + 8 * 8, conv_empty = conv_full + 16,
                   done = conv_empty + 16;
    const int raw_bytes = LS_A + cols * LS_KB * (HALF ? 2 : 1);
    const uint32_t raw0 = smem_u32(smem), conv0 = raw0 + ST * raw_bytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(raw_full + 8 * i, 1);
            mbar_init(raw_empty + 8 * i, HALF ? 1 : 4);  // the products' completion, or the converting group's warps
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(conv_full + 8 * i, 4);
            mbar_init(conv_empty + 8 * i, 1);
        }
        mbar_init(done, 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (P.n_kb) {
            prefetch_tmap(blockIdx.y == gridDim.y - 1 ? &P.tw2 : &P.tw);
            prefetch_tmap(&P.tx);
        }
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(256u));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmem_a = tmem + 128;
    const int rank = blockIdx.x, shares = gridDim.x, n0 = blockIdx.y * 128;
    const long long m0 = (long long)blockIdx.z * P.rows;
    const int kb0 = (int)((long long)P.n_kb * rank / shares), n_kb = (int)((long long)P.n_kb * (rank + 1) / shares) - kb0;

    if (warp == 0) {
        int i = 0;
        const bool last = blockIdx.y == gridDim.y - 1;
        const CUtensorMap* tw = last ? &P.tw2 : &P.tw;
        const uint32_t bytes = (uint32_t)((last ? P.w_rows : 128) * LS_KB + P.rows * LS_KB * (HALF ? 2 : 1));
        for (; i < n_kb; ++i) {
            const int s = i % ST;
            if (!wait_warp(raw_empty + 8 * s, ((i / ST) & 1) ^ 1, abort, P.status)) break;
            const uint32_t bar = raw_full + 8 * s, dst = raw0 + s * raw_bytes;
            mbar_arrive_expect_tx(bar, bytes);
            tma_load_2d(dst, tw, (kb0 + i) * LS_KB, n0, bar);
            tma_load_2d(dst + LS_A, &P.tx, (kb0 + i) * LS_KB, (int)m0, bar);
            if (HALF) tma_load_2d(dst + LS_A + cols * 128, &P.tx, (kb0 + i) * LS_KB + 64, (int)m0, bar);
        }
        for (int j = max(0, i - ST); j < i; ++j) {  // every copy has landed before this CTA's memory is used again
            drain_warp(raw_full + 8 * (j % ST), (j / ST) & 1);
        }
    } else if (warp == 1) {
        const uint32_t idesc = make_idesc(128, cols);
        const uint64_t bdesc = make_sdesc(HALF ? raw0 : conv0);
        for (int i = 0; i < n_kb; ++i) {
            const int c = i & 1, s = i % ST;
            if (!wait_warp(conv_full + 8 * c, (i >> 1) & 1, abort, P.status)) break;
            if (HALF && !wait_warp(raw_full + 8 * s, (i / ST) & 1, abort, P.status)) break;
            tc_fence_after();
            const uint64_t bd = bdesc + (uint64_t)((HALF ? s * raw_bytes + LS_A : c * cols * 256) >> 4);
#pragma unroll
            for (int kk = 0; kk < LS_KB / 16; ++kk)
                tc_mma_ta(tmem, tmem_a + 64 * c + 8 * kk, bd + (uint64_t)(((kk >> 2) * cols * 128) >> 4) + 2 * (kk & 3), idesc, i > 0 || kk > 0);
            tc_commit(conv_empty + 8 * c);
            if (HALF) tc_commit(raw_empty + 8 * s);
        }
        tc_commit(done);
        drain_warp(done, 0);
    } else if (warp >= 4) {
        const int grp = (warp - 4) >> 2, quad = warp & 3, t = threadIdx.x & 127, row = quad * 32 + lane;
        for (int i = grp; i < n_kb; i += 2) {
            const int s = i % ST;
            // In this order: with an odd number of stages the groups take turns on one, and a parity wait on raw_full
            // tells block i from block i - ST of the other group only once that one has landed.  Block i - 2's products
            // are complete here, so all before them are, and their blocks were read.
            if (!wait_warp(conv_empty + 8 * grp, ((i >> 1) & 1) ^ 1, abort, P.status)) break;
            if (!wait_warp(raw_full + 8 * s, (i / ST) & 1, abort, P.status)) break;
            tc_fence_after();
            const unsigned char* ra = smem + s * raw_bytes;
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {  // 64 codes of this thread's channel
                uint32_t r[32];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint4 v = *reinterpret_cast<const uint4*>(ra + row * 128 + (((4 * hf + q) ^ (row & 7)) << 4));
                    const uint32_t w[4] = {v.x ^ 0x80808080u, v.y ^ 0x80808080u, v.z ^ 0x80808080u, v.w ^ 0x80808080u};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        r[8 * q + 2 * e] = code_pair(w[e], LOW_PAIR);
                        r[8 * q + 2 * e + 1] = code_pair(w[e], HIGH_PAIR);
                    }
                }
                tmem_st32_nw(tmem_a + ((uint32_t)(quad * 32) << 16) + 64 * grp + 32 * hf, r);
            }
            if constexpr (!HALF) {
                const unsigned char* rb = ra + LS_A;
                unsigned char* cb = smem + ST * raw_bytes + grp * cols * 256;
                for (int rr = t >> 3; rr < cols; rr += 16) {  // 16 codes of one token
                    const int c = t & 7, hf = c >> 2;
                    const uint4 v = *reinterpret_cast<const uint4*>(rb + rr * 128 + ((c ^ (rr & 7)) << 4));
                    uint4 o[2];
                    uint32_t x = v.x ^ 0x80808080u, y = v.y ^ 0x80808080u;
                    o[0] = make_uint4(code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR));
                    x = v.z ^ 0x80808080u, y = v.w ^ 0x80808080u;
                    o[1] = make_uint4(code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR));
                    unsigned char* dst = cb + hf * cols * 128 + rr * 128;
                    const int j = 2 * (c & 3);
                    // (the second half's lanes begin with their odd chunk, else the two halves meet in the banks)
                    *reinterpret_cast<uint4*>(dst + (((j + hf) ^ (rr & 7)) << 4)) = hf ? o[1] : o[0];
                    *reinterpret_cast<uint4*>(dst + (((j + 1 - hf) ^ (rr & 7)) << 4)) = hf ? o[0] : o[1];
                }
                fence_proxy_async();
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (!HALF) mbar_arrive(raw_empty + 8 * s);
                mbar_arrive(conv_full + 8 * grp);
            }
        }
        // ---- this CTA's sums to shared memory: [token][128 channels]
        float* sums = reinterpret_cast<float*>(smem);
        if (n_kb > 0) wait_warp(done, 0, abort, P.status);
        tc_fence_after();
        for (int c = 16 * grp; c < cols; c += 32) {
            uint32_t v[16];
            tmem_ld16_nw(tmem + ((uint32_t)(quad * 32) << 16) + c, v);
            tmem_wait_ld();
            reg_fence(v);
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[(c + e) * 128 + row] = n_kb > 0 ? __uint_as_float(v[e]) : 0.0f;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256u));
    }
    // ---- four channels of one token per lane, a token per warp and step, summed over the cluster
    const int mine = (int)min((long long)P.rows, P.M - m0), c_lo = mine * rank / shares, c_hi = mine * (rank + 1) / shares;
    const int ch = n0 + 4 * lane;
    constexpr int TOKENS = LS_THREADS / 32;
    float sw[4], bias[4], sx = c_lo + warp < c_hi ? __ldg(P.sx + m0 + c_lo + warp) : 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // (on their way while the CTAs meet)
        sw[e] = ch + e < P.N ? __ldg(P.sw + ch + e) : 0.0f;
        bias[e] = P.bias && ch + e < P.N ? __ldg(P.bias + ch + e) : 0.0f;
    }
    if (shares > 1) cluster_sync();
    for (int c = c_lo + warp; c < c_hi; c += TOKENS) {
        const uint32_t at = raw0 + (uint32_t)(c * 32 + lane) * 16;
        float4 b[8], a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < shares) b[r] = ld_cluster_f4(cluster_addr(at, r));
        const float s = sx;
        if (c + TOKENS < c_hi) sx = __ldg(P.sx + m0 + c + TOKENS);
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < shares) a.x += b[r].x, a.y += b[r].y, a.z += b[r].z, a.w += b[r].w;
        const float v[4] = {fmaf(a.x * s, sw[0], bias[0]), fmaf(a.y * s, sw[1], bias[1]), fmaf(a.z * s, sw[2], bias[2]), fmaf(a.w * s, sw[3], bias[3])};
        const long long to = (m0 + c) * P.ys + ch;
        if (P.y_four && ch + 4 <= P.N) {
            if (P.y_type == FXPQ_FT_F32)
                store_f32<4>(static_cast<float*>(P.y) + to, v);
            else if (P.y_type == FXPQ_FT_F16)
                store_f32<4>(static_cast<__half*>(P.y) + to, v);
            else
                store_f32<4>(static_cast<__nv_bfloat16*>(P.y) + to, v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (ch + e < P.N) store_y(P.y, P.y_type, to + e, v[e]);
        }
    }
    if (shares > 1) cluster_sync();  // (the others have read this CTA's sums)
}


template <bool HALF>
fxpq_status launch_few(LinArgs& P, cudaStream_t st) {
    static std::atomic<uint64_t> set{0};
    if (!allow_smem(linear_few_kernel<HALF>, ls_smem(128, 4, HALF), set)) return FXPQ_ERR_CUDA;
    const long long tn = (P.N + 127) / 128, tm = (P.M + P.rows - 1) / P.rows;
    if (tn > 65535 || tm > 65535) return FXPQ_ERR_UNSUPPORTED;
    P.stages = P.cols <= 32 || P.cols > 64 ? 4 : 3;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.blockDim = dim3(LS_THREADS);
    c.dynamicSmemBytes = ls_smem(P.cols, P.stages, HALF);
    c.stream = st;
    c.attrs = at;
    // As many CTAs to a reduction as run at once, with at least 1024 codes each (4096 x 4096, 64 tokens: 10.9 us with four of
    // 1024 codes, 11.9 with eight of 512), or 512 where they leave half of the SMs free (1000 x 4096, one token: 5.5 and 6.8).  Clusters are placed within a group of SMs: 16 clusters of 8 CTAs that fill an SM
    // each left one for a second round (251 x 1001 of 4090: 19.4 us, 13.3 with clusters of 4).
    int shares = 1;
    for (; shares < 8 && P.n_kb >= (tn * tm * shares * 4 <= num_sms() ? 8 : 16) * shares; shares *= 2) {
        static std::atomic<int> room[9][4][DEVICES];  // by tile width and cluster size
        at[1].val.clusterDim.x = 2 * shares;
        c.gridDim = dim3(2 * shares, 1024, 1);
        c.numAttrs = 2;
        const int n = clusters_at_once(linear_few_kernel<HALF>, c, room[P.cols / 16][shares == 1 ? 1 : shares == 2 ? 2 : 3]);
        // (the query counts one CTA to an SM: it says 15 clusters of 8 where 32 of two CTAs to an SM ran at once)
        if (tn * tm > (P.cols <= 64 ? 2 * n + 2 : n)) break;
    }
    at[1].val.clusterDim.x = shares;
    c.gridDim = dim3((unsigned)shares, (unsigned)tn, (unsigned)tm);
    c.numAttrs = shares > 1 ? 2 : 1;
    (void)cudaLaunchKernelEx(&c, linear_few_kernel<HALF>, P);
    return after_launch("linear_few");
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
            else if (K > 16384 || (K > 8192 && M < 512))
                go(std::integral_constant<int, 1024>(), normed);
            else if (K > 8192)
                go(std::integral_constant<int, 512>(), normed);
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

// Codes of the tokens: bytes at d_x, or fp16 at half (one of them is null).
fxpq_status product_few(const int8_t* d_x, const __half* half, int64_t x_stride, const float* d_sx, const int8_t* d_w, int64_t w_stride,
                        const float* d_sw, const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type, void* d_y, int64_t y_stride,
                        cudaStream_t st) {
    LinArgs P;
    const int64_t tiles = (M + 127) / 128;  // M's equal parts
    P.rows = (int)((M + tiles - 1) / tiles);
    P.cols = (P.rows + 15) / 16 * 16;
    P.n_kb = (K + LS_KB - 1) / LS_KB;
    P.w_rows = N % 128 ? N % 128 : 128;
    P.y_four = aligned(d_y, 4 * ftype_bytes(y_type)) && y_stride % 4 == 0;
    if (K > 0) {
        if (!encode_rows(&P.tw, d_w, N, K, w_stride, 128) || !(half ? encode_half_rows(&P.tx, half, M, K, x_stride, P.rows) : encode_rows(&P.tx, d_x, M, K, x_stride, P.rows)))
            return FXPQ_ERR_CUDA;
        P.tw2 = P.tw;
        if (P.w_rows < 128 && !encode_rows(&P.tw2, d_w, N, K, w_stride, P.w_rows)) return FXPQ_ERR_CUDA;
    }
    P.sx = d_sx, P.sw = d_sw, P.bias = d_bias, P.y = d_y, P.ys = y_stride, P.M = M, P.N = N, P.y_type = y_type;
    P.status = status_ptr();
    return half ? launch_few<true>(P, st) : launch_few<false>(P, st);
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
    return product_few(d_x, nullptr, x_stride, d_sx, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, as_stream(stream));
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
    return product_few(nullptr, half, (int64_t)pitch, scale, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, st);
}

namespace fxpq {
namespace llm {
size_t half_pitch(int32_t K) { return codes_pitch(K); }
fxpq_status half_codes(const void* d_x, int32_t x_type, int64_t M, int32_t K, int64_t x_stride, __half* codes, float* scale, const RowNorm& norm,
                       cudaStream_t st) {
    return quantize_rows(d_x, x_type, M, K, x_stride, codes, (int64_t)codes_pitch(K), scale, st, norm);
}
}  // namespace llm
}  // namespace fxpq
