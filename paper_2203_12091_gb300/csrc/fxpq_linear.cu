// fxpq_linear.cu -- rows quantized to 8 bits with a scale each, and the product of 8-bit rows with scales for
// each token and each output channel.
#include <cfloat>

#include "fxpq_llm.cuh"
#include "fxpq_ptx.cuh"

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

__device__ __forceinline__ void store_y(void* y, int type, long long at, float v) {
    if (type == FXPQ_FT_F32)
        static_cast<float*>(y)[at] = v;
    else if (type == FXPQ_FT_F16)
        static_cast<__half*>(y)[at] = __float2half_rn(v);
    else
        static_cast<__nv_bfloat16*>(y)[at] = __float2bfloat16_rn(v);
}

struct LinArgs {
    CUtensorMap tw, tx;  // codes as [N][K], [M][K] bytes, boxes of 128 codes x 128 (tw) or `cols` (tx) rows
    const float *sx, *sw, *bias;
    void* y;
    long long ys, M;
    int N, y_type, n_kb;
    int cols;  // tokens of a tile: a multiple of 16, at most 128
    int stages;
    int* status;
};

// ------------------------------------------------------------------ few tokens
// y^T = w x^T on tcgen05 (kind::f16: the 8-bit kind does not exist on sm_103a; products of codes are exact in fp16): 128
// output channels on the accumulator's lanes, up to 128 tokens on its columns.  The weights are the traffic.  They
// arrive as codes (TMA, 128 x 128 bytes a block) and go through registers into tensor memory as the fp16 A operand,
// so that their shared-memory traffic stays at two bytes a code; the tokens' few rows are expanded in shared memory.
//   warp 0   copies;   warp 1   tensor memory, products;   warps 4-7, 8-11   converters (blocks in turn), then the epilogue.
// The reduction is shared by the CTAs of a cluster, whose fp32 sums meet through distributed shared memory: one launch, a
// fixed order.  Up to 64 tokens two CTAs fit an SM.
constexpr int LS_THREADS = 384, LS_KB = 128, LS_A = 128 * LS_KB;

__host__ __device__ inline int ls_smem(int cols, int stages) {  // raw stages, two expanded token stages
    const int ring = stages * (LS_A + cols * LS_KB) + 2 * cols * LS_KB * 2, sums = cols * 128 * 4;
    return 1024 + (ring > sums ? ring : sums);
}

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
    const int raw_bytes = LS_A + cols * LS_KB;
    const uint32_t raw0 = smem_u32(smem), conv0 = raw0 + ST * raw_bytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(raw_full + 8 * i, 1);
            mbar_init(raw_empty + 8 * i, 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(conv_full + 8 * i, 4);
            mbar_init(conv_empty + 8 * i, 1);
        }
        mbar_init(done, 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (P.n_kb) {
            prefetch_tmap(&P.tw);
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
    const long long m0 = (long long)blockIdx.z * cols;
    const int kb0 = (int)((long long)P.n_kb * rank / shares), n_kb = (int)((long long)P.n_kb * (rank + 1) / shares) - kb0;

    if (warp == 0) {
        int i = 0;
        for (; i < n_kb; ++i) {
            const int s = i % ST;
            if (!wait_warp(raw_empty + 8 * s, ((i / ST) & 1) ^ 1, abort, P.status)) break;
            const uint32_t bar = raw_full + 8 * s, dst = raw0 + s * raw_bytes;
            mbar_arrive_expect_tx(bar, (uint32_t)raw_bytes);
            tma_load_2d(dst, &P.tw, (kb0 + i) * LS_KB, n0, bar);
            tma_load_2d(dst + LS_A, &P.tx, (kb0 + i) * LS_KB, (int)m0, bar);
        }
        for (int j = max(0, i - ST); j < i; ++j) {  // every copy has landed before this CTA's memory is used again
            const long long t0 = clock64();
            while (!mbar_try_wait(raw_full + 8 * (j % ST), (j / ST) & 1) && clock64() - t0 < TC_WAIT_CYCLES) {
            }
        }
    } else if (warp == 1) {
        const uint32_t idesc = make_idesc(128, cols);
        const uint64_t bdesc = make_sdesc(conv0);
        for (int i = 0; i < n_kb; ++i) {
            const int c = i & 1;
            if (!wait_warp(conv_full + 8 * c, (i >> 1) & 1, abort, P.status)) break;
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < LS_KB / 16; ++kk)
                tc_mma_ta(tmem, tmem_a + 64 * c + 8 * kk, bdesc + (uint64_t)((c * cols * 256 + (kk >> 2) * cols * 128) >> 4) + 2 * (kk & 3), idesc,
                          i > 0 || kk > 0);
            tc_commit(conv_empty + 8 * c);
        }
        tc_commit(done);
        const long long t0 = clock64();
        while (!mbar_try_wait(done, 0) && clock64() - t0 < TC_WAIT_CYCLES) {
        }
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
            tmem_wait_st();
            fence_proxy_async();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(raw_empty + 8 * s);
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
    // ---- four channels of one token per thread and step, summed over the cluster
    if (shares > 1) cluster_sync();
    const int c_lo = cols * rank / shares, c_hi = (int)min((long long)(cols * (rank + 1) / shares), P.M - m0);
    for (int i = c_lo * 32 + threadIdx.x; i < c_hi * 32; i += LS_THREADS) {
        const int c = i >> 5, ch = n0 + 4 * (i & 31);
        const uint32_t at = raw0 + (uint32_t)i * 16;
        float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int r = 0; r < shares; ++r) {
            const float4 b = ld_cluster_f4(cluster_addr(at, r));
            a.x += b.x, a.y += b.y, a.z += b.z, a.w += b.w;
        }
        const float v[4] = {a.x, a.y, a.z, a.w}, sx = __ldg(P.sx + m0 + c);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (ch + e < P.N)
                store_y(P.y, P.y_type, (m0 + c) * P.ys + ch + e,
                        fmaf(v[e] * sx, __ldg(P.sw + ch + e), P.bias ? __ldg(P.bias + ch + e) : 0.0f));
    }
    if (shares > 1) cluster_sync();  // (the others have read this CTA's sums)
}

// Codes as [rows][K] bytes in boxes of 128 codes x `box` rows, 128-byte swizzle.
bool encode_rows(CUtensorMap* map, const int8_t* codes, long long rows, int K, long long stride, int box) {
    EncodeTiledFn enc = encode_tiled();
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
    const cuuint32_t b[2] = {(cuuint32_t)LS_KB, (cuuint32_t)box}, es[2] = {1, 1};
    return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(codes), dims, strides, b, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

fxpq_status launch_few(LinArgs& P, cudaStream_t st) {
    static bool set = false;
    if (!set) {
        if (cudaFuncSetAttribute(linear_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ls_smem(128, 4)) != cudaSuccess) return FXPQ_ERR_CUDA;
        set = true;
    }
    const long long tn = (P.N + 127) / 128, tm = (P.M + P.cols - 1) / P.cols;
    if (tn > 65535 || tm > 65535) return FXPQ_ERR_UNSUPPORTED;
    const int room = (P.cols <= 64 ? 2 : 1) * num_sms();
    int shares = 1;
    while (shares < 8 && tn * tm * shares * 2 <= room && P.n_kb >= 4 * shares) shares *= 2;
    P.stages = P.cols <= 32 ? 4 : 3;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = shares, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)shares, (unsigned)tn, (unsigned)tm);
    c.blockDim = dim3(LS_THREADS);
    c.dynamicSmemBytes = ls_smem(P.cols, P.stages);
    c.stream = st;
    c.attrs = at;
    c.numAttrs = shares > 1 ? 2 : 1;
    (void)cudaLaunchKernelEx(&c, linear_few_kernel, P);
    return after_launch("linear_few");
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
    LinArgs P;
    P.cols = M >= 128 ? 128 : (int)(M + 15) / 16 * 16;
    P.n_kb = (K + LS_KB - 1) / LS_KB;
    if (K > 0 && (!encode_rows(&P.tw, d_w, N, K, w_stride, 128) || !encode_rows(&P.tx, d_x, M, K, x_stride, P.cols))) return FXPQ_ERR_CUDA;
    P.sx = d_sx, P.sw = d_sw, P.bias = d_bias, P.y = d_y, P.ys = y_stride, P.M = M, P.N = N, P.y_type = y_type;
    P.status = status_ptr();
    return launch_few(P, as_stream(stream));
}

namespace {
// The workspace of fxpq_linear_tokens: codes, scales, then fxpq_linear_i8's.
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
size_t codes_pitch(int32_t K) { return ((size_t)K + 15) / 16 * 16; }
}  // namespace

extern "C" size_t fxpq_linear_tokens_workspace(int64_t M, int32_t N, int32_t K) {
    if (M <= 0 || N < 0 || K < 0) return 0;
    return up256((size_t)M * codes_pitch(K)) + up256((size_t)M * sizeof(float)) + fxpq_linear_i8_workspace(M, N, K);
}

extern "C" fxpq_status fxpq_linear_tokens(const void* d_x, int32_t x_type, int64_t x_stride, const int8_t* d_w, int64_t w_stride,
                                          const float* d_sw, const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type,
                                          void* d_y, int64_t y_stride, void* d_ws, size_t ws_bytes, void* stream) {
    if (M < 0 || N < 0 || K < 0 || !ftype_ok(x_type) || !ftype_ok(y_type)) return FXPQ_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return FXPQ_OK;
    const size_t need = fxpq_linear_tokens_workspace(M, N, K);
    if (!d_ws || ws_bytes < need || !aligned(d_ws, 256)) return FXPQ_ERR_WORKSPACE;
    const size_t pitch = codes_pitch(K), c = up256((size_t)M * pitch), s = up256((size_t)M * sizeof(float));
    int8_t* codes = static_cast<int8_t*>(d_ws);
    float* scale = reinterpret_cast<float*>(codes + c);
    const fxpq_status bad = check_linear(codes, pitch, scale, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride);
    if (bad != FXPQ_OK) return bad;  // (before anything is launched)
    const fxpq_status rc = fxpq_quantize_tokens(d_x, x_type, M, K, x_stride, codes, (int64_t)pitch, scale, stream);
    if (rc != FXPQ_OK) return rc;
    return fxpq_linear_i8(codes, (int64_t)pitch, scale, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, codes + c + s,
                          need - c - s, stream);
}
