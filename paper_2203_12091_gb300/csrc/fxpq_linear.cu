// fxpq_linear.cu -- rows quantized to 8 bits with a scale each, and the product of 8-bit rows with scales for
// each token and each output channel.
#include <atomic>
#include <cfloat>
#include <type_traits>

#include "fxpq_llm.cuh"
#include "fxpq_ptx.cuh"

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
template <typename T, typename C, int QT_THREADS>
__global__ void __launch_bounds__(QT_THREADS)
    quantize_tokens_kernel(const T* __restrict__ x, int K, long long x_stride, int vec, C* __restrict__ codes, long long c_stride, int c_vec,
                           float* __restrict__ scale, int* status) {
    constexpr bool HALF = sizeof(C) == 2;
    pdl_wait();
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

__device__ __forceinline__ void store_y(void* y, int type, long long at, float v) {
    if (type == FXPQ_FT_F32)
        static_cast<float*>(y)[at] = v;
    else if (type == FXPQ_FT_F16)
        static_cast<__half*>(y)[at] = __float2half_rn(v);
    else
        static_cast<__nv_bfloat16*>(y)[at] = __float2bfloat16_rn(v);
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
constexpr int LS_THREADS = 384, LS_KB = 128, LS_A = 128 * LS_KB;

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


// ------------------------------------------------------------------ many tokens
// The same product, bound by the tensor pipe: pairs of CTAs share tiles of 256 channels x 256 tokens (cta_group::2), so
// that a CTA reads only half of the tokens' operand from its shared memory.  Per 64 codes of the reduction (512 cycles of
// products) it moves 8 KB of weight codes in and out and 16 KB of tokens in and once through the tensor core: 384 cycles
// of shared memory, where one CTA alone would need 640, and both operands as fp16 in shared memory 512.  The tokens arrive
// as fp16 codes (written so by the quantizer, or expanded before), the weights as bytes, expanded into tensor memory.
//   warp 0  weights' copies;  1  tokens' copies;  2  tensor memory, products (CTA 0);  4-7  converters;  8-15  epilogue.
// The accumulators fill half of tensor memory, the weights' four stages the other half.  The epilogue scales and packs the
// sums into registers first, so that the next tile's products begin while it still stores.
constexpr int LM_THREADS = 512, LM_RAW = 3, LM_B = 8, LM_A = 4;
constexpr int LM_SMEM = 1024 + LM_RAW * LS_A + LM_B * 128 * 128;

struct ManyArgs {
    CUtensorMap tw, tx;  // weights' codes (boxes of 128 codes x 128 rows), tokens' fp16 codes (64 x 128)
    const float *sx, *sw, *bias;
    void* y;
    long long ys, M;
    int N, K, y_type, y_pair;  // y_pair: two 16-bit outputs in one aligned access
    int tiles_n, tiles_m, n_tiles;
    int* status;
};

// Tile t: groups of 8 token tiles, in a group the channel tiles outermost, so that the tiles of a moment share both operands.
__device__ __forceinline__ void tile_of(const ManyArgs& P, int t, int& tn, int& tm) {
    const int per = 8 * P.tiles_n, g = t / per, in = t - g * per, wide = min(8, P.tiles_m - 8 * g);
    tn = in / wide;
    tm = 8 * g + in - tn * wide;
}

// NT: tokens of a tile, 256 or, where those tiles would leave pairs idle, 128.
template <int NT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LM_THREADS, 1) linear_many_kernel(const __grid_constant__ ManyArgs P) {
    using namespace tc;
    constexpr int ROWS = NT / 2, STAGE = ROWS * 128;  // tokens of a CTA's half of the operand and of an epilogue warp; its stage
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    __shared__ __align__(8) uint64_t bars[2 * LM_RAW + 2 * LM_B + 2 * LM_A + 3];
    __shared__ __align__(16) float s_sx[8][ROWS];
    __shared__ int abort_flag;
    __shared__ uint32_t tmem_slot;
    volatile int* abort = &abort_flag;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t raw_full = smem_u32(bars), raw_empty = raw_full + 8 * LM_RAW, b_full = raw_empty + 8 * LM_RAW, b_empty = b_full + 8 * LM_B,
                   a_full = b_empty + 8 * LM_B, a_empty = a_full + 8 * LM_A, acc_full = a_empty + 8 * LM_A, acc_empty = acc_full + 8,
                   done = acc_empty + 8;
    const uint32_t raw0 = smem_u32(smem), b0 = raw0 + LM_RAW * LS_A;
    if (threadIdx.x == 0) {
        for (int i = 0; i < LM_RAW; ++i) {
            mbar_init(raw_full + 8 * i, 1);
            mbar_init(raw_empty + 8 * i, 4);
        }
        for (int i = 0; i < LM_B; ++i) {
            mbar_init(b_full + 8 * i, 1);  // (CTA 0's: its own arrival, the bytes of both)
            mbar_init(b_empty + 8 * i, 1);
        }
        for (int i = 0; i < LM_A; ++i) {
            mbar_init(a_full + 8 * i, 8);  // (CTA 0's: the converter warps of both)
            mbar_init(a_empty + 8 * i, 1);
        }
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, 16);  // (CTA 0's: the epilogue warps of both)
        mbar_init(done, 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&P.tw);
        prefetch_tmap(&P.tx);
    }
    pdl_wait();
    __syncthreads();
    cluster_sync();  // both CTAs' barriers exist
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    cluster_sync();
    const uint32_t tmem = tmem_slot, tmem_a = tmem + 256;
    const int n_kb = (P.K + LS_KB - 1) / LS_KB, n_half = (P.K + 63) / 64;

    if (warp == 0) {
        uint32_t it = 0;
        bool ok = true;
        for (int t = pair; t < P.n_tiles && ok; t += pairs) {
            int tn, tm;
            tile_of(P, t, tn, tm);
            for (int kb = 0; kb < n_kb; ++kb, ++it) {
                const uint32_t s = it % LM_RAW;
                if (!wait_warp(raw_empty + 8 * s, ((it / LM_RAW) & 1) ^ 1, abort, P.status)) {
                    ok = false;
                    break;
                }
                mbar_arrive_expect_tx(raw_full + 8 * s, LS_A);
                tma_load_2d(raw0 + s * LS_A, &P.tw, kb * LS_KB, tn * 256 + rank * 128, raw_full + 8 * s);
            }
        }
        for (uint32_t j = it > LM_RAW ? it - LM_RAW : 0; j < it; ++j) {  // every copy has landed
            drain_warp(raw_full + 8 * (j % LM_RAW), (j / LM_RAW) & 1);
        }
    } else if (warp == 1) {
        uint32_t it = 0;
        bool ok = true;
        const uint32_t lead = cluster_addr(b_full, 0);
        for (int t = pair; t < P.n_tiles && ok; t += pairs) {
            int tn, tm;
            tile_of(P, t, tn, tm);
            for (int hb = 0; hb < n_half; ++hb, ++it) {
                const uint32_t s = it % LM_B;
                if (!wait_warp(b_empty + 8 * s, ((it / LM_B) & 1) ^ 1, abort, P.status)) {
                    ok = false;
                    break;
                }
                if (rank == 0) mbar_arrive_expect_tx(b_full + 8 * s, 2 * STAGE);
                tma_load_2d_pair(b0 + s * STAGE, &P.tx, hb * 64, tm * NT + rank * ROWS, lead + 8 * s);
            }
        }
        if (rank == 0)
            for (uint32_t j = it > LM_B ? it - LM_B : 0; j < it; ++j) {
                drain_warp(b_full + 8 * (j % LM_B), (j / LM_B) & 1);
            }
    } else if (warp == 2) {
        if (rank == 0) {
            const uint32_t idesc = make_idesc(256, NT);
            const uint64_t bd0 = make_sdesc(b0);
            uint32_t ia = 0, ib = 0, it = 0;
            bool ok = true;
            for (int t = pair; t < P.n_tiles && ok; t += pairs, ++it) {
                if (!wait_warp_cluster(acc_empty, (it & 1) ^ 1, abort, P.status)) break;
                tc_fence_after();
                uint32_t acc = 0;
                for (int kb = 0; kb < n_kb && ok; ++kb, ++ia) {
                    const uint32_t c = ia % LM_A;
                    if (!wait_warp_cluster(a_full + 8 * c, (ia / LM_A) & 1, abort, P.status)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    for (int hf = 0; hf < min(2, n_half - 2 * kb); ++hf, ++ib) {
                        const uint32_t s = ib % LM_B;
                        if (!wait_warp_cluster(b_full + 8 * s, (ib / LM_B) & 1, abort, P.status)) {
                            ok = false;
                            break;
                        }
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) {
                            tc_mma_ta_pair(tmem, tmem_a + 64 * c + 32 * hf + 8 * kk, bd0 + s * (STAGE >> 4) + 2 * kk, idesc, acc);
                            acc = 1;
                        }
                        tc_commit_pair(b_empty + 8 * s);
                    }
                    if (ok) tc_commit_pair(a_empty + 8 * c);
                }
                if (ok) tc_commit_pair(acc_full);
            }
            tc_commit_pair(done);
        }
        drain_warp(done, 0);
    } else if (warp >= 4 && warp < 8) {
        const int quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lead = cluster_addr(a_full, 0);
        uint32_t it = 0;
        bool ok = true;
        for (int t = pair; t < P.n_tiles && ok; t += pairs)
            for (int kb = 0; kb < n_kb; ++kb, ++it) {
                const uint32_t s = it % LM_RAW, c = it % LM_A;
                if (!wait_warp(raw_full + 8 * s, (it / LM_RAW) & 1, abort, P.status) ||
                    !wait_warp_cluster(a_empty + 8 * c, ((it / LM_A) & 1) ^ 1, abort, P.status)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const unsigned char* ra = smem + s * LS_A;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
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
                    tmem_st32_nw(tmem_a + ((uint32_t)(quad * 32) << 16) + 64 * c + 32 * hf, r);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(raw_empty + 8 * s);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(lead + 8 * c);
            }
    } else if (warp >= 8) {
        const int quad = warp & 3, half = (warp - 8) >> 2;  // channels 32 quad + lane, tokens ROWS half ..
        const uint32_t lead = cluster_addr(acc_empty, 0), at = tmem + ((uint32_t)(quad * 32) << 16) + ROWS * half;
        float* sxs = s_sx[warp - 8];
        uint32_t it = 0;
        for (int t = pair; t < P.n_tiles; t += pairs, ++it) {
            int tn, tm;
            tile_of(P, t, tn, tm);
            const int ch = tn * 256 + rank * 128 + quad * 32 + lane;
            const long long m0 = (long long)tm * NT + ROWS * half;
            const float sw = ch < P.N ? __ldg(P.sw + ch) : 0.0f, bias = P.bias && ch < P.N ? __ldg(P.bias + ch) : 0.0f;
            for (int i = lane; i < ROWS; i += 32) sxs[i] = m0 + i < P.M ? __ldg(P.sx + m0 + i) : 0.0f;
            __syncwarp();
            if (!wait_warp_cluster(acc_full, it & 1, abort, P.status)) break;
            tc_fence_after();
            const int cols = (int)min((long long)ROWS, P.M - m0);
            if (P.y_type == FXPQ_FT_F32) {
                for (int c = 0; c < ROWS; c += 16) {
                    uint32_t v[16];
                    tmem_ld16_nw(at + c, v);
                    tmem_wait_ld();
                    reg_fence(v);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (c + e < cols && ch < P.N)
                            static_cast<float*>(P.y)[(m0 + c + e) * P.ys + ch] = fmaf(__uint_as_float(v[e]) * sxs[c + e], sw, bias);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(lead);
                continue;
            }
            uint32_t y[ROWS / 2];  // tokens 2 i, 2 i + 1 of this thread's channel
#pragma unroll
            for (int c = 0; c < ROWS; c += 16) {
                uint32_t v[16];
                tmem_ld16_nw(at + c, v);
                tmem_wait_ld();
                reg_fence(v);
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float2 sx = *reinterpret_cast<const float2*>(sxs + c + e);
                    const float a = fmaf(__uint_as_float(v[e]) * sx.x, sw, bias), b = fmaf(__uint_as_float(v[e + 1]) * sx.y, sw, bias);
                    if (P.y_type == FXPQ_FT_F16) {
                        y[(c + e) / 2] = h2_bits(__floats2half2_rn(a, b));
                    } else {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
                        y[(c + e) / 2] = *reinterpret_cast<const uint32_t*>(&h);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(lead);  // the accumulators may be overwritten
            unsigned short* out = static_cast<unsigned short*>(P.y);
            if (P.y_pair) {  // even lanes store the even token's two channels, odd lanes the odd token's
                const int odd = lane & 1, c0 = ch - odd;
#pragma unroll
                for (int i = 0; i < ROWS / 2; ++i) {
                    const uint32_t o = __shfl_xor_sync(0xffffffffu, y[i], 1);
                    const uint32_t w = odd ? __byte_perm(o, y[i], 0x7632) : __byte_perm(y[i], o, 0x5410);
                    const long long m = m0 + 2 * i + odd;
                    if (2 * i + odd < cols && c0 < P.N) {
                        if (c0 + 1 < P.N)
                            *reinterpret_cast<uint32_t*>(out + m * P.ys + c0) = w;
                        else
                            out[m * P.ys + c0] = (unsigned short)w;
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < ROWS / 2; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (2 * i + e < cols && ch < P.N) out[(m0 + 2 * i + e) * P.ys + ch] = (unsigned short)(y[i] >> (16 * e));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
    }
    cluster_sync();  // (the other CTA may still arrive on this one's barriers until here)
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

// Codes as [rows][K] bytes in boxes of 128 codes x `box` rows, 128-byte swizzle.
bool encode_rows(CUtensorMap* map, const int8_t* codes, long long rows, int K, long long stride, int box) {
    EncodeTiledFn enc = encode_tiled();
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
    const cuuint32_t b[2] = {(cuuint32_t)LS_KB, (cuuint32_t)box}, es[2] = {1, 1};
    return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(codes), dims, strides, b, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tokens' fp16 codes in boxes of 64 codes x `box` rows.
bool encode_half_rows(CUtensorMap* map, const __half* codes, long long rows, int K, long long pitch, int box) {
    EncodeTiledFn enc = encode_tiled();
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch * 2};
    const cuuint32_t b[2] = {64, (cuuint32_t)box}, es[2] = {1, 1};
    return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<__half*>(codes), dims, strides, b, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t codes_pitch(int32_t K) { return ((size_t)K + 15) / 16 * 16; }

// Many tokens go to the pairs of CTAs.
bool many_tokens(int64_t M, int32_t N, int32_t K) { return M > 256 && N >= 128 && K >= 128; }

template <int NT>
fxpq_status launch_many(ManyArgs& P, cudaStream_t st) {
    static bool set = false;
    if (!set) {
        if (cudaFuncSetAttribute(linear_many_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, LM_SMEM) != cudaSuccess) return FXPQ_ERR_CUDA;
        set = true;
    }
    const long long tn = ((long long)P.N + 255) / 256, tm = (P.M + NT - 1) / NT;
    if (tn * tm > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    P.tiles_n = (int)tn, P.tiles_m = (int)tm, P.n_tiles = (int)(tn * tm);
    P.y_pair = aligned(P.y, 4) && P.ys % 2 == 0;
    const int pairs = num_sms() / 2 > 0 ? num_sms() / 2 : 1;
    launch_pdl(linear_many_kernel<NT>, dim3(2 * (unsigned)(P.n_tiles < pairs ? P.n_tiles : pairs)), dim3(LM_THREADS), LM_SMEM, st, P);
    return after_launch("linear_many");
}

template <bool HALF>
fxpq_status launch_few(LinArgs& P, cudaStream_t st) {
    static bool set = false;
    if (!set) {
        if (cudaFuncSetAttribute(linear_few_kernel<HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, ls_smem(128, 4, HALF)) != cudaSuccess)
            return FXPQ_ERR_CUDA;
        set = true;
    }
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
        static std::atomic<int> room[2][9][4];  // clusters that run at once, by tile width and size, asked for once
        const int w = P.cols / 16, l = shares == 1 ? 1 : shares == 2 ? 2 : 3;
        int n = room[HALF][w][l].load(std::memory_order_relaxed);
        if (n == 0) {
            at[1].val.clusterDim.x = 2 * shares;
            c.gridDim = dim3(2 * shares, 1024, 1);
            c.numAttrs = 2;
            if (cudaOccupancyMaxActiveClusters(&n, linear_few_kernel<HALF>, &c) != cudaSuccess || n <= 0) {
                (void)cudaGetLastError();
                n = -1;
            }
            room[HALF][w][l].store(n, std::memory_order_relaxed);
        }
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
                          float* d_scale, cudaStream_t st) {
    const int e = ftype_bytes(x_type), vec = aligned(d_x, 16) && x_stride * e % 16 == 0;
    const int c_vec = aligned(d_codes, 8) && codes_stride % 8 == 0;
    const dim3 grid((unsigned)M);
    int* status = status_ptr();
    auto launch = [&](auto* x) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(x)>>;
        if (K <= 4096)
            launch_pdl(quantize_tokens_kernel<T, C, 128>, grid, dim3(128), 0, st, x, K, x_stride, vec, d_codes, codes_stride, c_vec, d_scale, status);
        else if (K > 8192)
            launch_pdl(quantize_tokens_kernel<T, C, 1024>, grid, dim3(1024), 0, st, x, K, x_stride, vec, d_codes, codes_stride, c_vec, d_scale, status);
        else
            launch_pdl(quantize_tokens_kernel<T, C, 256>, grid, dim3(256), 0, st, x, K, x_stride, vec, d_codes, codes_stride, c_vec, d_scale, status);
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

fxpq_status product_many(const __half* half, size_t pitch, const float* d_sx, const int8_t* d_w, int64_t w_stride, const float* d_sw,
                         const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type, void* d_y, int64_t y_stride, cudaStream_t st) {
    ManyArgs P;
    // Tiles of 256 tokens, or of 128 where their rounds over the pairs take less time.  A round of the narrow ones takes two
    // thirds of the wide ones' (8192 x 8192 of 4096: 13.2 and 20.1 us; every tile expands 256 channels' weights).
    const int64_t pairs = num_sms() / 2 > 0 ? num_sms() / 2 : 1, tn = ((int64_t)N + 255) / 256;
    const auto rounds = [&](int64_t nt) { return (tn * ((M + nt - 1) / nt) + pairs - 1) / pairs; };
    const int nt = 2 * rounds(128) < 3 * rounds(256) ? 128 : 256;
    if (!encode_rows(&P.tw, d_w, N, K, w_stride, 128) || !encode_half_rows(&P.tx, half, M, K, (long long)pitch, nt / 2)) return FXPQ_ERR_CUDA;
    P.sx = d_sx, P.sw = d_sw, P.bias = d_bias, P.y = d_y, P.ys = y_stride, P.M = M, P.N = N, P.K = K, P.y_type = y_type;
    P.status = status_ptr();
    return nt == 128 ? launch_many<128>(P, st) : launch_many<256>(P, st);
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
        return product_many(half, pitch, d_sx, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, as_stream(stream));
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
    if (many_tokens(M, N, K)) return product_many(half, pitch, scale, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, st);
    return product_few(nullptr, half, (int64_t)pitch, scale, d_w, w_stride, d_sw, d_bias, M, N, K, y_type, d_y, y_stride, st);
}
