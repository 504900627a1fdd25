#pragma once
// fxpq_linear.cuh -- products of rows (8-bit codes, or fp16) with 8-bit weights on tcgen05, and their launches.
#include <atomic>
#include <type_traits>

#include "fxpq_layer.cuh"
#include "fxpq_ptx.cuh"

namespace fxpq {
namespace llm {
namespace {

__device__ __forceinline__ void store_y(void* y, int type, long long at, float v) {
    if (type == FXPQ_FT_F32)
        static_cast<float*>(y)[at] = v;
    else if (type == FXPQ_FT_F16)
        static_cast<__half*>(y)[at] = __float2half_rn(v);
    else
        static_cast<__nv_bfloat16*>(y)[at] = __float2bfloat16_rn(v);
}

// What follows the sums of a product: PLAIN, y = sum * sx * sw + bias; LAYER, activation and residual after that; GATED, neighbouring
// channels' activation times value.  Both of the latter may keep the sums (scaled, in fp16, or as they are) for a gradient.
enum { PLAIN, LAYER, GATED };
struct Epi {
    const void* res;
    long long res_stride;
    void* pre;
    float pre_scale;
    int pre_f32, act;
    int vec;   // few: outputs, residuals and kept sums of four channels in aligned accesses each (bits 1, 2, 4)
    int fast;  // many: 16-bit outputs, pairs of everything aligned, no erfc
};

// Rows as they come, for products that form their codes themselves.
struct FloatRows {
    const void* x;
    long long x_stride;
    int x_type, x_vec, K;
    float* sx;  // the rows' scales, or null
    RowNorm norm;
};

struct LinArgs {
    // weights' codes as [N][K] bytes in boxes of 128 codes x 128 rows (tw), or x the rows that the last tile has (tw2: a box is
    // slow where it lies outside the tensor); tokens' as [M][K] bytes in boxes of 128 x `rows`, or as fp16 in 64 x `rows`
    CUtensorMap tw, tw2, tx;
    const float *sx, *sw, *bias;  // null: ones, ones, zeros
    void* y;
    long long ys, M;
    int N, y_type, n_kb;
    int rows, cols;  // tokens of a tile, and rounded up to 16, at most 128 (the columns past `rows` hold whatever the stage does)
    int w_rows;      // channels of the last tile
    int y_four;      // four outputs of a row in one aligned access
    int stages;
    int early;       // the kernel before is this call's quantizer, which lets this one begin: weights may be read before its codes exist
    int* status;
    Epi e;
    FloatRows f;
};

// N values at p + at, one aligned access if vec and all of them count.
template <int N>
__device__ __forceinline__ void store_some(void* p, int type, long long at, const float (&v)[N], int count, bool vec) {
    if (vec && count >= N) {
        if (type == FXPQ_FT_F32) {
            if constexpr (N == 4)
                *reinterpret_cast<float4*>(static_cast<float*>(p) + at) = make_float4(v[0], v[1], v[2], v[3]);
            else
                *reinterpret_cast<float2*>(static_cast<float*>(p) + at) = make_float2(v[0], v[1]);
        } else {
            uint32_t w[N / 2];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                if (type == FXPQ_FT_F16) {
                    w[i] = h2_bits(__floats2half2_rn(v[2 * i], v[2 * i + 1]));
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&h);
                }
            }
            unsigned short* q = static_cast<unsigned short*>(p) + at;
            if constexpr (N == 4)
                *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
            else
                *reinterpret_cast<uint32_t*>(q) = w[0];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < count) store_y(p, type, at + i, v[i]);
    }
}
__device__ __forceinline__ float load_y(const void* p, int type, long long at) {
    return type == FXPQ_FT_F32 ? static_cast<const float*>(p)[at]
                               : type == FXPQ_FT_F16 ? __half2float(static_cast<const __half*>(p)[at]) : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
}
__device__ __forceinline__ float2 pair_f32(uint32_t w, int type) {
    return type == FXPQ_FT_F16 ? __half22float2(*reinterpret_cast<const __half2*>(&w)) : __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
}

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

// How the tokens come: as bytes, as fp16 codes, or as rows of floats (up to 16), whose codes every CTA forms for its share of the reduction.
enum { BYTES, HALVES, FLOATS };
constexpr int LF_ROWS = 16, LF_BLOCK = LF_ROWS * LS_KB * 2, LF_MOST = 32;  // its tile, the bytes of its block of codes, blocks of a share

// bytes: stages and two expanded token stages; floats: stages of weights alone and all of the share's codes
__host__ __device__ inline int ls_smem(int cols, int stages, int tok, int blocks) {
    const int ring = tok == HALVES ? stages * (LS_A + cols * LS_KB * 2)
                                   : tok == FLOATS ? stages * LS_A + blocks * LF_BLOCK : stages * (LS_A + cols * LS_KB) + 2 * cols * LS_KB * 2;
    const int sums = cols * 128 * 4;
    return 1024 + (ring > sums ? ring : sums);
}

// Codes of up to 16 rows of floats by 256 threads (8 warps): every row's scale from the whole row, then the fp16 codes of n_kb blocks
// from block kb0 on into shared memory, as the products read them.  The same fp32 steps as the token quantizer's.
struct RowSpace {
    float top[LF_ROWS][8], far[LF_ROWS][8], sum[LF_ROWS][8], inv[LF_ROWS], sx[LF_ROWS];
};
template <typename T>
__device__ void own_codes(const FloatRows& F, int M, int kb0, int n_kb, unsigned char* blocks, RowSpace& S, int t, bool first, int* status) {
    const T* x = static_cast<const T*>(F.x);
    const int warp = t >> 5, lane = t & 31, K = F.K, groups = K / 8;
    const int parts = M <= 1 ? 8 : M <= 2 ? 4 : M <= 4 ? 2 : 1;  // warps of a row
    const auto join = []() { asm volatile("bar.sync 1, 256;" ::: "memory"); };
    // (a second time, in other units, for rows under a norm whose squares leave fp32)
    auto scan = [&](bool again) {
        for (int u = warp; u < M * parts; u += 8) {
            const int m = u / parts, p = u - m * parts;
            const T* row = x + m * F.x_stride;
            RowStats st;
            float per_unit = 1.0f;
            if (again) {
                st.far = S.far[m][0];
                per_unit = 1.0f / st.unit();
                st = RowStats();
            }
            constexpr int DEPTH = 4;  // groups of eight in flight
            for (int g0 = p * 32 + lane; g0 < groups; g0 += DEPTH * 32 * parts) {
                float v[DEPTH][8];
#pragma unroll
                for (int d = 0; d < DEPTH; ++d)
                    if (g0 + d * 32 * parts < groups) load_f32<8>(row + 8 * (g0 + d * 32 * parts), F.x_vec, v[d]);
#pragma unroll
                for (int d = 0; d < DEPTH; ++d) {
                    const int g = g0 + d * 32 * parts;
                    if (g >= groups) break;
                    float w[8];
                    if (F.norm.weight)
                        load_f32<8>(F.norm.weight + 8 * g, F.norm.vec, w);
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = 1.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) st.see(v[d][e], w[e], per_unit);
                }
            }
            if (p == 0 && 8 * groups + lane < K)
                st.see(to_f32(row[8 * groups + lane]), F.norm.weight ? __ldg(F.norm.weight + 8 * groups + lane) : 1.0f, per_unit);
            const bool bad = __any_sync(0xffffffffu, st.bad);
            st.meet();
            if (again) {
                if (lane == 0) S.sum[m][p] = st.sum;
            } else if (lane == 0) {
                S.top[m][p] = st.top, S.far[m][p] = st.far, S.sum[m][p] = st.sum;
                if (bad && first) latch_status(status, FXPQ_ERR_NONFINITE);
            }
        }
    };
    scan(false);
    join();
    RowStats st;
    float unit = 1.0f;
    if (t < M)
        for (int p = 0; p < parts; ++p) st.top = fmaxf(st.top, S.top[t][p]), st.far = fmaxf(st.far, S.far[t][p]), st.sum += S.sum[t][p];
    if (F.norm.weight) {
        if (t < M) unit = st.unit(), S.far[t][0] = st.far;
        int any;
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.or.pred q, 1, 256, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                     : "=r"(any)
                     : "r"((int)(unit != 1.0f))
                     : "memory");
        if (any) {
            scan(true);
            join();
            if (t < M) {
                st.sum = 0.0f;
                for (int p = 0; p < parts; ++p) st.sum += S.sum[t][p];
            }
        }
    }
    if (t < M) {
        float inv, scale;
        if (F.norm.weight) {
            scale = st.scale(K, F.norm.eps, unit, inv);
        } else {
            inv = st.inverse();
            scale = inv != 0.0f ? __fmul_rn(st.top, 1.0f / 127.0f) : 0.0f;
        }
        S.inv[t] = inv, S.sx[t] = scale;
        if (F.sx && first) F.sx[t] = scale;
    }
    join();
    const int chunks = n_kb * (LS_KB / 8);
    for (int i = t; i < M * chunks; i += 256) {
        const int m = i / chunks, c = i - m * chunks, k = kb0 * LS_KB + 8 * c, b = c >> 4, hf = (c >> 3) & 1;
        const T* row = x + m * F.x_stride;
        const float inv = S.inv[m];
        float v[8];
        if (k + 8 <= K) {
            float w[8];
            load_f32<8>(row + k, F.x_vec, v);
            if (F.norm.weight) load_f32<8>(F.norm.weight + k, F.norm.vec, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = RowStats::value(v[e], F.norm.weight ? w[e] : 1.0f);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = k + e < K ? RowStats::value(to_f32(row[k + e]), F.norm.weight ? __ldg(F.norm.weight + k + e) : 1.0f) : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], inv);
        *reinterpret_cast<uint4*>(blocks + b * LF_BLOCK + hf * LF_ROWS * 128 + m * 128 + (((c & 7) ^ (m & 7)) << 4)) =
            make_uint4(f32_codes_f16x2(v[0], v[1]), f32_codes_f16x2(v[2], v[3]), f32_codes_f16x2(v[4], v[5]), f32_codes_f16x2(v[6], v[7]));
    }
}

template <int TOK, int EPI>
__global__ void __launch_bounds__(LS_THREADS) linear_few_kernel(const __grid_constant__ LinArgs P) {
    using namespace tc;
    constexpr bool HALF = TOK == HALVES;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    __shared__ __align__(8) uint64_t bars[8 + 8 + 2 + 2 + 1 + 1];
    __shared__ int abort_flag;
    __shared__ std::conditional_t<TOK == FLOATS, RowSpace, char> rows_space;
    __shared__ uint32_t tmem_slot;
    volatile int* abort = &abort_flag;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, ST = P.stages, cols = P.cols;
    const uint32_t raw_full = smem_u32(bars), raw_empty = raw_full + 8 * 8, conv_full = raw_empty + 8 * 8, conv_empty = conv_full + 16,
                   done = conv_empty + 16, tok_full = done + 8;
    const int raw_bytes = TOK == FLOATS ? LS_A : LS_A + cols * LS_KB * (HALF ? 2 : 1);
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
        if (TOK == FLOATS) mbar_init(tok_full, 8);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (P.n_kb) {
            prefetch_tmap(blockIdx.y == gridDim.y - 1 ? &P.tw2 : &P.tw);
            if (TOK != FLOATS) prefetch_tmap(&P.tx);
        }
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(256u));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    const int rank = blockIdx.x, shares = gridDim.x, n0 = blockIdx.y * 128;
    const long long m0 = (long long)blockIdx.z * P.rows;
    const int kb0 = (int)((long long)P.n_kb * rank / shares), n_kb = (int)((long long)P.n_kb * (rank + 1) / shares) - kb0;
    const bool last = blockIdx.y == gridDim.y - 1;
    const CUtensorMap* tw = last ? &P.tw2 : &P.tw;
    const uint32_t bytes = (uint32_t)((last ? P.w_rows : 128) * LS_KB + (TOK == FLOATS ? 0 : P.rows * LS_KB * (HALF ? 2 : 1)));
    const int early = HALF && P.early ? min(ST, n_kb) : 0;
    if (warp == 0 && early) {
        __syncwarp();
        for (int i = 0; i < early; ++i) {
            mbar_arrive_expect_tx(raw_full + 8 * i, bytes);
            tma_load_2d(raw0 + i * raw_bytes, tw, (kb0 + i) * LS_KB, n0, raw_full + 8 * i);
        }
    }
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmem_a = tmem + 128;

    if (warp == 0) {
        int i = 0;
        for (; i < n_kb; ++i) {
            const int s = i % ST;
            if (!wait_warp(raw_empty + 8 * s, ((i / ST) & 1) ^ 1, abort, P.status)) break;
            const uint32_t bar = raw_full + 8 * s, dst = raw0 + s * raw_bytes;
            if (i >= early) {
                mbar_arrive_expect_tx(bar, bytes);
                tma_load_2d(dst, tw, (kb0 + i) * LS_KB, n0, bar);
            }
            if (TOK != FLOATS) tma_load_2d(dst + LS_A, &P.tx, (kb0 + i) * LS_KB, (int)m0, bar);
            if (HALF) tma_load_2d(dst + LS_A + cols * 128, &P.tx, (kb0 + i) * LS_KB + 64, (int)m0, bar);
        }
        for (int j = max(0, i - ST); j < i; ++j) {  // every copy has landed before this CTA's memory is used again
            drain_warp(raw_full + 8 * (j % ST), (j / ST) & 1);
        }
    } else if (warp == 1) {
        const uint32_t idesc = make_idesc(128, cols);
        const uint64_t bdesc = make_sdesc(HALF ? raw0 : conv0);
        if (TOK == FLOATS && n_kb > 0) wait_warp(tok_full, 0, abort, P.status);
        for (int i = 0; i < n_kb; ++i) {
            const int c = i & 1, s = i % ST;
            if (!wait_warp(conv_full + 8 * c, (i >> 1) & 1, abort, P.status)) break;
            if (HALF && !wait_warp(raw_full + 8 * s, (i / ST) & 1, abort, P.status)) break;
            tc_fence_after();
            const uint64_t bd = bdesc + (uint64_t)((HALF ? s * raw_bytes + LS_A : TOK == FLOATS ? i * LF_BLOCK : c * cols * 256) >> 4);
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
        if constexpr (TOK == FLOATS) {
            const int M = (int)P.M, tt = threadIdx.x - 128;
            const bool first = rank == 0 && blockIdx.y == 0;
            if (P.f.x_type == FXPQ_FT_F32)
                own_codes<float>(P.f, M, kb0, n_kb, smem + ST * raw_bytes, rows_space, tt, first, P.status);
            else if (P.f.x_type == FXPQ_FT_F16)
                own_codes<__half>(P.f, M, kb0, n_kb, smem + ST * raw_bytes, rows_space, tt, first, P.status);
            else
                own_codes<__nv_bfloat16>(P.f, M, kb0, n_kb, smem + ST * raw_bytes, rows_space, tt, first, P.status);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(tok_full);
        }
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
            if constexpr (TOK == BYTES) {
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
    auto scale_of = [&](int c) {
        if constexpr (TOK == FLOATS)
            return rows_space.sx[c];
        else
            return P.sx ? __ldg(P.sx + m0 + c) : 1.0f;
    };
    float sw[4], bias[4], sx = c_lo + warp < c_hi ? scale_of(c_lo + warp) : 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // (on their way while the CTAs meet)
        sw[e] = !P.sw ? 1.0f : ch + e < P.N ? __ldg(P.sw + ch + e) : 0.0f;
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
        if (c + TOKENS < c_hi) sx = scale_of(c + TOKENS);
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < shares) a.x += b[r].x, a.y += b[r].y, a.z += b[r].z, a.w += b[r].w;
        const float v[4] = {fmaf(a.x * s, sw[0], bias[0]), fmaf(a.y * s, sw[1], bias[1]), fmaf(a.z * s, sw[2], bias[2]), fmaf(a.w * s, sw[3], bias[3])};
        if constexpr (EPI != PLAIN) {
            const long long m = m0 + c;
            const int left = P.N - ch;
            if (P.e.pre) {
                const float k = P.e.pre_f32 ? 1.0f : P.e.pre_scale, keep[4] = {a.x * k, a.y * k, a.z * k, a.w * k};
                store_some<4>(P.e.pre, P.e.pre_f32 ? FXPQ_FT_F32 : FXPQ_FT_F16, m * P.N + ch, keep, left, P.e.vec & 4);
            }
            if constexpr (EPI == GATED) {
                const float y[2] = {activate(v[0], P.e.act) * v[1], activate(v[2], P.e.act) * v[3]};
                store_some<2>(P.y, P.y_type, m * P.ys + ch / 2, y, left / 2, P.e.vec & 1);
            } else {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = activate(v[e], P.e.act);
                if (P.e.res) {
                    const long long at = m * P.e.res_stride + ch;
                    if ((P.e.vec & 2) && left >= 4) {
                        if (P.y_type == FXPQ_FT_F32) {
                            const float4 r = *reinterpret_cast<const float4*>(static_cast<const float*>(P.e.res) + at);
                            y[0] += r.x, y[1] += r.y, y[2] += r.z, y[3] += r.w;
                        } else {
                            const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const unsigned short*>(P.e.res) + at);
                            const float2 p = pair_f32(w.x, P.y_type), q = pair_f32(w.y, P.y_type);
                            y[0] += p.x, y[1] += p.y, y[2] += q.x, y[3] += q.y;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e < left) y[e] += load_y(P.e.res, P.y_type, at + e);
                    }
                }
                store_some<4>(P.y, P.y_type, m * P.ys + ch, y, left, P.e.vec & 1);
            }
            continue;
        }
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
    Epi e;
};

// Tile t: groups of 8 token tiles, in a group the channel tiles outermost, so that the tiles of a moment share both operands.
__device__ __forceinline__ void tile_of(const ManyArgs& P, int t, int& tn, int& tm) {
    const int per = 8 * P.tiles_n, g = t / per, in = t - g * per, wide = min(8, P.tiles_m - 8 * g);
    tn = in / wide;
    tm = 8 * g + in - tn * wide;
}

// Channels c0, c0 + 1 (even, odd lane) of one token for each lane of a pair: the even lane gets the even token's, the odd lane the
// odd one's.  a, b: this lane's channel for the even and the odd token.
__device__ __forceinline__ float2 channel_pair(float a, float b, int odd) {
    const float o = __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
    return odd ? make_float2(o, b) : make_float2(a, o);
}

// SiLU and the tanh form of GELU as z / (1 + 2^t), t = c z (1 + b z^2).
struct SigAct {
    float c, b;
    __device__ __forceinline__ explicit SigAct(int act)
        : c(act == FXPQ_ACT_SILU ? -1.4426950408889634f : -1.4426950408889634f * GELU_A), b(act == FXPQ_ACT_SILU ? 0.0f : GELU_B) {}
    __device__ __forceinline__ float operator()(float z) const {
        float e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(c * z * fmaf(b, fminf(z * z, 1.0e30f), 1.0f)));
        return __fdividef(z, 1.0f + e);
    }
};

// The epilogue of a warp's 32 channels and ROWS tokens for LAYER and GATED.  Everything goes by pairs: two lanes exchange sums so that
// each holds two channels of one token.  The fast form holds all sums in registers (the epilogue's warps have taken the other
// warps'), and has given the accumulators back before it computes: for GATED 16384 of 4096, 8192 tokens, see fxpq_layer.cu.
template <int ROWS, int EPI, bool SIG, typename Sum>
__device__ __forceinline__ void epilogue_fast(const ManyArgs& P, Sum&& sum, const float* sxs, float2 sw, float2 bias, int c0, int odd, long long m0, int cols) {
    const bool f16 = P.y_type == FXPQ_FT_F16;
    const SigAct sig(P.e.act);
    const float low = P.e.act == FXPQ_ACT_RELU ? 0.0f : -__int_as_float(0x7f800000);
    cols = c0 < P.N ? cols - odd : 0;  // tokens 2 i + odd with 2 i < cols exist
    sxs += odd;
    const float ps = P.e.pre_scale;
    // (addresses that walk along the tokens: computed from the token each, they took more registers than there are)
    const long long y_step = 2 * P.ys * 2, r_step = 2 * P.e.res_stride * 2, p_step = 2LL * P.N * 2;
    char* pre = P.e.pre ? static_cast<char*>(P.e.pre) + ((m0 + odd) * P.N + c0) * 2 : nullptr;
    auto act = [&](float z) { return SIG ? sig(z) : fmaxf(z, low); };
    auto pack = [&](float a, float b) {
        if (f16) return h2_bits(__floats2half2_rn(a, b));
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    };
    auto pair = [&](int i) {  // z of channels c0, c0 + 1 for token 2 i + odd
        const float2 s = channel_pair(sum(2 * i), sum(2 * i + 1), odd);
        if (P.e.pre) {
            if (2 * i < cols) *reinterpret_cast<__half2*>(pre) = __floats2half2_rn(s.x * ps, s.y * ps);
            pre += p_step;
        }
        const float sx = sxs[2 * i];
        return make_float2(fmaf(s.x * sx, sw.x, bias.x), fmaf(s.y * sx, sw.y, bias.y));
    };
    if constexpr (EPI == GATED) {
        const int second = (threadIdx.x >> 1) & 1, reach = cols - 2 * second;
        char* y = static_cast<char*>(P.y) + ((m0 + odd + 2 * second) * P.ys + (c0 >> 1) - second) * 2;
#pragma unroll
        for (int i = 0; i < ROWS / 2; i += 2) {  // two columns of token 2 i + odd, or with `second` 2 i + 2 + odd
            const float2 p = pair(i), q = pair(i + 1);
            const float a = act(p.x) * p.y, b = act(q.x) * q.y;
            const float o = __shfl_xor_sync(0xffffffffu, second ? a : b, 2);
            if (2 * i < reach) *reinterpret_cast<uint32_t*>(y) = second ? pack(o, b) : pack(a, o);
            y += 2 * y_step;
        }
    } else {
        char* y = static_cast<char*>(P.y) + ((m0 + odd) * P.ys + c0) * 2;
        const char* res = static_cast<const char*>(P.e.res) + ((m0 + odd) * P.e.res_stride + c0) * 2;
#pragma unroll
        for (int i = 0; i < ROWS / 2; ++i) {
            const float2 p = pair(i);
            float a = act(p.x), b = act(p.y);
            if (2 * i < cols) {
                if (P.e.res) {
                    const float2 r = pair_f32(*reinterpret_cast<const uint32_t*>(res), P.y_type);
                    a += r.x, b += r.y;
                }
                *reinterpret_cast<uint32_t*>(y) = pack(a, b);
            }
            y += y_step, res += r_step;
        }
    }
}
// Any types, alignment and activation; 16 tokens of this lane's channel.
template <int EPI>
__device__ __forceinline__ void epilogue_any(const ManyArgs& P, const uint32_t (&v)[16], const float* sxs, float2 sw, float2 bias, int c0, int odd,
                                          long long m0, int cols) {
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        uint32_t a = 0, b = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k == i) a = v[2 * k], b = v[2 * k + 1];
        const float2 s = channel_pair(__uint_as_float(a), __uint_as_float(b), odd);
        const int t = 2 * i + odd, left = P.N - c0;
        if (t >= cols || left <= 0) continue;
        const long long m = m0 + t;
        if (P.e.pre) {
            const float k = P.e.pre_f32 ? 1.0f : P.e.pre_scale, keep[2] = {s.x * k, s.y * k};
            store_some<2>(P.e.pre, P.e.pre_f32 ? FXPQ_FT_F32 : FXPQ_FT_F16, m * P.N + c0, keep, left, false);
        }
        const float z0 = fmaf(s.x * sxs[t], sw.x, bias.x), z1 = fmaf(s.y * sxs[t], sw.y, bias.y), f = activate(z0, P.e.act);
        if constexpr (EPI == GATED) {
            store_y(P.y, P.y_type, m * P.ys + (c0 >> 1), f * z1);
        } else {
            float y[2] = {f, activate(z1, P.e.act)};
            if (P.e.res) {
                const long long at = m * P.e.res_stride + c0;
                y[0] += load_y(P.e.res, P.y_type, at);
                if (left > 1) y[1] += load_y(P.e.res, P.y_type, at + 1);
            }
            store_some<2>(P.y, P.y_type, m * P.ys + c0, y, left, false);
        }
    }
}

// Registers of a thread: the launch holds 512 x 128, of which the epilogue's warps take 256 x 176 and the others 128 x 56 (copies, products)
// and 128 x 96 (converters).
constexpr int LM_REGS = 128, LM_REGS_EPI = 176, LM_REGS_ISSUE = 56, LM_REGS_CONV = 96;
static_assert(LM_REGS_ISSUE + LM_REGS_CONV + 2 * LM_REGS_EPI <= 4 * LM_REGS, "the launch's registers");

// NT: tokens of a tile, 256 or, where those tiles would leave pairs idle, 128.
template <int NT, int EPI, bool SIG>
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

    if (warp < 4) {
        if constexpr (EPI != PLAIN) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LM_REGS_ISSUE));
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
        }
    } else if (warp < 8) {
        if constexpr (EPI != PLAIN) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LM_REGS_CONV));
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
    } else {
        if constexpr (EPI != PLAIN) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(LM_REGS_EPI));
        const int quad = warp & 3, half = (warp - 8) >> 2;  // channels 32 quad + lane, tokens ROWS half ..
        const uint32_t lead = cluster_addr(acc_empty, 0), at = tmem + ((uint32_t)(quad * 32) << 16) + ROWS * half;
        float* sxs = s_sx[warp - 8];
        uint32_t it = 0;
        for (int t = pair; t < P.n_tiles; t += pairs, ++it) {
            int tn, tm;
            tile_of(P, t, tn, tm);
            const int ch = tn * 256 + rank * 128 + quad * 32 + lane;
            const long long m0 = (long long)tm * NT + ROWS * half;
            const float sw = !P.sw ? 1.0f : ch < P.N ? __ldg(P.sw + ch) : 0.0f, bias = P.bias && ch < P.N ? __ldg(P.bias + ch) : 0.0f;
            for (int i = lane; i < ROWS; i += 32) sxs[i] = !P.sx ? 1.0f : m0 + i < P.M ? __ldg(P.sx + m0 + i) : 0.0f;
            __syncwarp();
            if (!wait_warp_cluster(acc_full, it & 1, abort, P.status)) break;
            tc_fence_after();
            const int cols = (int)min((long long)ROWS, P.M - m0);
            if constexpr (EPI != PLAIN) {
                const int odd = lane & 1, c0 = ch - odd;
                const float sw_o = __shfl_xor_sync(0xffffffffu, sw, 1), bias_o = __shfl_xor_sync(0xffffffffu, bias, 1);
                const float2 sw2 = odd ? make_float2(sw_o, sw) : make_float2(sw, sw_o), bias2 = odd ? make_float2(bias_o, bias) : make_float2(bias, bias_o);
                if (P.e.fast) {
                    uint32_t v[ROWS / 32][32];
#pragma unroll
                    for (int c = 0; c < ROWS / 32; ++c) tmem_ld32_nw(at + 32 * c, v[c]);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < ROWS / 32; ++c) reg_fence(v[c]);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(lead);
                    epilogue_fast<ROWS, EPI, SIG>(P, [&](int t) { return __uint_as_float(v[t / 32][t % 32]); }, sxs, sw2, bias2, c0, odd, m0, cols);
                } else {
                    for (int c = 0; c < ROWS; c += 16) {
                        uint32_t v[16];
                        tmem_ld16_nw(at + c, v);
                        tmem_wait_ld();
                        reg_fence(v);
                        epilogue_any<EPI>(P, v, sxs + c, sw2, bias2, c0, odd, m0 + c, cols - c);
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(lead);
                }
                __syncwarp();  // (the scales are read)
                continue;
            }
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

template <int NT, int EPI, bool SIG>
fxpq_status launch_many(ManyArgs& P, cudaStream_t st) {
    static bool set = false;
    const auto kernel = linear_many_kernel<NT, EPI, SIG>;
    if (!set) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LM_SMEM) != cudaSuccess) return FXPQ_ERR_CUDA;
        set = true;
    }
    const long long tn = ((long long)P.N + 255) / 256, tm = (P.M + NT - 1) / NT;
    if (tn * tm > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    P.tiles_n = (int)tn, P.tiles_m = (int)tm, P.n_tiles = (int)(tn * tm);
    P.y_pair = aligned(P.y, 4) && P.ys % 2 == 0;
    const int pairs = num_sms() / 2 > 0 ? num_sms() / 2 : 1;
    launch_pdl(kernel, dim3(2 * (unsigned)(P.n_tiles < pairs ? P.n_tiles : pairs)), dim3(LM_THREADS), LM_SMEM, st, P);
    return after_launch("linear_many");
}

template <int TOK, int EPI>
fxpq_status launch_few(LinArgs& P, cudaStream_t st) {
    static bool set = false;
    const auto kernel = linear_few_kernel<TOK, EPI>;
    if (!set) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, TOK == FLOATS ? ls_smem(LF_ROWS, 4, TOK, LF_MOST) : ls_smem(128, 4, TOK, 0)) !=
            cudaSuccess)
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
    auto smem_for = [&](int shares) { return (size_t)ls_smem(P.cols, P.stages, TOK, (P.n_kb + shares - 1) / shares); };
    c.stream = st;
    c.attrs = at;
    // As many CTAs to a reduction as run at once, with at least 1024 codes each (4096 x 4096, 64 tokens: 10.9 us with four of
    // 1024 codes, 11.9 with eight of 512), or 512 where they leave half of the SMs free (1000 x 4096, one token: 5.5 and 6.8).  Clusters are placed within a group of SMs: 16 clusters of 8 CTAs that fill an SM
    // each left one for a second round (251 x 1001 of 4090: 19.4 us, 13.3 with clusters of 4).
    int shares = 1;
    for (; shares < 8 && P.n_kb >= (tn * tm * shares * 4 <= num_sms() ? 8 : 16) * shares; shares *= 2) {
        static std::atomic<int> room[9][4];  // clusters that run at once, by tile width and size, asked for once
        const int w = P.cols / 16, l = shares == 1 ? 1 : shares == 2 ? 2 : 3;
        int n = room[w][l].load(std::memory_order_relaxed);
        if (n == 0) {
            at[1].val.clusterDim.x = 2 * shares;
            c.gridDim = dim3(2 * shares, 1024, 1);
            c.dynamicSmemBytes = smem_for(2 * shares);
            c.numAttrs = 2;
            if (cudaOccupancyMaxActiveClusters(&n, kernel, &c) != cudaSuccess || n <= 0) {
                (void)cudaGetLastError();
                n = -1;
            }
            room[w][l].store(n, std::memory_order_relaxed);
        }
        // (the query counts one CTA to an SM: it says 15 clusters of 8 where 32 of two CTAs to an SM ran at once)
        if (tn * tm > (P.cols <= 64 ? 2 * n + 2 : n)) break;
    }
    if (TOK == FLOATS)
        while (P.n_kb > LF_MOST * shares) shares *= 2;
    c.dynamicSmemBytes = smem_for(shares);
    at[1].val.clusterDim.x = shares;
    c.gridDim = dim3((unsigned)shares, (unsigned)tn, (unsigned)tm);
    c.numAttrs = shares > 1 ? 2 : 1;
    (void)cudaLaunchKernelEx(&c, kernel, P);
    return after_launch("linear_few");
}

// Rows of floats whose codes the product forms itself: few enough that every CTA reads them whole (at most 128 KB of 16-bit rows, what the
// quantizer's launch and the wait for it cost), and 8 shares of at most LF_MOST blocks.
bool float_rows_fit(int64_t M, int32_t K) { return M <= LF_ROWS && M * K <= 65536 && K <= 8 * LF_MOST * LS_KB; }

// Codes of the tokens: bytes at d_x, or fp16 at half, or formed from rows (the others are null).
template <int EPI>
fxpq_status product_few(const int8_t* d_x, const __half* half, int64_t x_stride, const float* d_sx, const int8_t* d_w, int64_t w_stride,
                        const float* d_sw, const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type, void* d_y, int64_t y_stride,
                        cudaStream_t st, const Epi& e = {}, const FloatRows* rows = nullptr, bool early = false) {
    LinArgs P;
    P.e = e, P.early = early;
    const int64_t tiles = (M + 127) / 128;  // M's equal parts
    P.rows = (int)((M + tiles - 1) / tiles);
    P.cols = (P.rows + 15) / 16 * 16;
    P.n_kb = (K + LS_KB - 1) / LS_KB;
    P.w_rows = N % 128 ? N % 128 : 128;
    P.y_four = aligned(d_y, 4 * ftype_bytes(y_type)) && y_stride % 4 == 0;
    if (K > 0) {
        if (!encode_rows(&P.tw, d_w, N, K, w_stride, 128)) return FXPQ_ERR_CUDA;
        if (!rows && !(half ? encode_half_rows(&P.tx, half, M, K, x_stride, P.rows) : encode_rows(&P.tx, d_x, M, K, x_stride, P.rows)))
            return FXPQ_ERR_CUDA;
        P.tw2 = P.tw;
        if (P.w_rows < 128 && !encode_rows(&P.tw2, d_w, N, K, w_stride, P.w_rows)) return FXPQ_ERR_CUDA;
    }
    P.sx = d_sx, P.sw = d_sw, P.bias = d_bias, P.y = d_y, P.ys = y_stride, P.M = M, P.N = N, P.y_type = y_type;
    P.status = status_ptr();
    if constexpr (EPI != PLAIN) {
        const int type = ftype_bytes(y_type), each = EPI == GATED ? 2 : 4, kept = e.pre_f32 ? 4 : 2;
        P.e.vec = (aligned(d_y, each * type) && y_stride % each == 0 ? 1 : 0) | (aligned(e.res, 4 * type) && e.res_stride % 4 == 0 ? 2 : 0) |
                  (aligned(e.pre, 4 * kept) && N % 4 == 0 ? 4 : 0);
        if (rows) {
            P.f = *rows;
            return launch_few<FLOATS, EPI>(P, st);
        }
        return launch_few<HALVES, EPI>(P, st);
    } else {
        return half ? launch_few<HALVES, PLAIN>(P, st) : launch_few<BYTES, PLAIN>(P, st);
    }
}

template <int EPI>
fxpq_status product_many(const __half* half, size_t pitch, const float* d_sx, const int8_t* d_w, int64_t w_stride, const float* d_sw,
                         const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type, void* d_y, int64_t y_stride, cudaStream_t st,
                         const Epi& e = {}) {
    ManyArgs P;
    P.e = e;
    // Tiles of 256 tokens, or of 128 where their rounds over the pairs take less time.  A round of the narrow ones takes two
    // thirds of the wide ones' (8192 x 8192 of 4096: 13.2 and 20.1 us; every tile expands 256 channels' weights).
    const int64_t pairs = num_sms() / 2 > 0 ? num_sms() / 2 : 1, tn = ((int64_t)N + 255) / 256;
    const auto rounds = [&](int64_t nt) { return (tn * ((M + nt - 1) / nt) + pairs - 1) / pairs; };
    const int nt = 2 * rounds(128) < 3 * rounds(256) ? 128 : 256;
    if (!encode_rows(&P.tw, d_w, N, K, w_stride, 128) || !encode_half_rows(&P.tx, half, M, K, (long long)pitch, nt / 2)) return FXPQ_ERR_CUDA;
    P.sx = d_sx, P.sw = d_sw, P.bias = d_bias, P.y = d_y, P.ys = y_stride, P.M = M, P.N = N, P.K = K, P.y_type = y_type;
    P.status = status_ptr();
    if constexpr (EPI != PLAIN) {
        const bool sig = e.act == FXPQ_ACT_SILU || e.act == FXPQ_ACT_GELU_TANH, gated = EPI == GATED;
        P.e.fast = y_type != FXPQ_FT_F32 && aligned(d_y, 4) && y_stride % 2 == 0 && N % (gated ? 4 : 2) == 0 && (gated ? sig : e.act != FXPQ_ACT_GELU) &&
                   aligned(e.res, 4) && e.res_stride % 2 == 0 && (!e.pre || (!e.pre_f32 && aligned(e.pre, 4)));
        if (gated || sig) return nt == 128 ? launch_many<128, EPI, true>(P, st) : launch_many<256, EPI, true>(P, st);
    }
    if constexpr (EPI != GATED) return nt == 128 ? launch_many<128, EPI, false>(P, st) : launch_many<256, EPI, false>(P, st);
    return FXPQ_ERR_UNSUPPORTED;
}
}  // namespace
}  // namespace llm
}  // namespace fxpq
