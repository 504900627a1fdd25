#pragma once
// fxpq_layer_few.cuh -- products of few rows with 8-bit weights, and what stands around them.
#include "fxpq_linear.cuh"

namespace fxpq {
namespace llm {
namespace {

// Rows as they come, for products that form their codes themselves.
struct FloatRows {
    const void* x;
    long long x_stride;
    int x_type, x_vec, K;
    float* sx;  // the rows' scales, or null
    RowNorm norm;
};

struct FewArgs {
    // weights' codes as [N][K] bytes in boxes of 128 codes x 128 rows (tw), or x the rows that the last tile has (tw2: a box is
    // slow where it lies outside the tensor); rows as fp16 in 64 x `rows`
    CUtensorMap tw, tw2, tx;
    const float *sx, *sw, *bias;  // null: ones, ones, zeros
    void* y;
    long long ys, M;
    int N, y_type, n_kb;
    int rows, cols;  // tokens of a tile, and rounded up to 16, at most 128 (the columns past `rows` hold whatever the stage does)
    int w_rows;      // channels of the last tile
    int stages;
    int early;       // the kernel before is this call's quantizer, which lets this one begin: weights may be read before its codes exist
    int* status;
    Epi e;
    FloatRows f;
};

// ------------------------------------------------------------------ few tokens
// y^T = w x^T on tcgen05 (kind::f16: the 8-bit kind does not exist on sm_103a; codes are exact in fp16, their products in fp32): 128
// output channels on the accumulator's lanes, up to 128 tokens on its columns.  The weights are the traffic.  They
// arrive as codes (TMA, 128 x 128 bytes a block) and go through registers into tensor memory as the fp16 A operand,
// so that their shared-memory traffic stays at two bytes a code.
//   warp 0   copies;   warp 1   tensor memory, products;   warps 4-7, 8-11   converters (blocks in turn), then the epilogue.
// The reduction is shared by the CTAs of a cluster, whose fp32 sums meet through distributed shared memory: one launch, a
// fixed order.  Up to 64 tokens two CTAs fit an SM.
constexpr int LF_THREADS = 384;

// How the rows come: as fp16 (codes, or a gradient's), or as rows of floats (up to 16), whose codes every CTA forms for its share of the
// reduction.
enum { HALVES, FLOATS };
// A half block of their codes has whole groups of 8 rows; the products read groups of 16: what follows (the 1 KB behind the last) stands in for
// columns that nobody reads.
constexpr int LF_ROWS = 16, LF_MOST = 32;  // (blocks of a share)
__host__ __device__ inline int lf_half(int rows) { return (rows + 7) / 8 * 8 * 128; }
constexpr int LF_SMEM = 220 * 1024;

// Operands of weights in tensor memory, one more (or two) than there are groups that form them: none waits for the product of its last.
__host__ __device__ inline int lf_operands(int cols) { return cols > 64 ? 4 : 3; }

// floats: stages of weights alone, and all of the share's codes
__host__ __device__ inline int lf_smem(int rows, int cols, int stages, int tok, int blocks) {
    const int ring = tok == HALVES ? stages * (LS_A + cols * LS_KB * 2) : stages * LS_A + blocks * 2 * lf_half(rows) + 1024;
    const int sums = cols * 128 * 4;
    return 1024 + (ring > sums ? ring : sums);
}

// Codes of up to 16 rows of floats by 256 threads (8 warps): every row's scale from the whole row, then the fp16 codes of n_kb blocks
// from block kb0 on into shared memory, as the products read them.  The same fp32 steps as the token quantizer's.
struct RowSpace {
    uint32_t top[LF_ROWS];  // [row][part]
    float sum[LF_ROWS], inv[LF_ROWS], sx[LF_ROWS];
};
template <typename T, bool NORM>
__device__ __forceinline__ void own_codes(const FloatRows& F, int M, int kb0, int n_kb, unsigned char* blocks, RowSpace& S, int t, bool first, int* status) {
    const T* x = static_cast<const T*>(F.x);
    const int warp = t >> 5, lane = t & 31, K = F.K, groups = K / 8;
    const int log_parts = M <= 1 ? 3 : M <= 2 ? 2 : M <= 4 ? 1 : 0, parts = 1 << log_parts, step = 32 * parts;  // warps of a row
    const auto join = []() { asm volatile("bar.sync 1, 256;" ::: "memory"); };
    auto eight = [&](const T* row, int k, float (&v)[8], float (&w)[8]) {
        load_f32<8>(row + k, F.x_vec, v);
        if constexpr (NORM) load_f32<8>(F.norm.weight + k, F.norm.vec, w);
    };
    for (int u = warp; u < M * parts; u += 8) {
        const int m = u >> log_parts, p = u & (parts - 1);
        const T* row = x + m * F.x_stride;
        RowScan<NORM> scan;
#pragma unroll 4
        for (int g = p * 32 + lane; g < groups; g += step) {
            float v[8], w[8];
            eight(row, 8 * g, v, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) scan.see(v[e], w[e]);
        }
        const int k = 8 * groups + lane;
        if (p == 0 && k < K) scan.see(to_f32(row[k]), NORM ? __ldg(F.norm.weight + k) : 1.0f);
        scan.meet();
        if (lane == 0) S.top[u] = scan.top, S.sum[u] = scan.sum;
    }
    join();
    for (int m = warp; m < M; m += 8) {
        RowScan<NORM> scan;
        for (int p = 0; p < parts; ++p) scan.join(S.top[m * parts + p], NORM ? S.sum[m * parts + p] : 0.0f);
        float inv = scan.inverse(), sx;
        if (scan.odd())
            careful_row(x + m * F.x_stride, K, F.norm.weight, F.norm.eps, inv, sx, first ? status : nullptr);
        else
            sx = scan.scale(K, F.norm.eps);
        if (lane == 0) {
            S.inv[m] = inv, S.sx[m] = sx;
            if (F.sx && first) F.sx[m] = sx;
        }
    }
    join();
    const int chunks = n_kb * (LS_KB / 8), half = lf_half(M);
    for (int u = warp; u < M * parts; u += 8) {
        const int m = u >> log_parts;
        const T* row = x + m * F.x_stride;
        const float inv = S.inv[m];
        unsigned char* to = blocks + m * 128;
#pragma unroll 2
        for (int c = (u & (parts - 1)) * 32 + lane; c < chunks; c += step) {
            const int k = kb0 * LS_KB + 8 * c;
            float v[8], w[8];
            if (k + 8 <= K) {
                eight(row, k, v, w);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = k + e < K ? to_f32(row[k + e]) : 0.0f, w[e] = NORM && k + e < K ? __ldg(F.norm.weight + k + e) : 1.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = scaled_code(NORM ? __fmul_rn(v[e], w[e]) : v[e], inv);
            *reinterpret_cast<uint4*>(to + (c >> 3) * half + (((c & 7) ^ (m & 7)) << 4)) =
                make_uint4(f32_codes_f16x2(v[0], v[1]), f32_codes_f16x2(v[2], v[3]), f32_codes_f16x2(v[4], v[5]), f32_codes_f16x2(v[6], v[7]));
        }
    }
}
template <typename T>
__device__ __forceinline__ void own_codes_of(const FloatRows& F, int M, int kb0, int n_kb, unsigned char* blocks, RowSpace& S, int t, bool first, int* status) {
    if (F.norm.weight)
        own_codes<T, true>(F, M, kb0, n_kb, blocks, S, t, first, status);
    else
        own_codes<T, false>(F, M, kb0, n_kb, blocks, S, t, first, status);
}

// Four residuals as they lie in memory.
struct Residual {
    uint32_t r[4];
    __device__ __forceinline__ void load(const void* p, int type, long long at, int left, bool whole) {
        if (type == FXPQ_FT_F32) {
            const uint32_t* q = static_cast<const uint32_t*>(p) + at;
            if (whole) {
                const uint4 w = *reinterpret_cast<const uint4*>(q);
                r[0] = w.x, r[1] = w.y, r[2] = w.z, r[3] = w.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < left) r[e] = q[e];
            }
        } else {
            const unsigned short* q = static_cast<const unsigned short*>(p) + at;
            if (whole) {
                const uint2 w = *reinterpret_cast<const uint2*>(q);
                r[0] = w.x, r[1] = w.y;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < left) r[e] = q[e];
            }
        }
    }
    __device__ __forceinline__ float4 values(int type, bool whole) const {
        if (type == FXPQ_FT_F32) return make_float4(__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[2]), __uint_as_float(r[3]));
        const float2 a = pair_f32(whole ? r[0] : __byte_perm(r[0], r[1], 0x5410), type), b = pair_f32(whole ? r[1] : __byte_perm(r[2], r[3], 0x5410), type);
        return make_float4(a.x, a.y, b.x, b.y);
    }
};

// What follows the sums a of token m and channels ch .. ch + 3, of which P.N may leave some out.  s, sw, bias: their scales and biases.
template <int EPI, typename Args>
__device__ __forceinline__ void finish_four(const Args& P, const Epi& e, long long m, int ch, float4 a, float s, const float (&sw)[4], const float (&bias)[4],
                                            const Residual& r, bool whole) {
    const int left = P.N - ch;
    float v[4] = {fmaf(a.x * s, sw[0], bias[0]), fmaf(a.y * s, sw[1], bias[1]), fmaf(a.z * s, sw[2], bias[2]), fmaf(a.w * s, sw[3], bias[3])};
    if (e.pre) {
        const float k = e.pre_f32 ? 1.0f : e.pre_scale, keep[4] = {a.x * k, a.y * k, a.z * k, a.w * k};
        store_some<4>(e.pre, e.pre_f32 ? FXPQ_FT_F32 : FXPQ_FT_F16, m * e.pre_stride + ch, keep, left, e.vec & 4);
    }
    if constexpr (EPI == GATED) {
        const float y[2] = {activate(v[0], e.act) * v[1], activate(v[2], e.act) * v[3]};
        store_some<2>(P.y, P.y_type, m * P.ys + ch / 2, y, left / 2, e.vec & 1);
    } else {
        if (e.act != FXPQ_ACT_NONE)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = activate(v[i], e.act);
        if (e.res) {
            const float4 f = r.values(P.y_type, whole);
            v[0] += f.x, v[1] += f.y, v[2] += f.z, v[3] += f.w;
        }
        store_some<4>(P.y, P.y_type, m * P.ys + ch, v, left, e.vec & 1);
    }
}
// Which of outputs, residuals and kept sums lie in aligned accesses of four channels (gated outputs: of two).
template <int EPI>
inline int fours(const Epi& e, int y_type, const void* y, int64_t y_stride) {
    const int type = ftype_bytes(y_type), each = EPI == GATED ? 2 : 4, kept = e.pre_f32 ? 4 : 2;
    return (aligned(y, each * type) && y_stride % each == 0 ? 1 : 0) | (aligned(e.res, 4 * type) && e.res_stride % 4 == 0 ? 2 : 0) |
           (aligned(e.pre, 4 * kept) && e.pre_stride % 4 == 0 ? 4 : 0);
}

// The sums that pairs of CTAs left in memory, added over a tile's shares in their order, and what follows them: a warp has four tokens of
// 128 channels (PARTS: of both their sums, half a tile apart).
template <int EPI>
__global__ void __launch_bounds__(256) finish_kernel(const __grid_constant__ ManyArgs P, int nt) {
    pdl_wait();
    constexpr int EACH = 4, AFTER = EPI == PARTS ? LAYER : EPI;
    const int tokens = EPI == PARTS ? nt / 2 : nt;  // of a tile
    const int tile = blockIdx.x >> 1, rank = blockIdx.x & 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int tn, tm;
    tile_of(P, P.whole + tile, tn, tm);
    const int ch = tn * 256 + rank * 128 + 4 * lane, left = P.N - ch, c0 = (blockIdx.y * 8 + warp) * EACH;
    const long long m0 = (long long)tm * tokens + c0;
    const int count = (int)min((long long)EACH, P.M - m0);
    if (left <= 0 || count <= 0) return;
    const bool whole = (P.e.vec & 2) && left >= 4;
    float4 a[EACH], b[EPI == PARTS ? EACH : 1];  // (PARTS: the second parts' sums)
    Residual r[EACH];
    float sw[4], bias[4], sx[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        a[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if constexpr (EPI == PARTS) b[i] = a[i];
        if (i >= count) continue;
        if (EPI == LAYER && P.e.res) r[i].load(P.e.res, P.y_type, (m0 + i) * P.e.res_stride + ch, left, whole);
        sx[i] = P.sx ? __ldg(P.sx + m0 + i) : 1.0f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sw[e] = !P.sw ? 1.0f : e < left ? __ldg(P.sw + ch + e) : 0.0f;
        bias[e] = P.bias && e < left ? __ldg(P.bias + ch + e) : 0.0f;
    }
    const float* part = P.part + (((long long)tile * 2 + rank) * nt + c0) * 128 + 4 * lane;
#pragma unroll 2
    for (int s = 0; s < P.shares; ++s, part += (long long)(P.n_tiles - P.whole) * 2 * nt * 128) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (i >= count) continue;
            const float4 f = *reinterpret_cast<const float4*>(part + i * 128);
            a[i].x += f.x, a[i].y += f.y, a[i].z += f.z, a[i].w += f.w;
            if constexpr (EPI == PARTS) {
                const float4 g = *reinterpret_cast<const float4*>(part + (tokens + i) * 128);
                b[i].x += g.x, b[i].y += g.y, b[i].z += g.z, b[i].w += g.w;
            }
        }
    }
    if constexpr (EPI == PARTS) {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            a[i] = make_float4(fmaf(a[i].x, PART, b[i].x), fmaf(a[i].y, PART, b[i].y), fmaf(a[i].z, PART, b[i].z), fmaf(a[i].w, PART, b[i].w));
    }
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
        finish_four<AFTER>(P, P.e, m0 + i, ch, a[0], sx[0], sw, bias, r[0], whole);
#pragma unroll
        for (int j = 0; j + 1 < EACH; ++j) a[j] = a[j + 1], sx[j] = sx[j + 1], r[j] = r[j + 1];
    }
}

// A place in a ring and the parity of its phase, without divisions (four of them took a third of a block's time).
struct Turn {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int by, int size) {  // by <= size
        at += by;
        if (at >= size) at -= size, phase ^= 1;
    }
};

template <int TOK, int EPI>
__global__ void __launch_bounds__(LF_THREADS, 2) layer_few_kernel(const __grid_constant__ FewArgs P) {
    using namespace tc;
    constexpr bool HALF = TOK == HALVES;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    __shared__ __align__(8) uint64_t bars[8 + 8 + 4 + 4 + 1 + 1];
    __shared__ int abort_flag;
    __shared__ std::conditional_t<TOK == FLOATS, RowSpace, char> rows_space;
    __shared__ float s_sx[HALF ? 128 : 1];
    __shared__ uint32_t tmem_slot;
    volatile int* abort = &abort_flag;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, ST = P.stages, cols = P.cols;
    const uint32_t raw_full = smem_u32(bars), raw_empty = raw_full + 8 * 8, conv_full = raw_empty + 8 * 8, conv_empty = conv_full + 4 * 8,
                   done = conv_empty + 4 * 8, tok_full = done + 8;
    const int NB = lf_operands(cols), columns = cols > 64 ? 512 : 256, acc_columns = cols > 64 ? 128 : 64;
    const int raw_bytes = HALF ? LS_A + cols * LS_KB * 2 : LS_A;
    const uint32_t raw0 = smem_u32(smem), conv0 = raw0 + ST * raw_bytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(raw_full + 8 * i, 1);
            mbar_init(raw_empty + 8 * i, HALF ? 1 : 4);  // the products' completion, or the converting group's warps
        }
        for (int i = 0; i < NB; ++i) {
            mbar_init(conv_full + 8 * i, 4);
            mbar_init(conv_empty + 8 * i, 1);
        }
        mbar_init(done, 1);
        if (TOK == FLOATS) mbar_init(tok_full, 8);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (P.n_kb) {
            prefetch_tmap(blockIdx.y == gridDim.y - 1 ? &P.tw2 : &P.tw);
            if (HALF) prefetch_tmap(&P.tx);
        }
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(columns));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    const int rank = blockIdx.x, shares = gridDim.x, n0 = blockIdx.y * 128;
    const long long m0 = (long long)blockIdx.z * P.rows;
    const int kb0 = (int)((long long)P.n_kb * rank / shares), n_kb = (int)((long long)P.n_kb * (rank + 1) / shares) - kb0;
    const bool last = blockIdx.y == gridDim.y - 1;
    const CUtensorMap* tw = last ? &P.tw2 : &P.tw;
    const uint32_t bytes = (uint32_t)((last ? P.w_rows : 128) * LS_KB + (HALF ? P.rows * LS_KB * 2 : 0));
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
    const uint32_t tmem = tmem_slot, tmem_a = tmem + acc_columns;

    if (HALF && (warp == 2 || warp == 3))  // the rows' scales, for the end
        for (int c = threadIdx.x - 64; c < P.rows; c += 64) s_sx[c] = !P.sx ? 1.0f : m0 + c < P.M ? __ldg(P.sx + m0 + c) : 0.0f;
    if (warp == 0) {
        int i = 0;
        Turn s;
        for (; i < n_kb; ++i, s.next(1, ST)) {
            if (!wait_warp(raw_empty + 8 * s.at, s.phase ^ 1, abort, P.status)) break;
            const uint32_t bar = raw_full + 8 * s.at, dst = raw0 + s.at * raw_bytes;
            if (i >= early) {
                mbar_arrive_expect_tx(bar, bytes);
                tma_load_2d(dst, tw, (kb0 + i) * LS_KB, n0, bar);
            }
            if (HALF) tma_load_2d(dst + LS_A, &P.tx, (kb0 + i) * LS_KB, (int)m0, bar);
            if (HALF) tma_load_2d(dst + LS_A + cols * 128, &P.tx, (kb0 + i) * LS_KB + 64, (int)m0, bar);
        }
        for (int j = max(0, i - ST); j < i; ++j) {  // every copy has landed before this CTA's memory is used again
            drain_warp(raw_full + 8 * (j % ST), (j / ST) & 1);
        }
    } else if (warp == 1) {
        const uint32_t idesc = make_idesc(128, cols);
        const uint64_t bdesc = make_sdesc(HALF ? raw0 : conv0);
        const int half_bytes = TOK == FLOATS ? lf_half(P.rows) : cols * 128;
        if (TOK == FLOATS && n_kb > 0) wait_warp(tok_full, 0, abort, P.status);
        Turn c, s;
        for (int i = 0; i < n_kb; ++i, c.next(1, NB), s.next(1, ST)) {
            if (!wait_warp(conv_full + 8 * c.at, c.phase, abort, P.status)) break;
            if (HALF && !wait_warp(raw_full + 8 * s.at, s.phase, abort, P.status)) break;
            tc_fence_after();
            const uint64_t bd = bdesc + (uint64_t)((HALF ? s.at * raw_bytes + LS_A : i * 2 * half_bytes) >> 4);
#pragma unroll
            for (int kk = 0; kk < LS_KB / 16; ++kk)
                tc_mma_ta(tmem, tmem_a + 64 * c.at + 8 * kk, bd + (uint64_t)(((kk >> 2) * half_bytes) >> 4) + 2 * (kk & 3), idesc, i > 0 || kk > 0);
            tc_commit(conv_empty + 8 * c.at);
            if (HALF) tc_commit(raw_empty + 8 * s.at);
        }
        tc_commit(done);
        drain_warp(done, 0);
    } else if (warp >= 4) {
        const int grp = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane;
        if constexpr (TOK == FLOATS) {
            const int M = (int)P.M, tt = threadIdx.x - 128;
            const bool first = rank == 0 && blockIdx.y == 0;
            if (P.f.x_type == FXPQ_FT_F32)
                own_codes_of<float>(P.f, M, kb0, n_kb, smem + ST * raw_bytes, rows_space, tt, first, P.status);
            else if (P.f.x_type == FXPQ_FT_F16)
                own_codes_of<__half>(P.f, M, kb0, n_kb, smem + ST * raw_bytes, rows_space, tt, first, P.status);
            else
                own_codes_of<__nv_bfloat16>(P.f, M, kb0, n_kb, smem + ST * raw_bytes, rows_space, tt, first, P.status);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(tok_full);
        }
        Turn s, c;
        s.next(grp, ST), c.next(grp, NB);
        for (int i = grp; i < n_kb; i += 2, s.next(2, ST), c.next(2, NB)) {
            // In this order: with an odd number of stages the groups take turns on one, and a parity wait on raw_full
            // tells block i from block i - ST of the other group only once that one has landed.  Block i - NB's products
            // are complete here, so all before them are, and their blocks were read (NB is at most ST).  The groups take turns on the
            // operands too, but block i - 2 had to see block i - 2 - NB complete, so no wait here is two phases behind.
            if (!wait_warp(conv_empty + 8 * c.at, c.phase ^ 1, abort, P.status)) break;
            if (!wait_warp(raw_full + 8 * s.at, s.phase, abort, P.status)) break;
            tc_fence_after();
            const unsigned char* ra = smem + s.at * raw_bytes;
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
                tmem_st32_nw(tmem_a + ((uint32_t)(quad * 32) << 16) + 64 * c.at + 32 * hf, r);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (!HALF) mbar_arrive(raw_empty + 8 * s.at);
                mbar_arrive(conv_full + 8 * c.at);
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
    // ---- four channels of one token per lane, a token per warp and step, summed over the cluster.  What comes from memory is asked for
    // before the CTA and the cluster meet, residuals four tokens ahead and as they are: converted where they were loaded, every token
    // waited for its own (64 x 32768: 2000 clocks a token and warp).
    constexpr int TOKENS = LF_THREADS / 32, AHEAD = 4;
    const int mine = (int)min((long long)P.rows, P.M - m0), c_lo = mine * rank / shares, c_hi = mine * (rank + 1) / shares;
    const int ch = n0 + 4 * lane, left = P.N - ch;
    const bool whole = (P.e.vec & 2) && left >= 4;
    float sw[4], bias[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sw[e] = !P.sw ? 1.0f : e < left ? __ldg(P.sw + ch + e) : 0.0f;
        bias[e] = P.bias && e < left ? __ldg(P.bias + ch + e) : 0.0f;
    }
    auto residual = [&](int c) {
        Residual r;
        if (EPI == LAYER && P.e.res && c < c_hi) r.load(P.e.res, P.y_type, (m0 + c) * P.e.res_stride + ch, left, whole);
        return r;
    };
    Residual queue[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) queue[i] = residual(c_lo + warp + i * TOKENS);
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
    }
    if (shares > 1) cluster_sync();
    for (int c = c_lo + warp; c < c_hi; c += TOKENS) {
        const Residual r = queue[0];
#pragma unroll
        for (int i = 0; i < AHEAD - 1; ++i) queue[i] = queue[i + 1];
        queue[AHEAD - 1] = residual(c + AHEAD * TOKENS);
        const uint32_t at = (uint32_t)(c * 32 + lane) * 16;
        float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (shares == 1) {
            a = *reinterpret_cast<const float4*>(smem + at);
        } else {
            float4 part[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < shares) part[i] = ld_cluster_f4(cluster_addr(raw0 + at, i));
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < shares) a.x += part[i].x, a.y += part[i].y, a.z += part[i].z, a.w += part[i].w;
        }
        float s = 1.0f;
        if constexpr (HALF)
            s = s_sx[c];
        else
            s = rows_space.sx[c];
        finish_four<EPI>(P, P.e, m0 + c, ch, a, s, sw, bias, r, whole);
    }
    if (shares > 1) cluster_sync();  // (the others have read this CTA's sums)
}

template <int TOK, int EPI>
fxpq_status launch_few(FewArgs& P, cudaStream_t st) {
    const auto kernel = layer_few_kernel<TOK, EPI>;
    static std::atomic<uint64_t> set{0};
    if (!allow_smem(kernel, TOK == FLOATS ? LF_SMEM : lf_smem(128, 128, 4, TOK, 0), set)) return FXPQ_ERR_CUDA;
    const long long tn = (P.N + 127) / 128, tm = (P.M + P.rows - 1) / P.rows;
    if (tn > 65535 || tm > 65535) return FXPQ_ERR_UNSUPPORTED;
    P.stages = P.cols <= 32 || P.cols > 64 ? 4 : 3;
    // Floats: two CTAs to an SM if their shares' codes leave room for three or four stages, else as many stages as fit one.  (Shares sized for
    // two CTAs to an SM of which only one fits take two rounds: 1 x 4096 of 16384 39 us.)
    auto two_fit = [&](int shares) {
        if (TOK == HALVES) return P.cols <= 64;
        const int blocks = (P.n_kb + shares - 1) / shares;
        for (P.stages = 4; P.stages >= 3; --P.stages)
            if (lf_smem(P.rows, P.cols, P.stages, TOK, blocks) <= LF_SMEM / 2) return true;
        for (P.stages = 8; P.stages > 4 && lf_smem(P.rows, P.cols, P.stages, TOK, blocks) > LF_SMEM;) --P.stages;
        return false;
    };
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.blockDim = dim3(LF_THREADS);
    auto smem_for = [&](int shares) { return (size_t)lf_smem(P.rows, P.cols, P.stages, TOK, (P.n_kb + shares - 1) / shares); };
    c.stream = st;
    c.attrs = at;
    // As many CTAs to a reduction as run at once, with at least 1024 codes each (4096 x 4096, 64 tokens: 10.9 us with four of
    // 1024 codes, 11.9 with eight of 512), or 512 where they leave half of the SMs free (1000 x 4096, one token: 5.5 and 6.8).  Clusters are placed within a group of SMs: 16 clusters of 8 CTAs that fill an SM
    // each left one for a second round (251 x 1001 of 4090: 19.4 us, 13.3 with clusters of 4).
    int shares = 1;
    for (; shares < 8 && P.n_kb >= (tn * tm * shares * 4 <= num_sms() ? 8 : 16) * shares; shares *= 2) {
        const int blocks = (P.n_kb + 2 * shares - 1) / (2 * shares), l = shares == 1 ? 1 : shares == 2 ? 2 : 3;
        if (TOK == FLOATS && blocks > LF_MOST) continue;  // (no CTA holds their codes)
        // By what their shared memory goes by: tile width, or floats' groups of rows and blocks of a share; and by their size.
        static std::atomic<int> room[TOK == FLOATS ? 2 * (LF_MOST + 1) : 9][4][DEVICES];
        const int w = TOK == FLOATS ? (P.rows > 8 ? LF_MOST + 1 : 0) + blocks : P.cols / 16;
        const bool two = two_fit(2 * shares);
        at[1].val.clusterDim.x = 2 * shares;
        c.gridDim = dim3(2 * shares, 1024, 1);
        c.dynamicSmemBytes = smem_for(2 * shares);
        c.numAttrs = 2;
        const int n = clusters_at_once(kernel, c, room[w][l]);
        // (the query counts one CTA to an SM: it says 15 clusters of 8 where 32 of two CTAs to an SM ran at once)
        if (tn * tm > (two ? 2 * n + 2 : n)) break;
    }
    if (TOK == FLOATS)
        while (P.n_kb > LF_MOST * shares) shares *= 2;
    (void)two_fit(shares);
    c.dynamicSmemBytes = smem_for(shares);
    at[1].val.clusterDim.x = shares;
    c.gridDim = dim3((unsigned)shares, (unsigned)tn, (unsigned)tm);
    c.numAttrs = shares > 1 ? 2 : 1;
    (void)cudaLaunchKernelEx(&c, kernel, P);
    return after_launch("linear_few");
}

// Rows of floats whose codes the product forms itself: few enough that every CTA may read them whole, and 8 shares of at most LF_MOST
// blocks.  On the GPU that takes as long as quantizer and product, or a little longer (4096 channels, 4096 inputs, 1, 4 and 8 rows: 9.7, 11.7
// and 13.0 us, as two launches 10.0, 12.6 and 12.6; 16 rows of 1024 10.2 and 7.6, of 3640 22 and 12); the host saves a launch and
// the codes' memory, 9 of 20 us.
bool float_rows_fit(int64_t M, int32_t K) { return M <= LF_ROWS && M * K <= (M <= 8 ? 32768 : 16384) && K <= 8 * LF_MOST * LS_KB; }

// Rows as fp16 at half, or formed from floats.
template <int EPI>
fxpq_status few_product(const __half* half, int64_t x_stride, const float* d_sx, const int8_t* d_w, int64_t w_stride,
                        const float* d_sw, const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type, void* d_y, int64_t y_stride,
                        cudaStream_t st, const Epi& e = {}, const FloatRows* rows = nullptr, bool early = false) {
    FewArgs P;
    P.e = e, P.early = early;
    const int64_t tiles = (M + 127) / 128;  // M's equal parts
    P.rows = (int)((M + tiles - 1) / tiles);
    P.cols = (P.rows + 15) / 16 * 16;
    P.n_kb = (K + LS_KB - 1) / LS_KB;
    P.w_rows = N % 128 ? N % 128 : 128;
    if (K > 0) {
        if (!encode_rows(&P.tw, d_w, N, K, w_stride, 128)) return FXPQ_ERR_CUDA;
        if (!rows && !encode_half_rows(&P.tx, half, M, K, x_stride, P.rows))
            return FXPQ_ERR_CUDA;
        P.tw2 = P.tw;
        if (P.w_rows < 128 && !encode_rows(&P.tw2, d_w, N, K, w_stride, P.w_rows)) return FXPQ_ERR_CUDA;
    }
    P.sx = d_sx, P.sw = d_sw, P.bias = d_bias, P.y = d_y, P.ys = y_stride, P.M = M, P.N = N, P.y_type = y_type;
    P.status = status_ptr();
    P.e.vec = fours<EPI>(e, y_type, d_y, y_stride);
    if (!rows) return launch_few<HALVES, EPI>(P, st);
    P.f = *rows;
    return launch_few<FLOATS, EPI>(P, st);
}

}  // namespace
}  // namespace llm
}  // namespace fxpq
