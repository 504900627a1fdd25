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
// channels' activation times value.  Both of the latter may keep the sums (scaled, in fp16, or as they are) for a gradient.  PARTS: the rows
// are a gradient's, in two parts (GradRows): y = (PART sum of the first + sum of the second) * sx.
enum { PLAIN, LAYER, GATED, PARTS };
struct Epi {
    const void* res;
    long long res_stride;
    void* pre;  // rows pre_stride apart
    float pre_scale;
    int pre_f32, act;
    long long pre_stride;
    int vec;   // outputs, residuals and kept sums (bits 1, 2, 4) of four channels (few rows; gated outputs two), or of two, in aligned accesses each
    int fast;  // many: 16-bit outputs, pairs of everything aligned
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
__device__ __forceinline__ float2 pair_f32(uint32_t w, int type) {
    return type == FXPQ_FT_F16 ? __half22float2(*reinterpret_cast<const __half2*>(&w)) : __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
}

constexpr int LS_KB = 128, LS_A = 128 * LS_KB;  // codes of a block of the reduction, bytes of a block of 128 channels

// ------------------------------------------------------------------ many tokens
// The same product, bound by the tensor pipe: pairs of CTAs share tiles of 256 channels x 256 tokens (cta_group::2), so
// that a CTA reads only half of the tokens' operand from its shared memory.  Per 64 codes of the reduction (512 cycles of
// products) it moves 8 KB of weight codes in and out and 16 KB of tokens in and once through the tensor core: 384 cycles
// of shared memory, where one CTA alone would need 640, and both operands as fp16 in shared memory 512.  The tokens arrive
// as fp16 codes (written so by the quantizer, or expanded before), the weights as bytes, expanded into tensor memory.
//   warp 0  weights' copies;  1  tokens' copies;  2  tensor memory, products (CTA 0);  4-7  converters;  8-15  epilogue (layers': 8-23).
// The accumulators fill half of tensor memory, the weights' four stages the other half.  The epilogue scales and packs the
// sums into registers first, so that the next tile's products begin while it still stores.
constexpr int LM_RAW = 3, LM_B = 8, LM_A = 4;
constexpr int LM_SMEM = 1024 + LM_RAW * LS_A + LM_B * 128 * 128;

struct ManyArgs {
    CUtensorMap tw, tx;  // weights' codes (boxes of 128 codes x 128 rows), tokens' fp16 codes (64 x 128)
    const float *sx, *sw, *bias;
    void* y;
    long long ys, M;
    int N, K, y_type, y_pair;  // y_pair: two 16-bit outputs in one aligned access
    int tiles_n, tiles_m, n_tiles;
    // Tiles from `whole` on are left to finish_kernel: their reductions are split into shares, work of pairs of their own, whose sums go
    // to `part` as they are, [share][tile - whole][CTA][token][128 channels].
    int whole, shares;
    float* part;
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

// Activations by their form: at most a cut, z times a sigmoid, z times the normal distribution's integral.
enum { CUT, SIGMOID, NORMAL };
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

// A warp's residuals, two channels of ROWS / 2 tokens a lane: the first asked for before the sums are there, the others two steps ahead.  (Asked
// for a step ahead, a tile's epilogue took 21 thousand clocks with them and 8 without; y may be the residual, so the compiler keeps
// every load behind the stores before it.)
template <int ROWS>
struct Residuals {
    const char* at;  // token odd's two channels
    long long step;  // two tokens, in bytes
    static constexpr int HELD = 8;
    uint32_t r[HELD];
    __device__ __forceinline__ void ask(int i, int cols) {  // of token 2 i + odd
        uint32_t w = 0;
        if (2 * i < cols) w = *reinterpret_cast<const uint32_t*>(at + i * step);
        r[i % HELD] = w;
    }
};

// The epilogue of a warp's 32 channels and ROWS tokens for LAYER and GATED: 16-bit outputs in aligned pairs.  Everything goes by pairs: two
// lanes exchange sums so that each holds two channels of one token.  All sums are in registers, and the accumulators have been given back
// before anything is computed, so that the next tile's products run meanwhile.  16 warps (of 96 registers) have half the code and
// twice the loads under way of 8 (of 192): 8071 x 2304 of 1024 with norm and tanh GELU 68 and 52 us, 2000 x 2 x 4096 of 1024 46 and 37.
template <int ROWS, int EPI, int FORM, typename Sum>
__device__ __forceinline__ void epilogue_fast(const ManyArgs& P, Sum&& sum, const float* sxs, float2 sw, float2 bias, int c0, int odd, long long m0, int cols, Residuals<ROWS>& held) {
    const bool f16 = P.y_type == FXPQ_FT_F16;
    const SigAct sig(P.e.act);
    const float low = P.e.act == FXPQ_ACT_RELU ? 0.0f : -__int_as_float(0x7f800000);
    cols = c0 < P.N ? cols - odd : 0;  // tokens 2 i + odd with 2 i < cols exist
    sxs += odd;
    const float ps = P.e.pre_scale;
    // (addresses that walk along the tokens: computed from the token each, they took more registers than there are)
    const int kept = P.e.pre_f32 ? 4 : 2;
    const long long y_step = 2 * P.ys * 2, p_step = 2 * P.e.pre_stride * kept;
    char* pre = P.e.pre ? static_cast<char*>(P.e.pre) + ((m0 + odd) * P.e.pre_stride + c0) * kept : nullptr;
    auto act = [&](float z) { return FORM == SIGMOID ? sig(z) : FORM == NORMAL ? gelu(z) : cut(z, low); };
    auto pack = [&](float a, float b) {
        if (f16) return h2_bits(__floats2half2_rn(a, b));
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    };
    // STEP pairs of tokens at a time, each step of the arithmetic for all of them: one pair after the other left the warps waiting for
    // every exchange and exponential in turn (8192 x 2 x 5632 of 2048: 24 thousand clocks a tile, its products 16).
    constexpr int STEP = EPI == LAYER ? 4 : 8;
    const int second = (threadIdx.x >> 1) & 1, reach = EPI == GATED ? cols - 2 * second : cols;
    char* y = static_cast<char*>(P.y) + (EPI == GATED ? (m0 + odd + 2 * second) * P.ys + (c0 >> 1) - second : (m0 + odd) * P.ys + c0) * 2;
#pragma unroll
    for (int i0 = 0; i0 < ROWS / 2; i0 += STEP) {
        float a[STEP], b[STEP];  // channels c0, c0 + 1 of token 2 (i0 + i) + odd
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            const float2 s = channel_pair(sum(2 * (i0 + i)), sum(2 * (i0 + i) + 1), odd);
            a[i] = s.x, b[i] = s.y;
        }
        if (P.e.pre) {
#pragma unroll
            for (int i = 0; i < STEP; ++i) {
                if (2 * (i0 + i) < cols) {
                    if (P.e.pre_f32)
                        *reinterpret_cast<float2*>(pre) = make_float2(a[i], b[i]);
                    else
                        *reinterpret_cast<__half2*>(pre) = __floats2half2_rn(a[i] * ps, b[i] * ps);
                }
                pre += p_step;
            }
        }
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            const float sx = sxs[2 * (i0 + i)];
            a[i] = fmaf(a[i] * sx, sw.x, bias.x), b[i] = fmaf(b[i] * sx, sw.y, bias.y);
        }
#pragma unroll
        for (int i = 0; i < STEP; ++i) a[i] = act(a[i]);
        if constexpr (EPI == GATED) {
#pragma unroll
            for (int i = 0; i < STEP; ++i) a[i] *= b[i];
#pragma unroll
            for (int i = 0; i < STEP; i += 2) {  // two columns of token 2 (i0 + i) + odd, or with `second` of the one two further on
                const float o = __shfl_xor_sync(0xffffffffu, second ? a[i] : a[i + 1], 2);
                if (2 * (i0 + i) < reach) *reinterpret_cast<uint32_t*>(y) = second ? pack(o, a[i + 1]) : pack(a[i], o);
                y += 2 * y_step;
            }
        } else {
#pragma unroll
            for (int i = 0; i < STEP; ++i) b[i] = act(b[i]);
            if (P.e.res) {
#pragma unroll
                for (int i = 0; i < STEP; ++i) {
                    const float2 f = pair_f32(held.r[(i0 + i) % held.HELD], P.y_type);
                    a[i] += f.x, b[i] += f.y;
                }
#pragma unroll
                for (int i = 0; i < STEP; ++i)
                    if (i0 + i + held.HELD < ROWS / 2) held.ask(i0 + i + held.HELD, cols);
            }
#pragma unroll
            for (int i = 0; i < STEP; ++i) {
                if (2 * (i0 + i) < cols) *reinterpret_cast<uint32_t*>(y) = pack(a[i], b[i]);
                y += y_step;
            }
        }
    }
}
// f of the activation as a constant.
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    switch (act) {
        case FXPQ_ACT_RELU: f(std::integral_constant<int, FXPQ_ACT_RELU>()); break;
        case FXPQ_ACT_SILU: f(std::integral_constant<int, FXPQ_ACT_SILU>()); break;
        case FXPQ_ACT_GELU: f(std::integral_constant<int, FXPQ_ACT_GELU>()); break;
        case FXPQ_ACT_GELU_TANH: f(std::integral_constant<int, FXPQ_ACT_GELU_TANH>()); break;
        default: f(std::integral_constant<int, FXPQ_ACT_NONE>());
    }
}
// n values of a column, rows `step` elements apart, into an array of any type.
template <int N>
__device__ __forceinline__ void store_column(void* p, int type, long long at, long long step, const float (&v)[N], int n) {
    if (type == FXPQ_FT_F32) {
        float* q = static_cast<float*>(p) + at;
#pragma unroll
        for (int i = 0; i < N; ++i, q += step)
            if (i < n) *q = v[i];
    } else {
        unsigned short* q = static_cast<unsigned short*>(p) + at;
#pragma unroll
        for (int i = 0; i < N; ++i, q += step) {
            const unsigned short w = type == FXPQ_FT_F16 ? __half_as_ushort(__float2half_rn(v[i])) : __bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
            if (i < n) *q = w;
        }
    }
}

// 16 tokens of any type, alignment and activation.  A lane keeps its channel, so that a token's 32 lie side by side whatever their
// alignment; only gate and value meet first, and then a lane has every other token.
template <int EPI>
__device__ __forceinline__ void epilogue_any(const ManyArgs& P, const uint32_t (&v)[16], const float* sxs, float sw, float bias, int ch, long long m0,
                                             int cols) {
    if (ch >= P.N) cols = 0;
    uint32_t r[16];  // residuals as they lie in memory (asked for before anything is stored: y may be the residual)
    const bool wide = P.y_type == FXPQ_FT_F32;
    if (EPI == LAYER && P.e.res) {
        const long long at = m0 * P.e.res_stride + ch;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            r[i] = 0;
            if (i < cols) r[i] = wide ? (static_cast<const uint32_t*>(P.e.res) + at)[i * P.e.res_stride] : (static_cast<const unsigned short*>(P.e.res) + at)[i * P.e.res_stride];
        }
    }
    float z[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = __uint_as_float(v[i]) * (P.e.pre_f32 ? 1.0f : P.e.pre_scale);
    if (P.e.pre) store_column(P.e.pre, P.e.pre_f32 ? FXPQ_FT_F32 : FXPQ_FT_F16, m0 * P.e.pre_stride + ch, P.e.pre_stride, z, cols);
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = fmaf(__uint_as_float(v[i]) * sxs[i], sw, bias);
    if constexpr (EPI == GATED) {
        const int odd = ch & 1;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 p = channel_pair(z[2 * i], z[2 * i + 1], odd);
            y[i] = p.x, z[i] = p.y;
        }
        with_act(P.e.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = activate(y[i], decltype(act)::value) * z[i];
        });
        store_column(P.y, P.y_type, (m0 + odd) * P.ys + (ch >> 1), 2 * P.ys, y, (cols - odd + 1) >> 1);
    } else {
        with_act(P.e.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = activate(z[i], decltype(act)::value);
        });
        if (P.e.res) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                z[i] += wide ? __uint_as_float(r[i]) : P.y_type == FXPQ_FT_F16 ? __half2float(__ushort_as_half((unsigned short)r[i])) : __uint_as_float(r[i] << 16);
        }
        store_column(P.y, P.y_type, m0 * P.ys + ch, P.ys, z, cols);
    }
}

// Registers of a thread where the epilogue has 16 warps: the launch holds 768 x 80, of which the epilogue's take 512 x 96 and the others
// 128 x 32 (copies, products) and 128 x 64 (converters).
constexpr int LM_REGS = 80, LM_REGS_EPI = 96, LM_REGS_ISSUE = 32, LM_REGS_CONV = 64;
static_assert(LM_REGS_ISSUE + LM_REGS_CONV + 4 * LM_REGS_EPI <= 6 * LM_REGS, "the launch's registers");

__device__ __forceinline__ void load_sums(uint32_t at, uint32_t (&v)[16]) { tc::tmem_ld16_nw(at, v); }
__device__ __forceinline__ void load_sums(uint32_t at, uint32_t (&v)[32]) { tc::tmem_ld32_nw(at, v); }

constexpr int many_threads(int epi) { return epi == PLAIN ? 512 : 768; }

// NT: tokens of a tile, 256 or, where those tiles would leave pairs idle, 128.
template <int NT, int EPI, int FORM>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(many_threads(EPI), 1) linear_many_kernel(const __grid_constant__ ManyArgs P) {
    using namespace tc;
    constexpr int EW = EPI == PLAIN ? 8 : 16, ROWS = NT * 4 / EW;      // warps of the epilogue, and each one's columns
    // Tokens of a tile, and of a warp.  PARTS: the tile's first half of columns are its tokens' first parts, CTA 0's half of the operand, the
    // second half their second, CTA 1's; a warp has the same tokens of both, and what it stores is joined in registers.
    constexpr int TILE = EPI == PARTS ? NT / 2 : NT, TOKENS = EPI == PARTS ? ROWS / 2 : ROWS;
    constexpr int HALF_ROWS = NT / 2, STAGE = HALF_ROWS * 128;         // tokens of a CTA's half of the operand, its stage
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    __shared__ __align__(8) uint64_t bars[2 * LM_RAW + 2 * LM_B + 2 * LM_A + 3];
    __shared__ __align__(16) float s_sx[EW][ROWS];
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
        mbar_init(acc_empty, 2 * EW);  // (CTA 0's: the epilogue warps of both)
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
    const int n_work = EPI == PLAIN ? P.n_tiles : P.whole + (P.n_tiles - P.whole) * P.shares;
    // Work t: a tile, and of its reduction the blocks first .. last - 1.
    const auto share_of = [&](int& t, int& first, int& last) {
        first = 0, last = n_kb;
        if (EPI == PLAIN || t < P.whole) return 0;
        const int share = (t - P.whole) % P.shares;
        t = P.whole + (t - P.whole) / P.shares;
        first = (int)((long long)n_kb * share / P.shares), last = (int)((long long)n_kb * (share + 1) / P.shares);
        return share;
    };

    if (warp < 4) {
        if constexpr (EPI != PLAIN) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LM_REGS_ISSUE));
        if (warp == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int u = pair; u < n_work && ok; u += pairs) {
                int tn, tm, t = u, first, last;
                share_of(t, first, last);
                tile_of(P, t, tn, tm);
                for (int kb = first; kb < last; ++kb, ++it) {
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
            for (int u = pair; u < n_work && ok; u += pairs) {
                int tn, tm, t = u, first, last;
                share_of(t, first, last);
                tile_of(P, t, tn, tm);
                for (int hb = 2 * first; hb < min(n_half, 2 * last); ++hb, ++it) {
                    const uint32_t s = it % LM_B;
                    if (!wait_warp(b_empty + 8 * s, ((it / LM_B) & 1) ^ 1, abort, P.status)) {
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_arrive_expect_tx(b_full + 8 * s, 2 * STAGE);
                    tma_load_2d_pair(b0 + s * STAGE, &P.tx, hb * 64, tm * TILE + rank * (EPI == PARTS ? (int)P.M : HALF_ROWS), lead + 8 * s);
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
                for (int u = pair; u < n_work && ok; u += pairs, ++it) {
                    int t = u, first, last;
                    share_of(t, first, last);
                    if (!wait_warp_cluster(acc_empty, (it & 1) ^ 1, abort, P.status)) break;
                    tc_fence_after();
                    uint32_t acc = 0;
                    for (int kb = first; kb < last && ok; ++kb, ++ia) {
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
        for (int u = pair; u < n_work && ok; u += pairs) {
            int t = u, first, last;
            share_of(t, first, last);
            for (int kb = first; kb < last; ++kb, ++it) {
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
        }
    } else {
        if constexpr (EPI != PLAIN) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(LM_REGS_EPI));
        const int quad = warp & 3, half = (warp - 8) >> 2;  // channels 32 quad + lane, tokens TOKENS half ..
        const uint32_t lead = cluster_addr(acc_empty, 0), at = tmem + ((uint32_t)(quad * 32) << 16) + TOKENS * half;
        float* sxs = s_sx[warp - 8];
        uint32_t it = 0;
        for (int u = pair; u < n_work; u += pairs, ++it) {
            int tn, tm, t = u, first, last;
            const int share = share_of(t, first, last);
            tile_of(P, t, tn, tm);
            const int ch = tn * 256 + rank * 128 + quad * 32 + lane;
            const long long m0 = (long long)tm * TILE + TOKENS * half;
            const float sw = !P.sw ? 1.0f : ch < P.N ? __ldg(P.sw + ch) : 0.0f, bias = P.bias && ch < P.N ? __ldg(P.bias + ch) : 0.0f;
            for (int i = lane; i < TOKENS; i += 32) sxs[i] = !P.sx ? 1.0f : m0 + i < P.M ? __ldg(P.sx + m0 + i) : 0.0f;
            __syncwarp();
            const int cols = (int)min((long long)TOKENS, P.M - m0);
            Residuals<TOKENS> held;
            if constexpr (EPI == LAYER) {
                const int odd = lane & 1, c0 = ch - odd;
                held.at = static_cast<const char*>(P.e.res) + ((m0 + odd) * P.e.res_stride + c0) * 2, held.step = 2 * P.e.res_stride * 2;
                if (P.e.fast && P.e.res && t < P.whole) {
#pragma unroll
                    for (int i = 0; i < held.HELD; ++i) held.ask(i, c0 < P.N ? cols - odd : 0);
                }
            }
            if (!wait_warp_cluster(acc_full, it & 1, abort, P.status)) break;
            tc_fence_after();
            if constexpr (EPI != PLAIN) {
                const int odd = lane & 1, c0 = ch - odd;
                const float sw_o = __shfl_xor_sync(0xffffffffu, sw, 1), bias_o = __shfl_xor_sync(0xffffffffu, bias, 1);
                const float2 sw2 = odd ? make_float2(sw_o, sw) : make_float2(sw, sw_o), bias2 = odd ? make_float2(bias_o, bias) : make_float2(bias, bias_o);
                constexpr int W = EPI == PARTS ? TOKENS : 32, APART = EPI == PARTS ? TILE : 32, AFTER = EPI == PARTS ? LAYER : EPI;
                uint32_t v[ROWS / W][W];  // (both parts)
#pragma unroll
                for (int c = 0; c < ROWS / W; ++c) load_sums(at + APART * c, v[c]);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < ROWS / W; ++c) reg_fence(v[c]);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(lead);  // the accumulators may be overwritten
                if (t >= P.whole) {
                    float* to = P.part + ((((long long)share * (P.n_tiles - P.whole) + t - P.whole) * 2 + rank) * NT + TOKENS * half) * 128 + quad * 32 + lane;
#pragma unroll
                    for (int i = 0; i < ROWS; ++i)
                        if ((EPI == PARTS ? i % W : i) < cols) to[(i / W * APART + i % W) * 128] = __uint_as_float(v[i / W][i % W]);
                    __syncwarp();  // (the scales are read)
                    continue;
                }
                if constexpr (EPI == PARTS) {
#pragma unroll
                    for (int i = 0; i < W; ++i) v[0][i] = __float_as_uint(fmaf(__uint_as_float(v[0][i]), PART, __uint_as_float(v[1][i])));
                }
                if (P.e.fast) {
                    epilogue_fast<TOKENS, AFTER, FORM>(P, [&](int t) { return __uint_as_float(v[t / W][t % W]); }, sxs, sw2, bias2, c0, odd, m0, cols, held);
                } else {  // 16 tokens at a time, in one place of the code: the others move up
#pragma unroll 1
                    for (int c = 0; c < TOKENS; c += 16) {
                        uint32_t now[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) now[i] = v[0][i];
                        epilogue_any<AFTER>(P, now, sxs + c, sw, bias, ch, m0 + c, cols - c);
#pragma unroll
                        for (int i = 0; i < TOKENS - 16; ++i) v[i / W][i % W] = v[(i + 16) / W][(i + 16) % W];
                    }
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
inline bool many_tokens(int64_t M, int32_t N, int32_t K) { return M > 256 && N >= 128 && K >= 128; }

inline int many_pairs() { return num_sms() / 2 > 0 ? num_sms() / 2 : 1; }
// Tiles of 256 tokens, or of 128 where their rounds over the pairs take less time.  A round of the narrow ones takes two
// thirds of the wide ones' (8192 x 8192 of 4096: 13.2 and 20.1 us; every tile expands 256 channels' weights).
inline int many_tile(int64_t M, int32_t N) {
    const int64_t pairs = many_pairs(), tn = ((int64_t)N + 255) / 256;
    const auto rounds = [&](int64_t nt) { return (tn * ((M + nt - 1) / nt) + pairs - 1) / pairs; };
    return 2 * rounds(128) < 3 * rounds(256) ? 128 : 256;
}
struct ManyPlan {
    int nt, whole, shares;
    float* part;
};

// Lets a kernel use so much dynamic shared memory, once on each device.  regs: what its launch has to hold of them a thread (0: any), for
// warps that take more later wait for ever if they are not there.
template <typename Kernel>
bool allow_smem(Kernel kernel, int bytes, std::atomic<uint64_t>& set, int regs = 0) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return false;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (set.load(std::memory_order_relaxed) & bit) return true;
    cudaFuncAttributes has;
    if (regs && (cudaFuncGetAttributes(&has, kernel) != cudaSuccess || has.numRegs < regs)) return false;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    set.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

// Clusters of c that run at once on the current device, at least one, or -1.  Asked for once on each device (the call takes some us): a `known`, zeros at
// first, belongs to one kernel, cluster size and amount of shared memory, for a choice may rest on sizes alone, not on the calls before.
constexpr int DEVICES = 16;
template <typename Kernel>
int clusters_at_once(Kernel kernel, const cudaLaunchConfig_t& c, std::atomic<int> (&known)[DEVICES]) {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return -1;
    if (dev < DEVICES) n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &c) != cudaSuccess || n <= 0) {
            (void)cudaGetLastError();
            n = -1;
        }
        if (dev < DEVICES) known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

template <int NT, int EPI, int FORM>
fxpq_status launch_many(ManyArgs& P, cudaStream_t st) {
    const auto kernel = linear_many_kernel<NT, EPI, FORM>;
    static std::atomic<uint64_t> set{0};
    if (!allow_smem(kernel, LM_SMEM, set, EPI == PLAIN ? 0 : LM_REGS)) return FXPQ_ERR_CUDA;
    constexpr int TILE = EPI == PARTS ? NT / 2 : NT;
    const long long tn = ((long long)P.N + 255) / 256, tm = (P.M + TILE - 1) / TILE;
    if (tn * tm > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    P.tiles_n = (int)tn, P.tiles_m = (int)tm, P.n_tiles = (int)(tn * tm);
    P.y_pair = aligned(P.y, 4) && P.ys % 2 == 0;
    P.whole = P.whole < P.n_tiles ? P.whole : P.n_tiles;
    const long long work = P.whole + (tn * tm - P.whole) * P.shares, pairs = many_pairs();
    if (work > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    launch_pdl(kernel, dim3(2 * (unsigned)(work < pairs ? work : pairs)), dim3(many_threads(EPI)), LM_SMEM, st, P);
    return after_launch("linear_many");
}

template <int EPI>
fxpq_status product_many(const __half* half, size_t pitch, const float* d_sx, const int8_t* d_w, int64_t w_stride, const float* d_sw,
                         const float* d_bias, int64_t M, int32_t N, int32_t K, int32_t y_type, void* d_y, int64_t y_stride, cudaStream_t st,
                         const Epi& e = {}, const ManyPlan* plan = nullptr, ManyArgs* args = nullptr) {
    ManyArgs mine;
    ManyArgs& P = args ? *args : mine;  // (what finish_kernel takes)
    P.e = e, P.whole = plan ? plan->whole : INT32_MAX, P.shares = plan ? plan->shares : 1, P.part = plan ? plan->part : nullptr;
    const int nt = plan ? plan->nt : many_tile(M, N);
    if (!encode_rows(&P.tw, d_w, N, K, w_stride, 128) || !encode_half_rows(&P.tx, half, EPI == PARTS ? 2 * M : M, K, (long long)pitch, nt / 2))
        return FXPQ_ERR_CUDA;
    P.sx = d_sx, P.sw = d_sw, P.bias = d_bias, P.y = d_y, P.ys = y_stride, P.M = M, P.N = N, P.K = K, P.y_type = y_type;
    P.status = status_ptr();
    const auto go = [&](auto form) {
        constexpr int FORM = decltype(form)::value;
        return nt == 128 ? launch_many<128, EPI, FORM>(P, st) : launch_many<256, EPI, FORM>(P, st);
    };
    if constexpr (EPI != PLAIN) {
        const int type = ftype_bytes(y_type), kept = e.pre_f32 ? 4 : 2;
        P.e.vec = (aligned(d_y, 2 * type) && y_stride % 2 == 0 ? 1 : 0) | (aligned(e.res, 2 * type) && e.res_stride % 2 == 0 ? 2 : 0) |
                  (aligned(e.pre, 2 * kept) && e.pre_stride % 2 == 0 ? 4 : 0);
        // (a gate that is cut, the rarest form, has no kernel of its own)
        P.e.fast = y_type != FXPQ_FT_F32 && P.e.vec == 7 && N % (EPI == GATED ? 4 : 2) == 0 && !(EPI == GATED && e.act == FXPQ_ACT_RELU);
    }
    if constexpr (EPI == LAYER || EPI == GATED) {
        if (e.act == FXPQ_ACT_GELU) return go(std::integral_constant<int, NORMAL>());
        if (EPI == GATED || e.act == FXPQ_ACT_SILU || e.act == FXPQ_ACT_GELU_TANH) return go(std::integral_constant<int, SIGMOID>());
    }
    if constexpr (EPI != GATED) return go(std::integral_constant<int, CUT>());
    return FXPQ_ERR_UNSUPPORTED;
}
}  // namespace
}  // namespace llm
}  // namespace fxpq
