// fxpq_attend_tile.cu -- attention of many query rows (prompts and chunks) on tcgen05.
//
// A CTA takes 256 query rows (tokens x grouped heads) of one sequence and key head as two tiles of 128 rows and walks
// the keys 128 at a time.  Two products of 128 x 128 x dim per tile and 128 keys bound it: S = Q K^T into tensor memory, then
// O += W V with the weights W as the operand in tensor memory, in place of S.  The two tiles alternate: one's products run
// during the other's exponentials.
//   warps 0-3, 4-7, 8-11, 12-15  softmax: X and Y of tile 0, X and Y of tile 1, a thread per row; X forms the weights of a step's
//                   first 64 keys and Y those of the others, at the same time; at the end each writes half of O / l
//   warps 16-19     converters: codes to fp16 operand tiles of 128 keys, once for both row tiles (none where the codes came
//                   expanded; the warps that follow are then 16 to 19)
//   warp 20         tensor memory, products;   warp 21   pages, scales, copies;   22, 23   none
// A step's weights are formed with the maximum m as it was; only where 16 of them sum past 2^15 (a few times per row) are
// they formed again, after the sums have been rescaled.  m then moves by whole powers of two, so that rescaling is
// exact.  X and Y share m: one barrier of their two warps tells both whether either's weights have to be formed again.
// (Told by one mbarrier each way instead, X and Y waited for one another in turn: 913 us for 2 prompts of 8192, with it 835.)
// A register that spills costs more than anything else here: with the converters' loop over its two halves unrolled, which
// spills 64 bytes, a step of 128 keys takes 1761 ns, so 1608.  The expanded form has no converters and leaves the softmax 112.
// With one thread a row forming the weights of 64 keys after the other a tile's chain was 2300 cycles of softmax for 128 keys.
// Codes arrive as they are stored ([keys][dim] bytes, one TMA box per page): K is a K-major operand and V, with the
// same bytes, an operand whose columns are contiguous, so that neither is transposed.
// Tried: two buffers of S of 64 keys, so that no softmax waits for a product.  The scores' products of 64 columns read Q twice
// as often, 3072 cycles of shared memory per 128 keys instead of 2560 (products alone: 2048), and 2 prompts of 8192
// tokens took 1335 us instead of 1165.
#include "fxpq_attend.cuh"

namespace fxpq {
namespace llm {
namespace {

using namespace tc;

constexpr int KEYS = 128, STEP = 64, ROWS = 256;  // keys of an operand tile, of X or Y
// Operand tiles K 0, V 0, K 1, .. pass through RAWS stages of codes (copies in flight) and CONVS expanded ones (the products hold V of one step and K of the next, a third is being written).
constexpr int RAWS = 3;
__host__ __device__ constexpr int convs(bool pre) { return pre ? 4 : 3; }
__host__ __device__ constexpr int threads(bool pre) { return pre ? 640 : 768; }  // (without converters)
constexpr float MANY = 32768.0f;  // 16 weights may sum to this much, so that each is within fp16's range
constexpr int TABS = 8;  // scale tables in flight: the copies run at most five tiles ahead of the softmax

template <int D, bool PRE>
struct Smem {  // offsets from the 1024-byte aligned base
    static constexpr int Q = 128 * D * 2, CONV = KEYS * D * 2, RAW = KEYS * D;
    static constexpr int conv0 = 2 * Q, raw0 = conv0 + convs(PRE) * CONV, bytes = raw0 + (PRE ? 0 : RAWS * RAW) + 1024;
};
static_assert(Smem<128, false>::bytes + 8192 <= 232448 && Smem<128, true>::bytes + 8192 <= 232448, "shared memory of a CTA");

// Operand whose columns (the rows of O^T) are contiguous: 64 of them in a 128-byte swizzled row, 8 reduction steps to a
// 1024-byte group, the next 64 columns 16 KB on.
__device__ __forceinline__ uint64_t make_sdesc_mn(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)(16384u >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1u << 46 |
           (uint64_t)2u << 61;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Whether the predicate holds in any thread of two warps.
__device__ __forceinline__ bool bar_any(int id, bool pred) {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %2, 0;\n\t"
        "bar.red.or.pred q, %1, 64, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(any)
        : "r"(id), "r"((uint32_t)pred)
        : "memory");
    return any != 0;
}

template <int D, bool PRE>
__global__ void __launch_bounds__(threads(PRE), 1) attend_tile_kernel(const __grid_constant__ AttendArgs A) {
    using S = Smem<D, PRE>;
    constexpr int CONVS = convs(PRE), ISSUER = PRE ? 16 : 20;  // the warp of the products
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    __shared__ __align__(8) uint64_t bars[2 * RAWS + 2 * CONVS + TABS + 2 + 2 + 2 + 1 + 1];
    __shared__ float tab[TABS][3][8];  // per 16 keys: key scale, log2 of the value scale lifted, its inverse
    __shared__ float row_cf[ROWS];  // what a row's scores are multiplied by, but for the key block's scale
    __shared__ float top_of[2][ROWS], end_l[2][ROWS];  // of X and Y: what m has to grow to, the normaliser at the end
    __shared__ volatile int quits[8];                  // X or Y of [tile][32 rows] waited too long
    __shared__ int abort_flag;
    __shared__ uint32_t tmem_slot;
    volatile int* abort = &abort_flag;
    const uint32_t raw_full = smem_u32(bars), raw_empty = raw_full + 8 * RAWS, conv_full = raw_empty + 8 * RAWS,
                   conv_empty = conv_full + 8 * CONVS, tab_full = conv_empty + 8 * CONVS, s_full = tab_full + 8 * TABS, p_full = s_full + 16, o_full = p_full + 16,
                   q_full = o_full + 16, drained = q_full + 8;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_full + 8 * i, 8);
            mbar_init(o_full + 8 * i, 1);
        }
        for (int i = 0; i < 8; ++i) quits[i] = 0;
        for (int i = 0; i < RAWS; ++i) {
            mbar_init(raw_full + 8 * i, 1);
            mbar_init(raw_empty + 8 * i, 4);
        }
        for (int i = 0; i < CONVS; ++i) {
            mbar_init(conv_full + 8 * i, PRE ? 1 : 4);
            mbar_init(conv_empty + 8 * i, 1);
        }
        for (int i = 0; i < TABS; ++i) mbar_init(tab_full + 8 * i, 1);
        mbar_init(q_full, 16);
        mbar_init(drained, 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&A.tk);
        prefetch_tmap(&A.tv);
    }
    pdl_wait();

    // ---- this CTA's rows and keys (uniform)
    const long long cand = gridDim.x / A.heads - 1 - blockIdx.x / A.heads;  // the longest of a causal sequence first
    const int h = blockIdx.x % A.heads;
    const int per_seq = A.s.starts ? 0 : (A.s.each * A.group + ROWS - 1) / ROWS;
    const int b = A.s.starts ? find_seq(A.s, cand, A.group, ROWS, 1) : (int)(cand / per_seq);
    const int rb = (int)(cand - (A.s.starts ? unit_base(max(__ldg(A.s.starts + b), 0), b, A.group, ROWS, 1) : (long long)b * per_seq));
    int first, count;
    new_rows(A.s, b, first, count);
    const int all_rows = count * A.group;
    if (rb < 0 || rb * ROWS >= all_rows || (A.few_only && all_rows <= A.few)) return;
    const int rows = min(ROWS, all_rows - rb * ROWS), tiles = rows > 128 ? 2 : 1;
    const int len = max(0, __ldg(A.s.lens + b)), end = (int)min((long long)len, (long long)A.s.max_pages * A.page);
    if (end < len && threadIdx.x == 0) latch_status(A.status, FXPQ_ERR_RANGE);
    const int last_pos = len - count + (rb * ROWS + rows - 1) / A.group;
    const int seen = last_pos < 0 ? 0 : A.causal ? min(last_pos + 1, end) : end;  // keys that any row sees
    const int n_all = (seen + KEYS - 1) / KEYS;
    const int j0 = (int)((long long)n_all * blockIdx.y / gridDim.y), n = (int)((long long)n_all * (blockIdx.y + 1) / gridDim.y) - j0;

    if (warp == ISSUER) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const uint32_t base = smem_u32(smem);

    // (the launch holds 768 x 80 registers, 512 x 96 + 256 x 48, or 640 x 96, 512 x 112 + 128 x 32)
    if (warp < 16)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PRE ? 112 : 96));
    else
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PRE ? 32 : 48));

    if (warp < 16) {
        // ================================================================ softmax: one row per thread
        const int t = warp >> 3, y = (warp >> 2) & 1, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16, ts = tmem + 128 * t + lanes, to = tmem + 256 + 128 * t + lanes;
        const int id = 1 + 4 * t + quad;  // the barrier of this X and Y, who both come to it in every step whatever happened
        {  // 16 rows a warp, 16 bytes a lane: whole rows at once (a row per thread took 15000 cycles; 2 prompts of 8192 835 us, so 775)
            constexpr int LANES = D / 8, EACH = 32 / LANES, IT = 8 / EACH;  // lanes of a row, rows of a load
            const bool f16 = A.q_f16;
            const int d = 8 * (lane % LANES), row0 = quad * 32 + 16 * y + lane / LANES;
#pragma unroll 1  // (in one go, 8 loads more in flight, a few registers of the loop below spill)
            for (int from = 0; from < 16; from += 8) {
                uint4 x[IT];
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    const int row = t * 128 + row0 + from + it * EACH, at = rb * ROWS + row, token = at / A.group;
                    x[it] = make_uint4(0u, 0u, 0u, 0u);
                    if (row < rows) {
                        const unsigned short* src = static_cast<const unsigned short*>(A.q) + (long long)(first + token) * A.q_token +
                                                    (long long)(h * A.group + at - token * A.group) * A.q_head + d;
                        if (A.q_vec)
                            x[it] = *reinterpret_cast<const uint4*>(src);
                        else
                            x[it] = make_uint4(src[0] | (uint32_t)src[1] << 16, src[2] | (uint32_t)src[3] << 16, src[4] | (uint32_t)src[5] << 16,
                                               src[6] | (uint32_t)src[7] << 16);
                    }
                }
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    const int row = row0 + from + it * EACH;
                    const uint32_t raw[4] = {x[it].x, x[it].y, x[it].z, x[it].w};
                    float2 v[4];
                    float top = 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[i] = f16 ? __half22float2(*reinterpret_cast<const __half2*>(&raw[i]))
                                   : make_float2(__uint_as_float(raw[i] << 16), __uint_as_float(raw[i] & 0xffff0000u));
                        const float big = fmaxf(fabsf(v[i].x), fabsf(v[i].y));  // (a row with a NaN is not scaled)
                        top = fmaxf(top, v[i].x != v[i].x || v[i].y != v[i].y ? INFINITY : big);
                    }
#pragma unroll
                    for (int o = LANES / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const int e = q_exponent(top);
                    const float up = pow2i(e);
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = h2_bits(__floats2half2_rn(v[i].x * up, v[i].y * up));
                    *reinterpret_cast<uint4*>(smem + t * S::Q + (d >> 6) * 16384 + row * 128 + ((((d >> 3) & 7) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                    if (d == 0) row_cf[t * 128 + row] = A.scale * LOG2E * pow2i(-e);
                }
            }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
        asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
        const float cf = row_cf[t * 128 + r];
        if (t < tiles) {
            const int pos = len - count + (rb * ROWS + t * 128 + r) / A.group;
            // keys that the row sees (rows past the last one hold zeros: what they see does not matter)
            const int limit = t * 128 + r >= rows ? 1 << 30 : pos < 0 ? 0 : A.causal ? min(pos + 1, end) : end;
            float m = NO_MAX, l = 0.0f;
            bool ok = true;
            const uint32_t sb = ts + STEP * y;
            for (int i = 0; i < n; ++i) {
                const int slot = i % TABS;
                // (a wait that is already over takes some 200 cycles, so the scores' comes last)
                if (!wait_warp(tab_full + 8 * slot, (i / TABS) & 1, abort, A.status) || !wait_warp(s_full + 8 * t, i & 1, abort, A.status)) {
                    quits[id - 1] = 1;
                    bar_any(id, true);
                    ok = false;
                    break;
                }
                tc_fence_after();
                const int room = limit - (j0 + i) * KEYS - STEP * y;  // of these 64 keys, those that the row sees
                const float *kf = tab[slot][0] + 4 * y, *lg = tab[slot][1] + 4 * y, *iv = tab[slot][2] + 4 * y;
                const bool masked = __any_sync(0xffffffffu, room < STEP);  // the last steps of a row
                uint32_t w[2][16];
                float part, over;  // the normaliser, the largest sum of 16 weights
                auto mask = [&](int c, uint32_t (&s)[32]) {
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[e] = 32 * c + e < room ? s[e] : 0xff800000u;
                    }
                };
                bool quit = false;
                for (int raised = 0;; raised = 1) {
                    float sums[4];
                    uint32_t both[2][32];  // (one round trip for all 64 scores)
                    tmem_ld32_nw(sb, both[0]);
                    tmem_ld32_nw(sb + 32, both[1]);
                    tmem_wait_ld();
                    reg_fence(both[0]);
                    reg_fence(both[1]);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t(&s)[32] = both[c];
                        float2 x[16];
                        mask(c, s);
#pragma unroll
                        for (int g = 0; g < 2; ++g) {  // 16 keys of one scale
                            // (FLT_MIN: a page outside the cache has scale 0, which must not meet the -inf of a masked score)
                            const float f = fmaxf(kf[2 * c + g] * cf, FLT_MIN), lv = lg[2 * c + g] - m;
#pragma unroll
                            for (int e = 8 * g; e < 8 * g + 8; ++e)
                                x[e] = __ffma2_rn(make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), make_float2(f, f), make_float2(lv, lv));
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = make_float2(ex2(x[e].x), ex2(x[e].y));
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            float2 a = __fadd2_rn(x[8 * g], x[8 * g + 1]), b2 = __fadd2_rn(x[8 * g + 2], x[8 * g + 3]);
                            a = __fadd2_rn(a, __fadd2_rn(x[8 * g + 4], x[8 * g + 5]));
                            b2 = __fadd2_rn(b2, __fadd2_rn(x[8 * g + 6], x[8 * g + 7]));
                            a = __fadd2_rn(a, b2);
                            sums[2 * c + g] = a.x + a.y;
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) w[c][e] = h2_bits(__floats2half2_rn(x[e].x, x[e].y));
                    }
                    over = fmaxf(max3(sums[0], sums[1], sums[2]), sums[3]);
                    part = fmaf(sums[0], iv[0], sums[1] * iv[1]) + fmaf(sums[2], iv[2], sums[3] * iv[3]);
                    if (!bar_any(id, over > MANY && !raised) || (quit = quits[id - 1])) break;
                    int row = 128 * t + r;
                    asm volatile("" : "+r"(row));  // (what follows is rare: nothing of it is to be kept in registers)
                    float top = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t s[32];
                        tmem_ld32_nw(sb + 32 * c, s);
                        tmem_wait_ld();
                        reg_fence(s);
                        mask(c, s);
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            float mx = -INFINITY;
#pragma unroll
                            for (int e = 16 * g; e < 16 * g + 16; e += 2) mx = max3(mx, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
                            top = fmaxf(top, mx == -INFINITY ? mx : fmaf(mx, kf[2 * c + g] * cf, lg[2 * c + g]));
                        }
                    }
                    top_of[y][row] = over > MANY ? ceilf(top) - LIFT : m;
                    asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
                    const float now = fmaxf(top_of[0][row], top_of[1][row]), f = now == m ? 1.0f : ex2(m - now);
                    m = now;
                    l *= f;
                    if (i > 0) {  // O holds all steps before (their products were issued before this step's scores); half of it each
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) {
                            const int c = (D / 32) * y + k;
                            uint32_t o[16];
                            tmem_ld16_nw(to + 16 * c, o);
                            tmem_wait_ld();
                            reg_fence(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tmem_st16_nw(to + 16 * c, o);
                        }
                    }
                }
                if (quit) {
                    ok = false;
                    break;
                }
                l += part;
                tmem_st16_nw(sb, w[0]);
                tmem_st16_nw(sb + 16, w[1]);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * t);
            }
            if (ok && n > 0) ok = wait_warp(o_full + 8 * t, 0, abort, A.status);
            tc_fence_after();
            end_l[y][128 * t + r] = l;
            asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
            if (ok) {
                int own = r;
                asm volatile("" : "+r"(own));  // (computed here: the loop has no register for it)
                const bool live = t * 128 + own < rows;
                const int rr = rb * ROWS + t * 128 + own, tok = rr / A.group;
                const long long orow = (long long)(first + tok) * A.q_heads + h * A.group + rr - tok * A.group;
                const bool split = gridDim.y > 1;
                float* part = A.part + ((long long)blockIdx.y * A.s.n_tokens * A.q_heads + orow) * (D + 4);
                l += end_l[1 - y][128 * t + r];
                const float inv = split ? 1.0f : l == 0.0f ? 0.0f : UNLIFT / l;
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    const int c = (D / 32) * y + k;
                    uint32_t o[16];
                    if (n > 0) {
                        tmem_ld16_nw(to + 16 * c, o);
                        tmem_wait_ld();
                        reg_fence(o);
                    }
                    float v[16];
                    // (rows that saw nothing hold zeros, or with a split nothing at all)
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = n > 0 ? __uint_as_float(o[e]) * inv : 0.0f;
                    if (live) {
                        if (split)
                            store_f32<16>(part + 4 + 16 * c, v);
                        else if (A.q_f16)
                            store_f32<16>(static_cast<__half*>(A.out) + orow * D + 16 * c, v);
                        else
                            store_f32<16>(static_cast<__nv_bfloat16*>(A.out) + orow * D + 16 * c, v);
                    }
                }
                if (live && split && !y) *reinterpret_cast<float2*>(part) = make_float2(m, l);
                if (live && !split && A.lse && !y) A.lse[orow] = l == 0.0f ? -INFINITY : (m + log2f(l)) * LN2;
            }
        }
    } else if (!PRE && warp < 20) {
        // ================================================================ converters
        const int t = threadIdx.x - 512;
        for (int u = 0; u < 2 * n; ++u) {  // K 0, V 0, K 1, V 1 ..
            const int rs = u % RAWS, cs = u % CONVS;
            if (!wait_warp(raw_full + 8 * rs, (u / RAWS) & 1, abort, A.status) ||
                !wait_warp(conv_empty + 8 * cs, ((u / CONVS) & 1) ^ 1, abort, A.status))
                break;
            const unsigned char* src = smem + S::raw0 + rs * S::RAW;
            unsigned char* dst = smem + S::conv0 + cs * S::CONV;
            constexpr int CH = D / 16, IT = KEYS * CH / 128;  // 16-code chunks of a row, of a thread
#pragma unroll 1
            for (int half = 0; half < IT / 4; ++half) {  // four loads in flight together
                uint4 v[4];
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int i = (4 * half + it) * 128 + t, row = i / CH, c = i % CH;
                    v[it] = *reinterpret_cast<const uint4*>(src + (D == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4)));
                }
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int i = (4 * half + it) * 128 + t, row = i / CH, c = i % CH, hf = c >> 2;
                    uint32_t x = v[it].x ^ 0x80808080u, y = v[it].y ^ 0x80808080u;
                    const uint4 o0 = make_uint4(code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR));
                    x = v[it].z ^ 0x80808080u, y = v[it].w ^ 0x80808080u;
                    const uint4 o1 = make_uint4(code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR));
                    unsigned char* d = dst + hf * 16384 + row * 128;
                    const int j = 2 * (c & 3), odd = D == 128 ? hf : 0;  // (lanes that would meet in a bank begin with the other chunk)
                    *reinterpret_cast<uint4*>(d + (((j + odd) ^ (row & 7)) << 4)) = odd ? o1 : o0;
                    *reinterpret_cast<uint4*>(d + (((j + 1 - odd) ^ (row & 7)) << 4)) = odd ? o0 : o1;
                }
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(raw_empty + 8 * rs);
                mbar_arrive(conv_full + 8 * cs);
            }
        }
    } else if (warp == ISSUER) {
        // ================================================================ products
        const uint32_t id_qk = make_idesc(128, KEYS), id_pv = make_idesc(128, D) | (1u << 16);
        // operand tile u of the ring (K 0, V 0, K 1, ..)
        auto have = [&](int u) { return wait_warp(conv_full + 8 * (u % CONVS), (u / CONVS) & 1, abort, A.status); };
        auto scores = [&](int t, int j) {  // 128 keys
            const uint64_t qd = make_sdesc(base + t * S::Q), kd = make_sdesc(base + S::conv0 + (2 * j % CONVS) * S::CONV);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
                tc_mma(tmem + 128 * t, qd + (kk >> 2) * (16384 >> 4) + 2 * (kk & 3), kd + (kk >> 2) * (16384 >> 4) + 2 * (kk & 3), id_qk, kk > 0);
            tc_commit(s_full + 8 * t);
            if (t == tiles - 1) tc_commit(conv_empty + 8 * (2 * j % CONVS));
        };
        bool ok = wait_warp(q_full, 0, abort, A.status);
        if (ok && n > 0 && have(0)) {
            tc_fence_after();
            for (int t = 0; t < tiles; ++t) scores(t, 0);
            for (int j = 0; j < n && ok; ++j) {
                const int uv = (2 * j + 1) % CONVS;
                if (!have(2 * j + 1)) break;
                for (int t = 0; t < tiles && ok; ++t) {
                    if (!wait_warp(p_full + 8 * t, j & 1, abort, A.status)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t vd = make_sdesc_mn(base + S::conv0 + uv * S::CONV);
#pragma unroll
                    for (int kk = 0; kk < KEYS / 16; ++kk)
                        tc_mma_ta(tmem + 256 + 128 * t, tmem + 128 * t + STEP * (kk >> 2) + 8 * (kk & 3), vd + kk * (2048 >> 4), id_pv, j > 0 || kk > 0);
                    if (j == n - 1) tc_commit(o_full + 8 * t);
                    if (t == tiles - 1) tc_commit(conv_empty + 8 * uv);
                    if (j + 1 < n) {
                        if (t == 0 && !have(2 * j + 2)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        scores(t, j + 1);
                    }
                }
            }
        }
        tc_commit(drained);  // every product issued here has completed once it fires
        drain_warp(drained, 0);
    } else if (warp == ISSUER + 1) {
        // ================================================================ pages, scales, copies
        const int* table = A.s.pages + (long long)b * A.s.pages_stride;
        struct Info {
            int pid;
            float ks, vs;
        };
        auto fetch = [&](int i0) {  // lane: 16 keys of one of four steps
            Info f;
            const long long p = (long long)(j0 + i0 + (lane >> 3)) * KEYS + 16 * (lane & 7);
            f.pid = -1;
            if (i0 + (lane >> 3) < n && p < seen) {
                f.pid = __ldg(table + p / A.page);
                if ((unsigned)f.pid >= (unsigned)A.n_pages) {
                    latch_status(A.status, FXPQ_ERR_RANGE);
                    f.pid = -1;
                }
            }
            f.ks = f.pid < 0 ? 0.0f : __ldg(A.k_scale + (long long)f.pid * A.heads + h);
            f.vs = f.pid < 0 ? 0.0f : __ldg(A.v_scale + (long long)f.pid * A.heads + h);
            return f;
        };
        Info cur = fetch(0), nxt = fetch(4);
        const int box = min(A.page, KEYS);
        int u = 0;
        bool ok = true;
        for (int i = 0; i < n && ok; ++i) {
            const int from = 8 * (i & 3), slot = i % TABS;
            if (lane >= from && lane < from + 8) {
                const float lv = cur.vs > 0.0f ? __log2f(cur.vs) + LIFT : -INFINITY;
                tab[slot][0][lane - from] = cur.ks;
                tab[slot][1][lane - from] = lv;
                tab[slot][2][lane - from] = cur.vs > 0.0f ? ex2(-lv) : 0.0f;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(tab_full + 8 * slot);
            if constexpr (PRE) {
                for (int v = 0; v < 2; ++v, ++u) {
                    const int cs = u % CONVS;
                    const uint32_t bar = conv_full + 8 * cs, dst = base + S::conv0 + cs * S::CONV;
                    if (!wait_warp(conv_empty + 8 * cs, ((u / CONVS) & 1) ^ 1, abort, A.status)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(bar, (uint32_t)S::CONV);
#pragma unroll
                    for (int d = 0; d < D; d += 64)
                        tma_load_3d(dst + (d >> 6) * 16384, v ? &A.tv : &A.tk, d, (j0 + i) * KEYS, b * A.heads + h, bar);
                }
            } else {
                const unsigned have = __ballot_sync(0xffffffffu, cur.pid >= 0) >> from;
                int boxes = 0;
                for (int g = 0; g < 8; g += box / 16) boxes += (have >> g) & 1;
                for (int v = 0; v < 2; ++v, ++u) {
                    const int rs = u % RAWS;
                    const uint32_t bar = raw_full + 8 * rs, dst = base + S::raw0 + rs * S::RAW;
                    if (!wait_warp(raw_empty + 8 * rs, ((u / RAWS) & 1) ^ 1, abort, A.status)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(bar, (uint32_t)(boxes * box * D));
                    for (int g = 0; g < 8; g += box / 16) {
                        const int pid = __shfl_sync(0xffffffffu, cur.pid, from + g);
                        if (pid >= 0) tma_load_3d(dst + 16 * g * D, v ? &A.tv : &A.tk, 0, 0, pid * A.heads + h, bar);
                    }
                }
            }
            if ((i & 3) == 3) {
                cur = nxt;
                nxt = fetch(i + 5);
            }
        }
        constexpr int RING = PRE ? CONVS : RAWS;  // every copy has landed
        for (int k = max(0, u - RING); k < u; ++k) drain_warp((PRE ? conv_full : raw_full) + 8 * (k % RING), (k / RING) & 1);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == ISSUER) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
    }
}

// Rows whose keys several CTAs shared: one warp per new token and query head.
template <int D>
__global__ void __launch_bounds__(128) attend_tile_join_kernel(const __grid_constant__ AttendArgs A, int shares) {
    pdl_wait();
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5), all = (long long)A.s.n_tokens * A.q_heads;
    const int lane = threadIdx.x & 31;
    if (row >= all) return;
    if (A.few_only) {
        const int t = (int)(row / A.q_heads), b = find_seq(A.s, t, 1, 1, 0);
        int first, count;
        new_rows(A.s, b, first, count);
        if (count * A.group <= A.few) return;
    }
    float top = NO_MAX, sum = 0.0f, a[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) a[e] = 0.0f;
    for (int c = 0; c < shares; ++c) {
        const float* p = A.part + (c * all + row) * (D + 4);
        const float2 ml = *reinterpret_cast<const float2*>(p);
        const float now = fmaxf(top, ml.x), f = ex2(top - now), g = ex2(ml.x - now);
        sum = sum * f + ml.y * g;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) {
            const float2 x = *reinterpret_cast<const float2*>(p + 4 + 64 * e + 2 * lane);
            a[2 * e] = a[2 * e] * f + x.x * g;
            a[2 * e + 1] = a[2 * e + 1] * f + x.y * g;
        }
        top = now;
    }
    const float inv = sum == 0.0f ? 0.0f : UNLIFT / sum;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) put_out(A, row * D + 64 * e + 2 * lane, a[2 * e] * inv, a[2 * e + 1] * inv);
    if (A.lse && lane == 0) A.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
}

// The codes of a batch as fp16, [sequence][head][token][dim], tokens up to a whole operand tile (zeros past the pages).
template <int D>
__global__ void __launch_bounds__(256) expand_kernel(const __grid_constant__ AttendArgs A, const int8_t* k, const int8_t* v, __half* kx, __half* vx,
                                                     int tokens) {
    pdl_wait();
    const int b = blockIdx.z, h = blockIdx.y, p0 = blockIdx.x * KEYS;
    const int len = max(0, __ldg(A.s.lens + b)), end = (int)min((long long)len, (long long)A.s.max_pages * A.page);
    if (p0 >= end) return;
    const int* table = A.s.pages + (long long)b * A.s.pages_stride;
    constexpr int CH = D / 16, ALL = KEYS * CH;
#pragma unroll 4
    for (int i = threadIdx.x; i < 2 * ALL; i += 256) {
        const int is_v = i / ALL, row = i % ALL / CH, c = i % CH, p = p0 + row;
        const int pid = p < end ? __ldg(table + p / A.page) : -1;
        uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
        if ((unsigned)pid < (unsigned)A.n_pages) {
            const uint4 w = *reinterpret_cast<const uint4*>((is_v ? v : k) + (((long long)pid * A.heads + h) * A.page + p % A.page) * D + 16 * c);
            uint32_t x = w.x ^ 0x80808080u, y = w.y ^ 0x80808080u;
            lo = make_uint4(code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR));
            x = w.z ^ 0x80808080u, y = w.w ^ 0x80808080u;
            hi = make_uint4(code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR));
        }
        uint4* dst = reinterpret_cast<uint4*>((is_v ? vx : kx) + (((long long)b * A.heads + h) * tokens + p) * D + 16 * c);
        dst[0] = lo;
        dst[1] = hi;
    }
}

bool encode_expanded(CUtensorMap* map, __half* x, int D, long long tokens, long long units) {
    EncodeTiledFn enc = encode_tiled();
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)tokens, (cuuint64_t)units}, strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)(D * tokens * 2)};
    const cuuint32_t box[3] = {64, KEYS, 1}, es[3] = {1, 1, 1};
    return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, x, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

long long expanded_tokens(const AttendArgs& A) { return ((long long)A.s.max_pages * A.page + KEYS - 1) / KEYS * KEYS; }

template <int D, bool PRE>
fxpq_status launch(AttendArgs& A, int shares, cudaStream_t st) {
    static bool set = false;
    if (!set) {
        if (cudaFuncSetAttribute(attend_tile_kernel<D, PRE>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D, PRE>::bytes) != cudaSuccess)
            return FXPQ_ERR_CUDA;
        set = true;
    }
    const long long blocks = tile_blocks(A.s.n_tokens, A.s.n_seqs, A.group, A.s.starts != nullptr);
    if (blocks * A.heads > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    launch_pdl(attend_tile_kernel<D, PRE>, dim3((unsigned)(blocks * A.heads), (unsigned)shares), dim3(threads(PRE)), Smem<D, PRE>::bytes, st, A);
    fxpq_status rc = after_launch("attend_tile");
    if (rc != FXPQ_OK || shares == 1) return rc;
    const long long rows = (long long)A.s.n_tokens * A.q_heads;
    launch_pdl(attend_tile_join_kernel<D>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, A, shares);
    return after_launch("attend_tile_join");
}

template <int D>
fxpq_status launch_expanded(AttendArgs& A, const int8_t* k, const int8_t* v, __half* x, int shares, cudaStream_t st) {
    const long long tokens = expanded_tokens(A), each = (long long)A.s.n_seqs * A.heads * tokens * D;
    launch_pdl(expand_kernel<D>, dim3((unsigned)(tokens / KEYS), (unsigned)A.heads, (unsigned)A.s.n_seqs), dim3(256), 0, st, A, k, v, x, x + each, (int)tokens);
    const fxpq_status rc = after_launch("attend_expand");
    if (rc != FXPQ_OK) return rc;
    if (!encode_expanded(&A.tk, x, D, tokens, (long long)A.s.n_seqs * A.heads) || !encode_expanded(&A.tv, x + each, D, tokens, (long long)A.s.n_seqs * A.heads))
        return FXPQ_ERR_CUDA;
    return launch<D, true>(A, shares, st);
}

}  // namespace

long long tile_blocks(int n_tokens, int n_seqs, int group, bool ragged) {
    return ragged ? unit_base(n_tokens, n_seqs, group, ROWS, 1)
                  : (long long)n_seqs * (((long long)(n_seqs ? n_tokens / n_seqs : 0) * group + ROWS - 1) / ROWS);
}
size_t attend_tile_workspace(int n_tokens, int q_heads, int dim, int shares) {
    return shares > 1 ? (size_t)shares * n_tokens * q_heads * (dim + 4) * sizeof(float) : 0;
}
size_t attend_expand_workspace(int n_seqs, int heads, int dim, long long max_tokens) {
    return (size_t)n_seqs * heads * ((max_tokens + KEYS - 1) / KEYS * KEYS) * dim * 2 * sizeof(__half);
}
fxpq_status launch_attend_tile(AttendArgs& A, int dim, int shares, cudaStream_t st) {
    return dim == 64 ? launch<64, false>(A, shares, st) : launch<128, false>(A, shares, st);
}
fxpq_status launch_attend_tile_expanded(AttendArgs& A, const int8_t* k, const int8_t* v, int dim, void* ws, int shares, cudaStream_t st) {
    return dim == 64 ? launch_expanded<64>(A, k, v, static_cast<__half*>(ws), shares, st)
                     : launch_expanded<128>(A, k, v, static_cast<__half*>(ws), shares, st);
}

}  // namespace llm
}  // namespace fxpq
