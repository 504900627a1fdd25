// fxpq_attend_tile.cu -- attention of many query rows (prompts and chunks) on tcgen05.
//
// A CTA takes 256 query rows (tokens x grouped heads) of one sequence and key head as two tiles of 128 rows and walks
// the keys 128 at a time.  Two products of 128 x 128 x dim per tile and step bound it: S = Q K^T into tensor memory,
// then O += W V with the weights W as the operand in tensor memory, in place of S.  The two tiles alternate, so that one
// tile's products run during the other's exponentials.
//   warps 0-3, 4-7  a tile's softmax each, a thread per row: maximum, weights to fp16, sums (rescaled when the
//                   maximum has grown by 2^8, a few times per row); at the end O / l
//   warps 8-11      converters: codes to fp16 operand tiles, once for both row tiles
//   warp 12         tensor memory, products;   warp 13   pages, scales, copies;   14, 15   none
// Registers are split 184 : 72 between the softmax warps, which keep a row's 128 scores in them, and the others.
// Codes arrive as they are stored ([keys][dim] bytes, one TMA box per page): K is a K-major operand and V, with the
// same bytes, an operand whose columns are contiguous, so that neither is transposed.
#include "fxpq_attend.cuh"

namespace fxpq {
namespace llm {
namespace {

using namespace tc;

constexpr int KEYS = 128, ROWS = 256, THREADS = 16 * 32;
constexpr int TABS = 8;  // scale tables in flight: the copies run at most five steps ahead of the softmax

template <int D>
struct Smem {  // offsets from the 1024-byte aligned base
    static constexpr int Q = 128 * D * 2, CONV = KEYS * D * 2, RAW = KEYS * D;
    static constexpr int conv0 = 2 * Q, raw0 = conv0 + 4 * CONV, bytes = raw0 + 2 * RAW + 1024;
};
static_assert(Smem<128>::bytes + 2048 <= 232448, "shared memory of a CTA");

// Operand whose columns (the rows of O^T) are contiguous: 64 of them in a 128-byte swizzled row, 8 reduction steps to a
// 1024-byte group, the next 64 columns 16 KB on.
__device__ __forceinline__ uint64_t make_sdesc_mn(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)(16384u >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1u << 46 |
           (uint64_t)2u << 61;
}

// Two fp32 values in a register pair, with the packed arithmetic of this architecture.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1) attend_tile_kernel(const __grid_constant__ AttendArgs A) {
    using S = Smem<D>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    __shared__ __align__(8) uint64_t bars[2 + 2 + 4 + 4 + TABS + 2 + 2 + 2 + 1 + 1];
    __shared__ float tab[TABS][3][8];  // per 16 keys: key scale, log2 of the value scale, its inverse
    __shared__ int abort_flag;
    __shared__ uint32_t tmem_slot;
    volatile int* abort = &abort_flag;
    const uint32_t raw_full = smem_u32(bars), raw_empty = raw_full + 16, conv_full = raw_empty + 16, conv_empty = conv_full + 32,
                   tab_full = conv_empty + 32, s_full = tab_full + 8 * TABS, p_full = s_full + 16, o_full = p_full + 16,
                   q_full = o_full + 16, drained = q_full + 8;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(raw_full + 8 * i, 1);
            mbar_init(raw_empty + 8 * i, 4);
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_full + 8 * i, 4);
            mbar_init(o_full + 8 * i, 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(conv_full + 8 * i, 4);
            mbar_init(conv_empty + 8 * i, 1);
        }
        for (int i = 0; i < TABS; ++i) mbar_init(tab_full + 8 * i, 1);
        mbar_init(q_full, 8);
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

    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const uint32_t base = smem_u32(smem);
    // (the launch holds 512 x 128 registers: 256 x 184 + 256 x 72 of them)
    if (warp < 8)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    else
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");

    if (warp < 8) {
        // ================================================================ softmax: one row per thread
        const int t = warp >> 2, quad = warp & 3, r = quad * 32 + lane, rr = rb * ROWS + t * 128 + r, tok = rr / A.group;
        const bool live = t * 128 + r < rows;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16, ts = tmem + 128 * t + lanes, to = tmem + 256 + 128 * t + lanes;
        const long long qrow = (long long)(first + tok) * A.q_token + (long long)(h * A.group + rr - tok * A.group) * A.q_head;
        float cf;
        {
            float top = 0.0f;
            bool odd = false;
            if (live)
#pragma unroll 4
                for (int d = 0; d < D; d += 8) {
                    float x[8];
                    load_q8(A, qrow + d, x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        odd |= !(fabsf(x[e]) <= FLT_MAX);
                        top = fmaxf(top, fabsf(x[e]));
                    }
                }
            const int e = odd ? 0 : q_exponent(top);
            const float up = pow2i(e);
            cf = A.scale * LOG2E * pow2i(-e);
#pragma unroll 4
            for (int d = 0; d < D; d += 8) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = 0.0f;
                if (live) load_q8(A, qrow + d, x);
                *reinterpret_cast<uint4*>(smem + t * S::Q + (d >> 6) * 16384 + r * 128 + ((((d >> 3) & 7) ^ (r & 7)) << 4)) =
                    make_uint4(h2_bits(__floats2half2_rn(x[0] * up, x[1] * up)), h2_bits(__floats2half2_rn(x[2] * up, x[3] * up)),
                               h2_bits(__floats2half2_rn(x[4] * up, x[5] * up)), h2_bits(__floats2half2_rn(x[6] * up, x[7] * up)));
            }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
        if (t < tiles) {
            const int pos = len - count + tok;
            const int limit = !live || pos < 0 ? 0 : A.causal ? min(pos + 1, end) : end;
            float m = NO_MAX, l = 0.0f;
            bool ok = true;
            for (int i = 0; i < n; ++i) {
                const int slot = i % TABS;
                if (!wait_warp(tab_full + 8 * slot, (i / TABS) & 1, abort, A.status) ||
                    !wait_warp(s_full + 8 * t, i & 1, abort, A.status)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const int k0 = (j0 + i) * KEYS, room = limit - k0;  // keys of this step that the row sees
                uint32_t s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32_nw(ts + 32 * c, s[c]);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 4; ++c) reg_fence(s[c]);
                if (__any_sync(0xffffffffu, live && room < KEYS)) {  // the last steps of a row
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[c][e] = 32 * c + e < room ? s[c][e] : 0xff800000u;
                }
                // ---- the largest t, 16 keys (one scale) at a time
                float top = -INFINITY;
#pragma unroll
                for (int g = 0; g < 8; ++g) {
                    const uint32_t* x = s[g >> 1] + 16 * (g & 1);
                    float mx = __uint_as_float(x[0]);
#pragma unroll
                    for (int e = 1; e < 15; e += 2) mx = max3(mx, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                    mx = fmaxf(mx, __uint_as_float(x[15]));
                    top = fmaxf(top, mx == -INFINITY ? mx : fmaf(mx, tab[slot][0][g] * cf, tab[slot][1][g]));
                }
                const bool grow = top > m + LAZY;
                if (__any_sync(0xffffffffu, grow)) {
                    const float f = grow ? ex2(m - top) : 1.0f;
                    m = grow ? top : m;
                    l *= f;
                    if (i > 0) {  // (the products that wrote O are complete: S of this step followed them)
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t o[16];
                            tmem_ld16_nw(to + 16 * c, o);
                            tmem_wait_ld();
                            reg_fence(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                            tmem_st16_nw(to + 16 * c, o);
                        }
                        tmem_wait_st();
                    }
                }
                // ---- weights, in place of S
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const int g = 2 * c + hf;
                        // (FLT_MIN: a page outside the cache has scale 0, which must not meet the -inf of a masked score)
                        const float f = fmaxf(tab[slot][0][g] * cf, FLT_MIN), lv = tab[slot][1][g] - m;
                        const uint64_t f2 = pack2(f, f), lv2 = pack2(lv, lv);
                        uint64_t sum = 0;
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            float x, y;
                            unpack2(fma2(pack2(__uint_as_float(s[c][16 * hf + e]), __uint_as_float(s[c][16 * hf + e + 1])), f2, lv2), x, y);
                            x = ex2(x);
                            y = ex2(y);
                            sum = add2(sum, pack2(x, y));
                            w[8 * hf + e / 2] = h2_bits(__floats2half2_rn(x, y));
                        }
                        float a, b2;
                        unpack2(sum, a, b2);
                        l = fmaf(a + b2, tab[slot][2][g], l);
                    }
                    tmem_st16_nw(ts + 16 * c, w);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * t);
            }
            if (ok && n > 0) ok = wait_warp(o_full + 8 * t, 0, abort, A.status);
            tc_fence_after();
            if (ok) {
                const long long orow = (long long)(first + tok) * A.q_heads + h * A.group + rr - tok * A.group;
                const bool split = gridDim.y > 1;
                float* part = A.part + ((long long)blockIdx.y * A.s.n_tokens * A.q_heads + orow) * (D + 4);
                const float inv = split ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
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
                if (live && split) *reinterpret_cast<float2*>(part) = make_float2(m, l);
                if (live && !split && A.lse) A.lse[orow] = l == 0.0f ? -INFINITY : (m + log2f(l)) * LN2;
            }
        }
    } else if (warp < 12) {
        // ================================================================ converters
        const int t = threadIdx.x - 256;
        for (int u = 0; u < 2 * n; ++u) {  // K 0, V 0, K 1, V 1 ..
            if (!wait_warp(raw_full + 8 * (u & 1), (u >> 1) & 1, abort, A.status) ||
                !wait_warp(conv_empty + 8 * (u & 3), ((u >> 2) & 1) ^ 1, abort, A.status))
                break;
            const unsigned char* src = smem + S::raw0 + (u & 1) * S::RAW;
            unsigned char* dst = smem + S::conv0 + (u & 3) * S::CONV;
            constexpr int CH = D / 16;  // 16-code chunks of a row
#pragma unroll 4
            for (int it = 0; it < KEYS * CH / 128; ++it) {
                const int i = it * 128 + t, row = i / CH, c = i % CH, hf = c >> 2;
                const uint32_t at = D == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
                const uint4 v = *reinterpret_cast<const uint4*>(src + at);
                uint32_t x = v.x ^ 0x80808080u, y = v.y ^ 0x80808080u;
                const uint4 o0 = make_uint4(code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR));
                x = v.z ^ 0x80808080u, y = v.w ^ 0x80808080u;
                const uint4 o1 = make_uint4(code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR));
                unsigned char* d = dst + hf * 16384 + row * 128;
                const int j = 2 * (c & 3), odd = D == 128 ? hf : 0;  // (lanes that would meet in a bank begin with the other chunk)
                *reinterpret_cast<uint4*>(d + (((j + odd) ^ (row & 7)) << 4)) = odd ? o1 : o0;
                *reinterpret_cast<uint4*>(d + (((j + 1 - odd) ^ (row & 7)) << 4)) = odd ? o0 : o1;
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(raw_empty + 8 * (u & 1));
                mbar_arrive(conv_full + 8 * (u & 3));
            }
        }
    } else if (warp == 12) {
        // ================================================================ products
        const uint32_t id_qk = make_idesc(128, KEYS), id_pv = make_idesc(128, D) | (1u << 16);
        bool ok = wait_warp(q_full, 0, abort, A.status);
        auto scores = [&](int t, int i) {
            const uint64_t qd = make_sdesc(base + t * S::Q), kd = make_sdesc(base + S::conv0 + ((2 * i) & 3) * S::CONV);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
                tc_mma(tmem + 128 * t, qd + (kk >> 2) * (16384 >> 4) + 2 * (kk & 3), kd + (kk >> 2) * (16384 >> 4) + 2 * (kk & 3), id_qk, kk > 0);
        };
        if (ok && n > 0 && wait_warp(conv_full, 0, abort, A.status)) {
            tc_fence_after();
            for (int t = 0; t < tiles; ++t) {
                scores(t, 0);
                tc_commit(s_full + 8 * t);
            }
            tc_commit(conv_empty);
            for (int i = 0; i < n && ok; ++i) {
                const int uv = (2 * i + 1) & 3, uk = (2 * i + 2) & 3;
                if (!wait_warp(conv_full + 8 * uv, ((2 * i + 1) >> 2) & 1, abort, A.status)) break;
                const uint64_t vd = make_sdesc_mn(base + S::conv0 + uv * S::CONV);
                for (int t = 0; t < tiles; ++t) {
                    if (!wait_warp(p_full + 8 * t, i & 1, abort, A.status)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int kk = 0; kk < KEYS / 16; ++kk)
                        tc_mma_ta(tmem + 256 + 128 * t, tmem + 128 * t + 8 * kk, vd + kk * (2048 >> 4), id_pv, i > 0 || kk > 0);
                    if (t == tiles - 1) tc_commit(conv_empty + 8 * uv);
                    if (i + 1 < n) {
                        if (t == 0 && !wait_warp(conv_full + 8 * uk, ((2 * i + 2) >> 2) & 1, abort, A.status)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        scores(t, i + 1);
                        tc_commit(s_full + 8 * t);
                        if (t == tiles - 1) tc_commit(conv_empty + 8 * uk);
                    } else
                        tc_commit(o_full + 8 * t);
                }
            }
        }
        tc_commit(drained);  // every product issued here has completed once it fires
        drain_warp(drained, 0);
    } else if (warp == 13) {
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
                const float lv = cur.vs > 0.0f ? __log2f(cur.vs) : -INFINITY;
                tab[slot][0][lane - from] = cur.ks;
                tab[slot][1][lane - from] = lv;
                tab[slot][2][lane - from] = cur.vs > 0.0f ? ex2(-lv) : 0.0f;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(tab_full + 8 * slot);
            const unsigned have = __ballot_sync(0xffffffffu, cur.pid >= 0) >> from;
            int boxes = 0;
            for (int g = 0; g < 8; g += box / 16) boxes += (have >> g) & 1;
            for (int v = 0; v < 2; ++v, ++u) {
                const uint32_t bar = raw_full + 8 * (u & 1), dst = base + S::raw0 + (u & 1) * S::RAW;
                if (!wait_warp(raw_empty + 8 * (u & 1), ((u >> 1) & 1) ^ 1, abort, A.status)) {
                    ok = false;
                    break;
                }
                mbar_arrive_expect_tx(bar, (uint32_t)(boxes * box * D));
                for (int g = 0; g < 8; g += box / 16) {
                    const int pid = __shfl_sync(0xffffffffu, cur.pid, from + g);
                    if (pid >= 0) tma_load_3d(dst + 16 * g * D, v ? &A.tv : &A.tk, 0, 0, pid * A.heads + h, bar);
                }
            }
            if ((i & 3) == 3) {
                cur = nxt;
                nxt = fetch(i + 5);
            }
        }
        for (int k = max(0, u - 2); k < u; ++k) {  // every copy has landed
            drain_warp(raw_full + 8 * (k & 1), (k >> 1) & 1);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
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
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) put_out(A, row * D + 64 * e + 2 * lane, a[2 * e] * inv, a[2 * e + 1] * inv);
    if (A.lse && lane == 0) A.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
}

template <int D>
fxpq_status launch(AttendArgs& A, int shares, cudaStream_t st) {
    static bool set = false;
    if (!set) {
        if (cudaFuncSetAttribute(attend_tile_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D>::bytes) != cudaSuccess)
            return FXPQ_ERR_CUDA;
        set = true;
    }
    const long long blocks = tile_blocks(A.s.n_tokens, A.s.n_seqs, A.group, A.s.starts != nullptr);
    if (blocks * A.heads > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    launch_pdl(attend_tile_kernel<D>, dim3((unsigned)(blocks * A.heads), (unsigned)shares), dim3(THREADS), Smem<D>::bytes, st, A);
    fxpq_status rc = after_launch("attend_tile");
    if (rc != FXPQ_OK || shares == 1) return rc;
    const long long rows = (long long)A.s.n_tokens * A.q_heads;
    launch_pdl(attend_tile_join_kernel<D>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, A, shares);
    return after_launch("attend_tile_join");
}

}  // namespace

long long tile_blocks(int n_tokens, int n_seqs, int group, bool ragged) {
    return ragged ? unit_base(n_tokens, n_seqs, group, ROWS, 1)
                  : (long long)n_seqs * (((long long)(n_seqs ? n_tokens / n_seqs : 0) * group + ROWS - 1) / ROWS);
}
size_t attend_tile_workspace(int n_tokens, int q_heads, int dim, int shares) {
    return shares > 1 ? (size_t)shares * n_tokens * q_heads * (dim + 4) * sizeof(float) : 0;
}
fxpq_status launch_attend_tile(AttendArgs& A, int dim, int shares, cudaStream_t st) {
    return dim == 64 ? launch<64>(A, shares, st) : launch<128>(A, shares, st);
}

}  // namespace llm
}  // namespace fxpq
