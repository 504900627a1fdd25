// fxpq_attend_stream.cu -- attention of few query rows (decoding): the cache is read once, at the memory's rate.
//
// A unit is one sequence, one key head and up to 8 NT query rows (tokens x grouped heads).  Bytes bound it: 2 dim
// per token against 4 dim multiply-adds per row.  tcgen05 would want 128 rows, and codes expanded to fp16 in shared
// memory cost six bytes of its traffic per code (23 codes per cycle and SM arrive, it moves 128 bytes); here a code
// is written and read there once, expanded in registers, and multiplied by warp-level m16n8k16 products with the
// tokens on the 16-row side, so that 8 query rows fill a product.
//
// Every warp streams tiles of 32 tokens through its own ring of TMA boxes (no barrier between warps until the unit
// ends) and keeps its own running maximum, sum and 8 NT x dim sums.  S^T = K q^T: the operand's registers are bytes of
// a row of K, with the reduction's order permuted alike for q so that a thread's bytes are consecutive.  O^T = V^T w^T:
// w^T is S^T's registers transposed by movmatrix, V^T two rows' bytes interleaved.  Rows of a tile are assigned to
// the product's rows in an order in which neither read has bank conflicts under the TMA's swizzle.
#include "fxpq_attend.cuh"

namespace fxpq {
namespace llm {
namespace {

using namespace tc;

constexpr int TILE = 32;          // tokens of a stage
constexpr int WARPS = 4;
// CTAs of an SM (one streams while another merges) and the bytes of stages of each.  With 8 rows a unit three of them fit
// the registers: a warp's chain of loads, products and exponentials leaves the SM's issue slots half empty with two.
__host__ __device__ constexpr int ctas_of(int NT) { return NT == 1 ? 3 : 2; }
__host__ __device__ constexpr int ring_of(int NT) { return (NT == 1 ? 64 : 96) * 1024; }

template <int D, int NT>
__host__ __device__ constexpr int stages() { return ring_of(NT) / WARPS / (TILE * D * 2); }

// Row of a 16-token half tile that product row g (and g + 8: eight rows on) stands for.
template <int D>
__device__ __forceinline__ int row_of(int g) {
    // D = 128: pairs (2 i, 2 i + 1) differ in bit 2, rows 0 2 4 6 and 1 3 5 7 differ beyond bit 0;
    // D = 64: pairs differ in bit 0, rows 0 2 4 6 and 1 3 5 7 differ in bits 0 and 2
    constexpr uint32_t order = D == 128 ? 0x37156240u : 0x65742130u;
    return (order >> (4 * g)) & 7;
}
// Byte offset of 16-byte chunk c of a stage's row r under the swizzle of its row size.
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
    return D == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two weights as fp16, the first in the low half.  They are at most 2^15, but past 2^15 where scores are so large that
// m + LAZY + LIFT rounds up (from 2^27 on fp32's steps are 16), and must not become infinite there.
__device__ __forceinline__ uint32_t weight_pair(float a, float b) {
    uint32_t w;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}

// Work of a batch in tiles.  Sequence b has blocks_b row blocks (0 where it is not this kernel's) of heads units, each
// of tiles_b tiles; units lie one after the other, sequences outermost, then heads, then row blocks.
struct Seq {
    int first, count, len, end, tiles, blocks;  // end: the tokens that its pages hold
};
template <int NT>
__device__ __forceinline__ Seq seq_of(const AttendArgs& A, int b) {
    Seq q;
    new_rows(A.s, b, q.first, q.count);
    q.len = max(0, __ldg(A.s.lens + b));
    q.end = (int)min((long long)q.len, (long long)A.s.max_pages * A.page);
    const long long rows = (long long)q.count * A.group;
    q.blocks = rows > 0 && rows <= A.few ? (int)((rows + 8 * NT - 1) / (8 * NT)) : 0;
    q.tiles = max(1, (int)(((long long)q.end + TILE - 1) / TILE));  // (a sequence without tokens has a unit that writes zeros)
    return q;
}
// The sequence that tile w of the whole batch belongs to and the batch's tiles before it; w < 0: the total alone.  A whole
// warp.
template <int NT>
__device__ __forceinline__ int find_tile(const AttendArgs& A, long long w, long long& before) {
    const int lane = threadIdx.x & 31;
    long long base = 0;
    for (int b0 = 0; b0 < A.s.n_seqs; b0 += 32) {
        long long n = 0;
        if (b0 + lane < A.s.n_seqs) {
            const Seq q = seq_of<NT>(A, b0 + lane);
            n = (long long)q.blocks * q.tiles * A.heads;
        }
        long long up = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, up, d);
            if (lane >= d) up += o;
        }
        const unsigned in = __ballot_sync(0xffffffffu, w >= 0 && n > 0 && w >= base + up - n && w < base + up);
        if (in) {
            const int l = __ffs(in) - 1;
            before = base + __shfl_sync(0xffffffffu, up - n, l);
            return b0 + l;
        }
        base += __shfl_sync(0xffffffffu, up, 31);
    }
    before = base;
    return -1;
}
__device__ __forceinline__ long long share_of(const AttendArgs& A, long long total, int ctas) {
    const long long s = (total + ctas - 1) / ctas;
    return s > A.share_min ? s : A.share_min;
}

// Partial results: per CTA two slots (a unit that began before its share: 0, one that goes on after it: 1) of 8 NT rows of
// dim sums, maximum and normaliser.
template <int D, int NT>
__device__ __forceinline__ float* slot_at(const AttendArgs& A, int cta, int slot) {
    return A.part + (long long)(2 * cta + slot) * (8 * NT) * (D + 2);
}

template <int D, int NT>
__global__ void __launch_bounds__(32 * WARPS, ctas_of(NT)) attend_stream_kernel(const __grid_constant__ AttendArgs A) {
    constexpr int ST = stages<D, NT>(), STAGE = TILE * D * 2, KS = D / 16, MT = D / 16;
    constexpr bool QREG = NT <= 2;  // query fragments in registers; the widest instance keeps them in shared memory
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    __shared__ __align__(8) uint64_t bars[WARPS * ST];
    __shared__ int abort_flag;
    __shared__ float s_m[WARPS][8 * NT], s_l[WARPS][8 * NT];
    __shared__ uint2 s_q[QREG ? 1 : KS * NT * 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, tig = lane & 3;
    const uint32_t ring = smem_u32(smem) + warp * ST * STAGE, bar0 = smem_u32(bars + warp * ST);
    volatile int* abort = &abort_flag;
    if (lane == 0) {
        for (int i = 0; i < ST; ++i) mbar_init(bar0 + 8 * i, 1);
        if (warp == 0) abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        prefetch_tmap(&A.tk);
        prefetch_tmap(&A.tv);
    }
    pdl_wait();
    __syncthreads();

    // this CTA's part of the batch: [w, w_end) in tiles, starting in sequence b
    long long w, w_end, seq_base;
    int b;
    Seq q;
    if (A.whole) {  // one unit
        const int per_seq = A.heads;
        // (units of a whole launch: row block by row block of each sequence, see unit_base)
        const long long x = blockIdx.x / per_seq;
        const int h = (int)(blockIdx.x - x * per_seq);
        b = A.s.starts ? find_seq(A.s, x, A.group, 8 * NT, 1) : (int)(x / ((A.s.each * A.group + 8 * NT - 1) / (8 * NT)));
        q = seq_of<NT>(A, b);
        const int rb = (int)(x - (A.s.starts ? unit_base(max(__ldg(A.s.starts + b), 0), b, A.group, 8 * NT, 1)
                                              : (long long)b * ((A.s.each * A.group + 8 * NT - 1) / (8 * NT))));
        if (rb < 0 || rb >= q.blocks) return;
        seq_base = 0;
        w = ((long long)h * q.blocks + rb) * q.tiles;
        w_end = w + q.tiles;
    } else {
        long long total;
        find_tile<NT>(A, -1, total);
        const long long share = share_of(A, total, gridDim.x);
        w = share * blockIdx.x;
        w_end = min(total, w + share);
        if (w >= w_end) return;
        b = find_tile<NT>(A, w, seq_base);
        q = seq_of<NT>(A, b);
    }
    const long long w_begin = w;
    uint32_t filled = 0, used = 0;  // stages of this warp's ring, counted on over all units
    bool ok = true;
    while (w < w_end && ok) {
        while (w - seq_base >= (long long)q.blocks * q.tiles * A.heads) {  // the next sequence
            seq_base += (long long)q.blocks * q.tiles * A.heads;
            q = seq_of<NT>(A, ++b);
        }
        const long long in_seq = w - seq_base;
        const int unit = (int)(in_seq / q.tiles), t_lo = (int)(in_seq - (long long)unit * q.tiles);
        const int h = unit / q.blocks, rb = unit - h * q.blocks;
        const int t_hi = (int)min((long long)q.tiles, t_lo + (w_end - w));
        const int rows = min(8 * NT, q.count * A.group - rb * 8 * NT);
        if (q.end < q.len && threadIdx.x == 0) latch_status(A.status, FXPQ_ERR_RANGE);

        // ---- this warp's tiles t_lo + warp, + WARPS ..: pages and scales of 32 of them at a time, one per lane
        const int* table = A.s.pages + (long long)b * A.s.pages_stride;
        const bool two = A.page < TILE;  // two pages to a tile
        struct Info {
            int pid[2];
            float ks[2], vs[2];
        };
        auto fetch = [&](int j0) {
            Info f;
            const int tile = t_lo + warp + WARPS * (j0 + lane);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int p = tile * TILE + 16 * i, pi = p / A.page;
                int id = -1;
                if (tile < t_hi && p < q.end && (i == 0 || two)) {
                    id = __ldg(table + pi);
                    if ((unsigned)id >= (unsigned)A.n_pages) {
                        latch_status(A.status, FXPQ_ERR_RANGE);
                        id = -1;
                    }
                }
                f.pid[i] = id;
                f.ks[i] = id < 0 ? 0.0f : __ldg(A.k_scale + (long long)id * A.heads + h);
                f.vs[i] = id < 0 ? 0.0f : __ldg(A.v_scale + (long long)id * A.heads + h);
            }
            return f;
        };
        const int n_mine = t_hi - t_lo > warp ? (t_hi - t_lo - warp + WARPS - 1) / WARPS : 0;
        Info cur = fetch(0), nxt = fetch(32);
        auto issue = [&](int j, const Info& f) {  // tile j of this warp into the ring's next stage
            const int p0 = __shfl_sync(0xffffffffu, f.pid[0], j & 31), p1 = __shfl_sync(0xffffffffu, f.pid[1], j & 31);
            const uint32_t s = filled % ST, bar = bar0 + 8 * s, dst = ring + s * STAGE;
            ++filled;
            const int boxes = (p0 >= 0) + (two && p1 >= 0), bytes = min(A.page, TILE) * D * 2;
            mbar_arrive_expect_tx(bar, (uint32_t)(boxes * bytes));
            const int at = two ? 0 : (t_lo + warp + WARPS * j) * TILE % A.page;
            if (p0 >= 0) {
                tma_load_3d(dst, &A.tk, 0, at, p0 * A.heads + h, bar);
                tma_load_3d(dst + TILE * D, &A.tv, 0, at, p0 * A.heads + h, bar);
            }
            if (two && p1 >= 0) {
                tma_load_3d(dst + 16 * D, &A.tk, 0, 0, p1 * A.heads + h, bar);
                tma_load_3d(dst + TILE * D + 16 * D, &A.tv, 0, 0, p1 * A.heads + h, bar);
            }
        };
        int issued = 0;
        for (; issued < min(ST - 1, n_mine); ++issued) issue(issued, cur);

        // ---- query fragments: row nt 8 + g, 16 values from 16 tig (and 64 + 16 tig)
        uint32_t qf[QREG ? KS : 1][QREG ? NT : 1][2];
        float cf[NT][2];     // log2(e) * scale / (the row's power of two), of the two columns 2 tig, 2 tig + 1
        int limit[NT][2];    // keys before this position are seen
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = nt * 8 + g, rr = rb * 8 * NT + r, i = rr / A.group;
            float v[D / 64][16], top = 0.0f;
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float x[8];
                    if (r < rows)
                        load_q8(A, (long long)(q.first + i) * A.q_token + (long long)(h * A.group + rr - i * A.group) * A.q_head + 64 * c + 16 * tig + 8 * u, x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[c][8 * u + e] = r < rows ? x[e] : 0.0f;
                        const float ax = fabsf(v[c][8 * u + e]);
                        top = ax > top || ax != ax ? ax : top;
                    }
                }
            bool odd = !(top <= FLT_MAX);
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                odd |= __shfl_xor_sync(0xffffffffu, (int)odd, d) != 0;
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            }
            const int e = odd ? 0 : q_exponent(top);
            const float up = pow2i(e), c0 = A.scale * LOG2E * pow2i(-e);
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const uint32_t x = h2_bits(__floats2half2_rn(v[c][4 * s] * up, v[c][4 * s + 1] * up));
                    const uint32_t y = h2_bits(__floats2half2_rn(v[c][4 * s + 2] * up, v[c][4 * s + 3] * up));
                    if constexpr (QREG) {
                        qf[4 * c + s][nt][0] = x;
                        qf[4 * c + s][nt][1] = y;
                    } else if (warp == 0)
                        s_q[((4 * c + s) * NT + nt) * 32 + lane] = make_uint2(x, y);
                }
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) {
                cf[nt][e2] = __shfl_sync(0xffffffffu, c0, 4 * (2 * tig + e2));
                const int rc = rb * 8 * NT + nt * 8 + 2 * tig + e2, pos = q.len - q.count + rc / A.group;
                limit[nt][e2] = pos < 0 ? 0 : A.causal ? min(pos + 1, q.end) : q.end;
            }
        }
        if constexpr (!QREG) __syncthreads();  // (the previous unit ended with one too)
        const int first_pos = q.len - q.count + rb * 8 * NT / A.group;
        const int free_of_mask = first_pos < 0 ? 0 : A.causal ? min(first_pos + 1, q.end) : q.end;  // every row sees all keys before this

        float m[NT][2], l[NT][2], o[MT][NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = NO_MAX;
            l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][nt][e] = 0.0f;
        }
        for (int j = 0; j < n_mine && ok; ++j) {
            const uint32_t s = used % ST;
            if (!wait_warp(bar0 + 8 * s, (used / ST) & 1, abort, A.status)) {
                ok = false;
                break;
            }
            ++used;
            if (issued < n_mine) {  // into the stage read one tile ago (every lane is past it)
                issue(issued, issued / 32 == j / 32 ? cur : nxt);
                ++issued;
            }
            const uint32_t sk = ring + s * STAGE, sv = sk + TILE * D;
            // ---- scores of 32 tokens
            float c[2][NT][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[mt][nt][e] = 0.0f;
                const int r0 = 16 * mt + row_of<D>(g);
#pragma unroll
                for (int hf = 0; hf < D / 64; ++hf) {
                    const uint4 x = lds128(sk + chunk_at<D>(r0, tig + 4 * hf)), y = lds128(sk + chunk_at<D>(r0 + 8, tig + 4 * hf));
                    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {
                        const uint32_t u = xs[ks] ^ 0x80808080u, v = ys[ks] ^ 0x80808080u;
                        const uint32_t a[4] = {code_pair(u, LOW_PAIR), code_pair(v, LOW_PAIR), code_pair(u, HIGH_PAIR), code_pair(v, HIGH_PAIR)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            if constexpr (QREG) {
                                mma16816(c[mt][nt], a, qf[4 * hf + ks][nt][0], qf[4 * hf + ks][nt][1]);
                            } else {
                                const uint2 b2 = s_q[((4 * hf + ks) * NT + nt) * 32 + lane];
                                mma16816(c[mt][nt], a, b2.x, b2.y);
                            }
                        }
                    }
                }
            }
            // ---- t + LIFT, the lazily followed maximum, weights
            const int tile = t_lo + warp + WARPS * j, src = j & 31;
            float ks[2], lv[2], iv[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float k = __shfl_sync(0xffffffffu, i && two ? cur.ks[1] : cur.ks[0], src);
                const float v = __shfl_sync(0xffffffffu, i && two ? cur.vs[1] : cur.vs[0], src);
                ks[i] = k;
                lv[i] = v > 0.0f ? __log2f(v) + LIFT : -INFINITY;
                iv[i] = v > 0.0f ? ex2(-lv[i]) : 0.0f;
            }
            const bool masked = tile * TILE + TILE > free_of_mask;
            bool over = false;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float t = fmaf(c[mt][nt][e], ks[mt] * cf[nt][e & 1], lv[mt]);
                        if (masked && tile * TILE + 16 * mt + row_of<D>(g) + 8 * (e >> 1) >= limit[nt][e & 1]) t = -INFINITY;
                        c[mt][nt][e] = t;
                        over |= t > m[nt][e & 1] + (LAZY + LIFT);
                    }
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(fmaxf(c[0][nt][e], c[0][nt][e + 2]), fmaxf(c[1][nt][e], c[1][nt][e + 2]));
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        if (top > m[nt][e] + (LAZY + LIFT)) {
                            const float now = top - LIFT, f = ex2(m[nt][e] - now);
                            m[nt][e] = now;
                            l[nt][e] *= f;
#pragma unroll
                            for (int i = 0; i < MT; ++i) {
                                o[i][nt][e] *= f;
                                o[i][nt][e + 2] *= f;
                            }
                        }
                    }
            }
            uint32_t wt[2][NT][2];  // weights, tokens along the reduction
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = ex2(c[mt][nt][e] - m[nt][e & 1]);
                    l[nt][0] = fmaf(p[0] + p[2], iv[mt], l[nt][0]);
                    l[nt][1] = fmaf(p[1] + p[3], iv[mt], l[nt][1]);
                    wt[mt][nt][0] = transpose8x8(weight_pair(p[0], p[1]));
                    wt[mt][nt][1] = transpose8x8(weight_pair(p[2], p[3]));
                }
            // ---- values: four rows of this thread, their bytes interleaved by pairs of rows
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                uint32_t v[4][D / 32];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 16 * mt + row_of<D>(2 * tig + (i & 1)) + 8 * (i >> 1);
                    if constexpr (D == 128) {
                        const uint4 x = lds128(sv + chunk_at<D>(r, g));
                        v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
                    } else {
                        const uint2 x = lds64(sv + chunk_at<D>(r, g >> 1) + 8 * (g & 1));
                        v[i][0] = x.x, v[i][1] = x.y;
                    }
                }
#pragma unroll
                for (int u = 0; u < D / 32; ++u)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t sel = half ? 0x7362 : 0x5140;
                        const uint32_t x = __byte_perm(v[0][u], v[1][u], sel) ^ 0x80808080u;
                        const uint32_t y = __byte_perm(v[2][u], v[3][u], sel) ^ 0x80808080u;
                        const uint32_t a[4] = {code_pair(x, LOW_PAIR), code_pair(x, HIGH_PAIR), code_pair(y, LOW_PAIR), code_pair(y, HIGH_PAIR)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16816(o[2 * u + half][nt], a, wt[mt][nt][0], wt[mt][nt][1]);
                    }
            }
            if ((j & 31) == 31) {
                cur = nxt;
                nxt = fetch(j + 33);
            }
        }
        // ---- the warps' results together, through the ring's memory
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], d);
                if (g == 0) {
                    s_m[warp][nt * 8 + 2 * tig + e] = m[nt][e];
                    s_l[warp][nt * 8 + 2 * tig + e] = l[nt][e];
                }
            }
        __syncthreads();
        if (abort_flag) ok = false;
        float* sums = reinterpret_cast<float*>(smem);  // [WARPS][8 NT][D + 4]
        constexpr int PITCH = D + 4;
        static_assert(WARPS * 8 * NT * PITCH * 4 <= ring_of(NT), "merge buffer within the ring");
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = nt * 8 + 2 * tig + e;
                float top = s_m[0][r];
#pragma unroll
                for (int i = 1; i < WARPS; ++i) top = fmaxf(top, s_m[i][r]);
                const float f = ex2(m[nt][e] - top);
                float* dst = sums + (warp * 8 * NT + r) * PITCH + (D / 8) * g;
#pragma unroll
                for (int i = 0; i < MT; ++i) *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(o[i][nt][e] * f, o[i][nt][e + 2] * f);
            }
        __syncthreads();
        const bool complete = t_lo == 0 && t_hi == q.tiles;
        float* part = complete ? nullptr : slot_at<D, NT>(A, blockIdx.x, w == w_begin && t_lo > 0 ? 0 : 1);
        for (int i = threadIdx.x; i < rows * (D / 2); i += 32 * WARPS) {
            const int r = i / (D / 2), d = 2 * (i - r * (D / 2));
            float top = s_m[0][r], sum = 0.0f, a = 0.0f, c2 = 0.0f;
#pragma unroll
            for (int k = 1; k < WARPS; ++k) top = fmaxf(top, s_m[k][r]);
#pragma unroll
            for (int k = 0; k < WARPS; ++k) {
                const float2 x = *reinterpret_cast<const float2*>(sums + (k * 8 * NT + r) * PITCH + d);
                a += x.x;
                c2 += x.y;
                sum = fmaf(s_l[k][r], ex2(s_m[k][r] - top), sum);
            }
            if (complete) {
                const int rr = rb * 8 * NT + r, tok = rr / A.group;
                const long long row = (long long)(q.first + tok) * A.q_heads + h * A.group + rr - tok * A.group;
                const float inv = sum == 0.0f ? 0.0f : UNLIFT / sum;
                put_out(A, row * D + d, a * inv, c2 * inv);
                if (A.lse && d == 0) A.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
            } else {
                *reinterpret_cast<float2*>(part + r * (D + 2) + 2 + d) = make_float2(a, c2);
                if (d == 0) *reinterpret_cast<float2*>(part + r * (D + 2)) = make_float2(top, sum);
            }
        }
        fence_proxy_async();  // (the ring's memory goes back to the copies)
        __syncthreads();
        w += t_hi - t_lo;
    }
    // every copy that this warp issued has landed before it leaves (it has, unless a wait ran out)
    for (; used < filled; ++used) {
        drain_warp(bar0 + 8 * (used % ST), (used / ST) & 1);
    }
}

// Units that several CTAs shared: one warp per new token and query head.
template <int D, int NT>
__global__ void __launch_bounds__(128) attend_join_kernel(const __grid_constant__ AttendArgs A, int ctas) {
    pdl_wait();
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= (long long)A.s.n_tokens * A.q_heads) return;
    const int t = (int)(row / A.q_heads), hq = (int)(row - (long long)t * A.q_heads), h = hq / A.group;
    const int b = A.s.starts ? find_seq(A.s, t, 1, 1, 0) : t / A.s.each;
    const Seq q = seq_of<NT>(A, b);
    const int i = t - q.first;
    if (q.blocks == 0 || i < 0 || i >= q.count) return;
    long long total, base = 0;
    find_tile<NT>(A, -1, total);
    const long long share = share_of(A, total, ctas);
    {  // the batch's tiles before sequence b
        for (int b0 = 0; b0 < b; b0 += 32) {
            long long n = 0;
            if (b0 + lane < b) {
                const Seq p = seq_of<NT>(A, b0 + lane);
                n = (long long)p.blocks * p.tiles * A.heads;
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
            base += n;
        }
    }
    const int rr = i * A.group + hq - h * A.group, rb = rr / (8 * NT), r = rr - rb * 8 * NT;
    const long long lo = base + ((long long)h * q.blocks + rb) * q.tiles, hi = lo + q.tiles;
    const int c0 = (int)(lo / share), c1 = (int)((hi - 1) / share);
    if (c0 == c1) return;
    float top = NO_MAX, sum = 0.0f, a[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) a[e] = 0.0f;
    for (int c = c0; c <= c1; ++c) {
        // (the CTA in whose share the unit begins wrote slot 1, unless it begins with the share: then slot 1 as well)
        const float* p = slot_at<D, NT>(A, c, c == c0 ? 1 : 0) + r * (D + 2);
        const float2 ml = *reinterpret_cast<const float2*>(p);
        const float now = fmaxf(top, ml.x), f = ex2(top - now), g = ex2(ml.x - now);
        sum = sum * f + ml.y * g;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) {
            const float2 x = *reinterpret_cast<const float2*>(p + 2 + 64 * e + 2 * lane);
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

template <int D, int NT>
fxpq_status launch(AttendArgs& A, bool whole, cudaStream_t st) {
    static bool set = false;  // (setting it twice does no harm)
    if (!set) {
        if (cudaFuncSetAttribute(attend_stream_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_of(NT) + 1024) != cudaSuccess)
            return FXPQ_ERR_CUDA;
        set = true;
    }
    A.whole = whole;
    A.share_min = 16;
    const int ctas = ctas_of(NT) * num_sms();
    long long grid = ctas;
    if (whole)
        grid = A.heads * (A.s.starts ? unit_base(A.s.n_tokens, A.s.n_seqs, A.group, 8 * NT, 1)
                                     : (long long)A.s.n_seqs * ((A.s.each * A.group + 8 * NT - 1) / (8 * NT)));
    if (grid > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    launch_pdl(attend_stream_kernel<D, NT>, dim3((unsigned)grid), dim3(32 * WARPS), ring_of(NT) + 1024, st, A);
    fxpq_status rc = after_launch("attend_stream");
    if (rc != FXPQ_OK || whole) return rc;
    const long long rows = (long long)A.s.n_tokens * A.q_heads;
    launch_pdl(attend_join_kernel<D, NT>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, A, ctas);
    return after_launch("attend_join");
}

}  // namespace

int stream_nt(long long rows) { return rows <= 8 ? 1 : rows <= 16 ? 2 : 4; }

size_t attend_stream_workspace(int dim, int nt) {
    return (size_t)2 * ctas_of(nt) * num_sms() * 8 * nt * (dim + 2) * sizeof(float);
}

fxpq_status launch_attend_stream(AttendArgs& A, int dim, int nt, bool whole, cudaStream_t st) {
    if (dim == 64) return nt == 1 ? launch<64, 1>(A, whole, st) : nt == 2 ? launch<64, 2>(A, whole, st) : launch<64, 4>(A, whole, st);
    return nt == 1 ? launch<128, 1>(A, whole, st) : nt == 2 ? launch<128, 2>(A, whole, st) : launch<128, 4>(A, whole, st);
}

}  // namespace llm
}  // namespace fxpq
