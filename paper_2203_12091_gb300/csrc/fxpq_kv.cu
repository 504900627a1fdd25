// fxpq_kv.cu -- the paged cache of 8-bit keys and values: appending with the position rotation, reading back.
#include <cfloat>

#include "fxpq_llm.cuh"
#include "fxpq_ptx.cuh"

namespace fxpq {
namespace llm {

bool batch_ok(const fxpq_kv_batch* b) {
    return b && b->n_seqs >= 0 && b->n_tokens >= 0 && b->max_pages >= 0 && b->pages_stride >= b->max_pages &&
           (b->n_seqs == 0 ? b->n_tokens == 0 : (b->d_pages || b->max_pages == 0) && b->d_lens != nullptr) &&
           (b->d_starts || b->n_seqs == 0 || b->n_tokens % b->n_seqs == 0) && aligned(b->d_pages, 4) && aligned(b->d_lens, 4) &&
           aligned(b->d_starts, 4);
}
bool cache_ok(const fxpq_kv_cache* c) {
    return c && c->n_pages > 0 && c->heads > 0 && c->d_k && c->d_v && c->d_k_scale && c->d_v_scale && aligned(c->d_k, 16) &&
           aligned(c->d_v, 16) && aligned(c->d_k_scale, 4) && aligned(c->d_v_scale, 4) &&
           (c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128) &&
           (c->dim == 64 || c->dim == 128);
}

namespace {

constexpr int FL_LO = -32, FL_HI = 40;

struct AppendArgs {
    Seqs s;
    fxpq_kv_cache c;
    const void *k, *v, *q;
    long long k_token, k_head, v_token, v_head, q_token, q_head;
    void* q_out;
    const float *cos_t, *sin_t;
    int q_heads, n_pos, rot, inter, vec, vec16;  // aligned to four elements; keys and values to 16 bytes
    int per_seq, units;  // pages that a sequence's new tokens may touch (uniform batches), in all
    int kinds;           // work units of a page
    int* status;
};

__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }  // -126 <= e <= 127

// The smallest 2^-FL, FL in [FL_LO, FL_HI], with a <= 127 * 2^-FL: a = m 2^e with m in [1, 2) gives
// FL = 6 - e where m <= 127 / 64, else 5 - e.
__device__ __forceinline__ float block_scale(float a) {
    const int bits = __float_as_int(a), e = (bits >> 23) - 127;  // (zero and subnormals: e = -127)
    int fl = 6 - e - ((bits & 0x7fffff) > 0x7e0000);
    fl = min(max(fl, FL_LO), FL_HI);
    return pow2(-fl);
}

// One multiplication by the inverse where it is exact (a scale that is a power of two), else a division.
struct Divider {
    float s, inv;
    bool exact;
    __device__ __forceinline__ explicit Divider(float scale) : s(scale) {
        const int bits = __float_as_int(scale), e = bits >> 23;
        exact = (bits & 0x7fffff) == 0 && e >= 1 && e <= 253;
        inv = exact ? __int_as_float((254 - e) << 23) : 0.0f;
    }
    __device__ __forceinline__ float operator()(float x) const { return exact ? x * inv : __fdiv_rn(x, s); }
};

__device__ __forceinline__ int code_of(float x) {  // rounded half to even, clipped
    return max(-128, min(127, __float2int_rn(x)));
}

// Eight values of a head: octet j of `rot / 8` rotated ones is the four pairs 4 j .., the others are values 8 j ..
// lo: the offset of the first four, hi of the others.
__device__ __forceinline__ void octet_at(int j, int rot, int inter, int& lo, int& hi) {
    const bool half = 8 * j < rot && !inter;
    lo = half ? 4 * j : 8 * j;
    hi = half ? rot / 2 + 4 * j : 8 * j + 4;
}

// Cosines and sines of octet o's four pairs at a position.
__device__ __forceinline__ void load_turn(const AppendArgs& A, int pos, int o, float (&c)[4], float (&s)[4]) {
    if (8 * o >= A.rot) return;
    const long long at = (long long)pos * (A.rot / 2) + 4 * o;
    const float4 c4 = *reinterpret_cast<const float4*>(A.cos_t + at), s4 = *reinterpret_cast<const float4*>(A.sin_t + at);
    c[0] = c4.x, c[1] = c4.y, c[2] = c4.z, c[3] = c4.w;
    s[0] = s4.x, s[1] = s4.y, s[2] = s4.z, s[3] = s4.w;
}
// The octet's pairs (a[i], b[i]), or interleaved (x[2 i], x[2 i + 1]) of a, b = x[0 .. 3], x[4 .. 7], turned: every product and
// sum rounded to fp32.
__device__ __forceinline__ void turn(float (&a)[4], float (&b)[4], const float (&c)[4], const float (&s)[4], int inter) {
    auto pair = [](float& u, float& w, float c, float s) {
        const float x = u, y = w;
        u = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
        w = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
    };
    if (inter) {
        pair(a[0], a[1], c[0], s[0]);
        pair(a[2], a[3], c[1], s[1]);
        pair(b[0], b[1], c[2], s[2]);
        pair(b[2], b[3], c[3], s[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) pair(a[i], b[i], c[i], s[i]);
    }
}

// A unit: the new tokens of one sequence in one page, by TG threads (a warp, or a block).  Units of a page: one for each
// head of the keys and of the values, then those of the queries, a share of Q_HEADS heads each (TG = 32) or of Q_ROWS rows
// with all heads (TG = 256: PART 0 is the keys' and values' launch, 1 the queries').
// Bytes bound the prompts, so loads in flight count: a block's 16-bit rows are staged in shared memory by asynchronous
// copies and read from there for the maximum and for the codes.  Read twice from memory 32768 tokens of 32 + 8 + 8 heads took 215
// us; kept in registers (110 to 157 of them) 313, or spilled 282.
// For single tokens one launch of a warp per head saves the barriers.
constexpr int Q_HEADS = 8, Q_ROWS = 8;

// Eight values as stored.
template <typename T>
struct Raw {
    alignas(16) T lo[4], hi[4];
    __device__ __forceinline__ void load(const T* __restrict__ a, const T* __restrict__ b, bool vec) {
        if (vec) {
            if constexpr (sizeof(T) == 4) {
                *reinterpret_cast<uint4*>(lo) = *reinterpret_cast<const uint4*>(a);
                *reinterpret_cast<uint4*>(hi) = *reinterpret_cast<const uint4*>(b);
            } else {
                *reinterpret_cast<uint2*>(lo) = *reinterpret_cast<const uint2*>(a);
                *reinterpret_cast<uint2*>(hi) = *reinterpret_cast<const uint2*>(b);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) lo[e] = a[e], hi[e] = b[e];
        }
    }
    __device__ __forceinline__ void get(float (&a)[4], float (&b)[4]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = to_f32(lo[e]), b[e] = to_f32(hi[e]);
    }
};

template <typename T, int TG, int PART>
__global__ void __launch_bounds__(TG == 32 ? 128 : TG) kv_append_kernel(const __grid_constant__ AppendArgs A) {
    constexpr bool STAGED = TG > 32 && PART == 0 && sizeof(T) == 2;
    __shared__ __align__(16) unsigned char stage[STAGED ? 128 * 128 * 2 : 16];  // the largest block's rows
    pdl_wait();
    constexpr int UNITS = TG == 32 ? 4 : 1;
    const int sub = TG == 32 ? threadIdx.x >> 5 : 0, t = TG == 32 ? threadIdx.x & 31 : threadIdx.x;
    const unsigned unit = blockIdx.x * UNITS + sub;  // page-major
    const int cand = (int)(unit / (unsigned)A.kinds);
    int kind = (int)(unit - (unsigned)cand * A.kinds);
    if (cand >= A.units) return;  // (whole unit)
    const Seqs& S = A.s;
    const int page = A.c.page, D = A.c.dim, oct = D / 8, oct_bits = D == 128 ? 4 : 3;
    const int b = S.starts ? find_seq(S, cand, 1, page, 2) : cand / A.per_seq;
    int first, count;
    new_rows(S, b, first, count);
    const int j = cand - (S.starts ? (int)unit_base(max(__ldg(S.starts + b), 0), b, 1, page, 2) : b * A.per_seq);
    const int len = __ldg(S.lens + b);
    int p0 = len - count;  // position of the first new token
    const bool queries = TG == 32 ? kind >= 2 * A.c.heads : PART == 1;
    if (TG == 32 && queries) kind -= 2 * A.c.heads;
    if (p0 < 0) {  // rows before the sequence's start are padding: not appended, their queries zeros
        const int pad = min(count, -p0);
        if (j == 0 && queries && kind == 0) {
            T* out = static_cast<T*>(A.q_out) + (long long)first * A.q_heads * D;
            const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (long long i = t; i < (long long)pad * A.q_heads * (D / 4); i += TG) store_f32<4>(out + 4 * i, z);
        }
        first += pad;
        count -= pad;
        p0 = 0;
    }
    if (count <= 0) return;
    const int pi = p0 / page + j;  // this unit's page of the sequence
    const int from = max(p0, pi * page), to = min(len, (pi + 1) * page);
    if (from >= to) return;
    const int row0 = first + (from - p0), n = to - from, slot0 = from - pi * page;
    if constexpr (TG == 32 || PART == 1) if (queries) {  // ---- rotated, rounded once
        const T* q = static_cast<const T*>(A.q);
        T* out = static_cast<T*>(A.q_out);
        const int r_lo = TG == 32 ? 0 : kind * Q_ROWS, h_lo = TG == 32 ? kind * Q_HEADS : 0;
        const int h_n = TG == 32 ? min(Q_HEADS, A.q_heads - h_lo) : A.q_heads, r_n = TG == 32 ? n : min(Q_ROWS, n - r_lo);
        const int o = t & (oct - 1);
        int lo, hi;
        octet_at(o, A.rot, A.inter, lo, hi);
        constexpr int TOGETHER = TG == 32 ? 1 : 4;  // octets of a thread whose loads are in flight at once
        const int step = TG >> oct_bits, all = r_n * h_n;  // lanes run over octets, then heads, then rows
        const float per_head = 1.0f / (float)h_n;          // i / h_n = floor((i + 1/2) per_head): i stays far below 2^22
        for (int i0 = t >> oct_bits; i0 < all; i0 += TOGETHER * step) {
            Raw<T> x[TOGETHER];
#pragma unroll
            for (int u = 0; u < TOGETHER; ++u) {
                const int i = min(i0 + u * step, all - 1), r = (int)(((float)i + 0.5f) * per_head), h = h_lo + i - r * h_n;
                const T* src = q + (long long)(row0 + r_lo + r) * A.q_token + (long long)h * A.q_head;
                x[u].load(src + lo, src + hi, A.vec);
            }
#pragma unroll
            for (int u = 0; u < TOGETHER; ++u) {
                const int i = i0 + u * step;
                if (i >= all) break;
                const int r = (int)(((float)i + 0.5f) * per_head), h = h_lo + i - r * h_n, pos = from + r_lo + r;
                float a[4], c[4];
                x[u].get(a, c);
                if (A.rot && pos >= A.n_pos) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[e] = c[e] = 0.0f;
                } else if (8 * o < A.rot) {
                    float cs[4], sn[4];
                    load_turn(A, pos, o, cs, sn);
                    turn(a, c, cs, sn, A.inter);
                }
                T* dst = out + ((long long)(row0 + r_lo + r) * A.q_heads + h) * D;
                store_f32<4>(dst + lo, a);
                store_f32<4>(dst + hi, c);
            }
        }
        return;
    }
    if constexpr (TG > 32 && PART == 1) return;
    const int pid = pi < S.max_pages ? __ldg(S.pages + (long long)b * S.pages_stride + pi) : -1;
    const bool is_v = kind >= A.c.heads;
    const int head = kind - (is_v ? A.c.heads : 0);
    if ((unsigned)pid >= (unsigned)A.c.n_pages) {
        if (t == 0) latch_status(A.status, FXPQ_ERR_RANGE);
        return;
    }
    const int rot = is_v ? 0 : A.rot;
    const T* x = static_cast<const T*>(is_v ? A.v : A.k) + (long long)row0 * (is_v ? A.v_token : A.k_token) + (long long)head * (is_v ? A.v_head : A.k_head);
    long long ts = is_v ? A.v_token : A.k_token;
    const long long block = (long long)pid * A.c.heads + head;
    int8_t* codes = (is_v ? A.c.d_v : A.c.d_k) + block * page * D;
    float* scale = (is_v ? A.c.d_v_scale : A.c.d_k_scale) + block;
    const int usable = A.rot ? max(0, min(n, A.n_pos - from)) : n;  // tokens past the tables are not appended
    if (usable < n && t == 0) latch_status(A.status, FXPQ_ERR_RANGE);
    if (usable == 0) return;
    const float before = slot0 > 0 ? *scale : 0.0f;
    const int o = t & (oct - 1), r_first = t >> oct_bits, r_step = TG >> oct_bits;  // this thread's octet and rows
    int lo, hi;
    octet_at(o, rot, A.inter, lo, hi);
    auto turned = [&](const Raw<T>& v, int r, float (&a)[4], float (&c)[4]) {
        v.get(a, c);
        if (8 * o < rot) {
            float cs[4], sn[4];
            load_turn(A, from + r, o, cs, sn);
            turn(a, c, cs, sn, A.inter);
        }
    };
    Raw<T> v;
    float a[4], c[4];
    bool vec = A.vec;
    if constexpr (STAGED) {
        T* rows = reinterpret_cast<T*>(stage);
        const int per = D / 8, bits = oct_bits;  // 16-byte pieces of a row
        if (A.vec16) {
            for (int i = t; i < usable * per; i += TG)
                tc::cp_async16(tc::smem_u32(rows + 8 * i), x + (i >> bits) * ts + 8 * (i & (per - 1)), 16);
            tc::cp_async_commit();
            tc::cp_async_wait<0>();
        } else {
            for (int i = t; i < usable * D; i += TG) rows[i] = x[(i >> (bits + 3)) * ts + (i & (D - 1))];
        }
        __syncthreads();
        x = rows;
        ts = D;
        vec = true;
    }
    // The largest magnitude, as bits: infinities and NaN are above every finite value, and only where one is found are
    // they sorted out.
    __shared__ uint32_t part[TG > 32 ? TG / 32 : 1];
    auto largest = [&](bool finite) {
        uint32_t top = 0;
#pragma unroll 2
        for (int r = r_first; r < usable; r += r_step) {
            v.load(x + r * ts + lo, x + r * ts + hi, vec);
            turned(v, r, a, c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t p = __float_as_uint(a[e]) & 0x7fffffffu, q = __float_as_uint(c[e]) & 0x7fffffffu;
                if (finite) p = p < 0x7f800000u ? p : 0u, q = q < 0x7f800000u ? q : 0u;
                top = max(top, max(p, q));
            }
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if constexpr (TG > 32) {
            __syncthreads();
            if ((t & 31) == 0) part[t >> 5] = top;
            __syncthreads();
            top = part[0];
#pragma unroll
            for (int w = 1; w < TG / 32; ++w) top = max(top, part[w]);
        }
        return top;
    };
    uint32_t top_bits = largest(false);
    const bool bad = top_bits >= 0x7f800000u;
    if (bad) {
        if (t == 0) latch_status(A.status, FXPQ_ERR_NONFINITE);
        top_bits = largest(true);
    }
    const float top = __uint_as_float(top_bits);
    const float after = fmaxf(before, block_scale(top));  // (every thread has read *scale)
    if (t == 0 && after != before) *scale = after;
    if (before > 0.0f && after != before) {  // the block's older codes, rounded again
        const float ratio = __fdiv_rn(before, after);
        for (int i = t; i < slot0 * D / 4; i += TG) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[i];
            int v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = code_of((float)(int8_t)(w >> (8 * e)) * ratio);
            reinterpret_cast<uint32_t*>(codes)[i] = pack_i8(v[0], v[1], v[2], v[3]);
        }
    }
    const Divider over(after);
    // Where the scale is a power of two and nothing is clipped, one fused multiply-add rounds: the product is exact, adding
    // 1.5 * 2^23 rounds it half to even and leaves the code in the low byte.
    const bool plain = over.exact && !bad && top <= 127.0f * after;
    const bool again = TG > 32 || usable > r_step;  // (a warp with one round of rows still has it)
#pragma unroll 2
    for (int r = r_first; r < usable; r += r_step) {
        if (again) v.load(x + r * ts + lo, x + r * ts + hi, vec);
        turned(v, r, a, c);
        uint32_t va[4], vc[4];
        if (plain) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                va[e] = __float_as_uint(fmaf(a[e], over.inv, 12582912.0f));
                vc[e] = __float_as_uint(fmaf(c[e], over.inv, 12582912.0f));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                va[e] = fabsf(a[e]) <= FLT_MAX ? code_of(over(a[e])) : 0;
                vc[e] = fabsf(c[e]) <= FLT_MAX ? code_of(over(c[e])) : 0;
            }
        }
        int8_t* dst = codes + (slot0 + r) * D;
        *reinterpret_cast<uint32_t*>(dst + lo) = pack_i8(va[0], va[1], va[2], va[3]);
        *reinterpret_cast<uint32_t*>(dst + hi) = pack_i8(vc[0], vc[1], vc[2], vc[3]);
    }
}

// 16 codes per thread and step.
template <typename T>
__global__ void __launch_bounds__(256) kv_values_kernel(const fxpq_kv_cache c, const int* list, T* k_out, T* v_out, int* status) {
    pdl_wait();
    const int pid = __ldg(list + blockIdx.x);
    const bool ok = (unsigned)pid < (unsigned)c.n_pages;
    if (!ok && threadIdx.x == 0) latch_status(status, FXPQ_ERR_RANGE);
    const int per_head = c.page * c.dim / 16, all = per_head * c.heads;
    T* out = blockIdx.z ? v_out : k_out;
    if (!out) return;
    const int8_t* src = (blockIdx.z ? c.d_v : c.d_k) + (long long)pid * all * 16;
    const float* scales = (blockIdx.z ? c.d_v_scale : c.d_k_scale) + (long long)pid * c.heads;
    for (int i = blockIdx.y * blockDim.x + threadIdx.x; i < all; i += gridDim.y * blockDim.x) {
        float v[16];
        uint4 w = make_uint4(0, 0, 0, 0);
        float s = 0.0f;
        if (ok) {
            w = *reinterpret_cast<const uint4*>(src + 16 * i);
            s = __ldg(scales + i / per_head);
        }
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = (float)(int8_t)(u[e / 4] >> (8 * (e % 4))) * s;
        store_f32<16>(out + ((long long)blockIdx.x * all + i) * 16, v);
    }
}

template <typename T>
bool vec_ok(const fxpq_kv_rows* r) {  // four elements in one access
    return !r || !r->d_x || (aligned(r->d_x, 4 * sizeof(T)) && r->token_stride % 4 == 0 && r->head_stride % 4 == 0);
}

template <typename T>
fxpq_status launch_append(AppendArgs& A, bool wide, cudaStream_t st) {
    if (!wide) {
        A.kinds = 2 * A.c.heads + (A.q_heads + Q_HEADS - 1) / Q_HEADS;
        launch_pdl(kv_append_kernel<T, 32, 0>, dim3((unsigned)(((long long)A.units * A.kinds + 3) / 4)), dim3(128), 0, st, A);
        return after_launch("kv_append");
    }
    A.kinds = 2 * A.c.heads;
    launch_pdl(kv_append_kernel<T, 256, 0>, dim3((unsigned)(A.units * A.kinds)), dim3(256), 0, st, A);
    const fxpq_status rc = after_launch("kv_append");
    if (rc != FXPQ_OK || A.q_heads == 0) return rc;
    A.kinds = A.c.page / Q_ROWS;
    launch_pdl(kv_append_kernel<T, 256, 1>, dim3((unsigned)(A.units * A.kinds)), dim3(256), 0, st, A);
    return after_launch("kv_append_queries");
}

}  // namespace
}  // namespace llm
}  // namespace fxpq

using namespace fxpq;
using namespace fxpq::llm;

extern "C" fxpq_status fxpq_kv_append(const fxpq_kv_cache* cache, const fxpq_kv_batch* batch, int32_t type, const fxpq_kv_rows* k,
                                      const fxpq_kv_rows* v, const fxpq_kv_rows* q, int32_t q_heads, void* d_q_out,
                                      const float* d_cos, const float* d_sin, int32_t n_positions, int32_t rot,
                                      int32_t interleaved, void* stream) {
    if (!cache_ok(cache) || !batch_ok(batch) || !ftype_ok(type) || !k || !v || interleaved < 0 || interleaved > 1)
        return FXPQ_ERR_INVALID_ARG;
    const bool has_q = q && q->d_x;
    if (has_q && q_heads > 1 << 16) return FXPQ_ERR_UNSUPPORTED;
    if (rot < 0 || rot > cache->dim || rot % 8 || (rot && (!d_cos || !d_sin || n_positions < 0 || !aligned(d_cos, 16) || !aligned(d_sin, 16))) ||
        (has_q && (q_heads <= 0 || !d_q_out || !aligned(d_q_out, 16))))
        return FXPQ_ERR_INVALID_ARG;
    const size_t e = ftype_bytes(type);
    if (batch->n_tokens > 0 && (!k->d_x || !v->d_x || !aligned(k->d_x, e) || !aligned(v->d_x, e) || (has_q && !aligned(q->d_x, e))))
        return FXPQ_ERR_INVALID_ARG;
    if (batch->n_tokens == 0) return FXPQ_OK;
    AppendArgs A;
    A.s = make_seqs(*batch);
    A.c = *cache;
    A.k = k->d_x, A.k_token = k->token_stride, A.k_head = k->head_stride;
    A.v = v->d_x, A.v_token = v->token_stride, A.v_head = v->head_stride;
    A.q = has_q ? q->d_x : nullptr, A.q_token = has_q ? q->token_stride : 0, A.q_head = has_q ? q->head_stride : 0;
    A.q_out = d_q_out;
    A.q_heads = has_q ? q_heads : 0;
    A.cos_t = d_cos, A.sin_t = d_sin;
    A.n_pos = rot ? n_positions : 0;
    A.rot = rot;
    A.inter = interleaved;
    A.status = status_ptr();
    // n tokens lie in at most floor((n + page - 2) / page) + 1 pages, which floor(n / page) + 2 covers
    A.per_seq = batch->d_starts ? 0 : (A.s.each + cache->page - 2) / cache->page + 1;
    const long long cands = batch->d_starts ? unit_base(batch->n_tokens, batch->n_seqs, 1, cache->page, 2) : (long long)A.per_seq * batch->n_seqs;
    const bool wide = batch->n_tokens >= 8LL * batch->n_seqs;
    if (cands * (2LL * cache->heads + A.q_heads + cache->page) > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    A.units = (int)cands;
    const fxpq_kv_rows* rq = has_q ? q : nullptr;
    A.vec16 = type != FXPQ_FT_F32;
    for (const fxpq_kv_rows* r : {k, v}) A.vec16 &= aligned(r->d_x, 16) && r->token_stride % 8 == 0 && r->head_stride % 8 == 0;
    if (type == FXPQ_FT_F32) {
        A.vec = vec_ok<float>(k) && vec_ok<float>(v) && vec_ok<float>(rq);
        return launch_append<float>(A, wide, as_stream(stream));
    } else if (type == FXPQ_FT_F16) {
        A.vec = vec_ok<__half>(k) && vec_ok<__half>(v) && vec_ok<__half>(rq);
        return launch_append<__half>(A, wide, as_stream(stream));
    } else {
        A.vec = vec_ok<__nv_bfloat16>(k) && vec_ok<__nv_bfloat16>(v) && vec_ok<__nv_bfloat16>(rq);
        return launch_append<__nv_bfloat16>(A, wide, as_stream(stream));
    }
}

extern "C" fxpq_status fxpq_kv_values(const fxpq_kv_cache* cache, const int32_t* d_list, int32_t n, int32_t type, void* d_k_out,
                                      void* d_v_out, void* stream) {
    if (!cache_ok(cache) || n < 0 || !ftype_ok(type) || (n > 0 && !d_list) || !aligned(d_list, 4) || !aligned(d_k_out, 16) || !aligned(d_v_out, 16))
        return FXPQ_ERR_INVALID_ARG;
    if (n == 0 || (!d_k_out && !d_v_out)) return FXPQ_OK;
    const int all = cache->page * cache->dim / 16 * cache->heads;
    const dim3 grid((unsigned)n, (unsigned)((all + 1023) / 1024), 2);
    cudaStream_t st = as_stream(stream);
    int* status = status_ptr();
    if (type == FXPQ_FT_F32)
        launch_pdl(kv_values_kernel<float>, grid, dim3(256), 0, st, *cache, d_list, static_cast<float*>(d_k_out), static_cast<float*>(d_v_out), status);
    else if (type == FXPQ_FT_F16)
        launch_pdl(kv_values_kernel<__half>, grid, dim3(256), 0, st, *cache, d_list, static_cast<__half*>(d_k_out), static_cast<__half*>(d_v_out), status);
    else
        launch_pdl(kv_values_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, *cache, d_list, static_cast<__nv_bfloat16*>(d_k_out),
                   static_cast<__nv_bfloat16*>(d_v_out), status);
    return after_launch("kv_values");
}
