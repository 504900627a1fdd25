// fxpq_kv.cu -- the paged cache of 8-bit keys and values: appending with the position rotation, reading back.
#include <cfloat>

#include "fxpq_llm.cuh"

namespace fxpq {
namespace llm {

bool batch_ok(const fxpq_kv_batch* b) {
    return b && b->n_seqs >= 0 && b->n_tokens >= 0 && b->max_pages >= 0 && b->pages_stride >= b->max_pages &&
           (b->n_seqs == 0 ? b->n_tokens == 0 : (b->d_pages || b->max_pages == 0) && b->d_lens != nullptr) &&
           (b->d_starts || b->n_seqs == 0 || b->n_tokens % b->n_seqs == 0);
}
bool cache_ok(const fxpq_kv_cache* c) {
    return c && c->n_pages > 0 && c->heads > 0 && c->d_k && c->d_v && c->d_k_scale && c->d_v_scale && aligned(c->d_k, 16) &&
           aligned(c->d_v, 16) && (c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128) &&
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
    int q_heads, n_pos, rot, inter, vec;
    int per_seq, units;  // work units: pages that a sequence's new tokens may touch (uniform batches), in all
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

template <typename T>
__device__ __forceinline__ void load_octet(const T* row, int j, int rot, int inter, bool vec, const float* cos_p,
                                           const float* sin_p, float (&a)[4], float (&b)[4]) {
    int lo, hi;
    octet_at(j, rot, inter, lo, hi);
    load_f32<4>(row + lo, vec, a);
    load_f32<4>(row + hi, vec, b);
    if (8 * j < rot) {
        const float4 c4 = *reinterpret_cast<const float4*>(cos_p + 4 * j), s4 = *reinterpret_cast<const float4*>(sin_p + 4 * j);
        const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // pairs (a[i], b[i]), or interleaved (x[2 i], x[2 i + 1]) of a, b = x[0 .. 3], x[4 .. 7]
            float& u = !inter ? a[i] : i < 2 ? a[2 * i] : b[2 * i - 4];
            float& w = !inter ? b[i] : i < 2 ? a[2 * i + 1] : b[2 * i - 3];
            const float x = u, y = w;
            u = __fsub_rn(__fmul_rn(x, c[i]), __fmul_rn(y, s[i]));
            w = __fadd_rn(__fmul_rn(y, c[i]), __fmul_rn(x, s[i]));
        }
    }
}

// A unit: the new tokens of one sequence in one page, for one head of the keys, values or queries, by TG
// threads (a warp, or the whole block).  One pass over the rows for the largest value, one (from L1) for the codes.
template <typename T, int TG>
__global__ void __launch_bounds__(TG == 32 ? 128 : TG) kv_append_kernel(const __grid_constant__ AppendArgs A) {
    pdl_wait();
    constexpr int UNITS = TG == 32 ? 4 : 1;
    const int sub = TG == 32 ? threadIdx.x >> 5 : 0, t = TG == 32 ? threadIdx.x & 31 : threadIdx.x;
    const int all_heads = 2 * A.c.heads + A.q_heads;
    const long long unit = (long long)blockIdx.x * UNITS + sub;  // page-major, heads innermost
    const int cand = (int)(unit / all_heads);
    int head = (int)(unit - (long long)cand * all_heads);
    if (cand >= A.units) return;  // (whole unit)
    const Seqs& S = A.s;
    const int page = A.c.page, D = A.c.dim, oct = D / 8;
    const int b = S.starts ? find_seq(S, cand, 1, page, 2) : cand / A.per_seq;
    int first, count;
    new_rows(S, b, first, count);
    const int j = cand - (S.starts ? (int)unit_base(max(__ldg(S.starts + b), 0), b, 1, page, 2) : b * A.per_seq);
    const int len = __ldg(S.lens + b);
    int p0 = len - count;  // position of the first new token
    if (p0 < 0) {          // rows before the sequence's start are padding: not appended, their queries zeros
        const int pad = min(count, -p0);
        if (j == 0 && head >= 2 * A.c.heads) {
            T* out = static_cast<T*>(A.q_out) + ((long long)first * A.q_heads + head - 2 * A.c.heads) * D;
            const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int i = t; i < pad * D / 4; i += TG)
                store_f32<4>(out + (long long)(i / (D / 4)) * A.q_heads * D + 4 * (i % (D / 4)), z);
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
    int pid = pi < A.s.max_pages ? __ldg(S.pages + (long long)b * S.pages_stride + pi) : -1;
    if (head >= 2 * A.c.heads) {  // ---- queries: rotate, round once
        head -= 2 * A.c.heads;
        const T* q = static_cast<const T*>(A.q);
        T* out = static_cast<T*>(A.q_out);
        for (int i = t; i < n * oct; i += TG) {
            const int r = i / oct, o = i - r * oct, pos = from + r;
            float a[4], c[4];
            int lo, hi;
            octet_at(o, A.rot, A.inter, lo, hi);
            const bool ok = A.rot == 0 || pos < A.n_pos;
            if (ok) {
                const long long cs = (long long)pos * (A.rot / 2);
                load_octet(q + (long long)(row0 + r) * A.q_token + (long long)head * A.q_head, o, A.rot, A.inter, A.vec,
                           A.cos_t + cs, A.sin_t + cs, a, c);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) a[e] = c[e] = 0.0f;
            }
            T* dst = out + ((long long)(row0 + r) * A.q_heads + head) * D;
            store_f32<4>(dst + lo, a);
            store_f32<4>(dst + hi, c);
        }
        return;
    }
    const bool is_v = head >= A.c.heads;
    if (is_v) head -= A.c.heads;
    if ((unsigned)pid >= (unsigned)A.c.n_pages) {
        if (t == 0) latch_status(A.status, FXPQ_ERR_RANGE);
        return;
    }
    const int rot = is_v ? 0 : A.rot;
    const T* x = static_cast<const T*>(is_v ? A.v : A.k);
    const long long ts = is_v ? A.v_token : A.k_token, hs = is_v ? A.v_head : A.k_head;
    const long long block = (long long)pid * A.c.heads + head;
    int8_t* codes = (is_v ? A.c.d_v : A.c.d_k) + block * page * D;
    float* scale = (is_v ? A.c.d_v_scale : A.c.d_k_scale) + block;
    const int usable = A.rot ? max(0, min(n, A.n_pos - from)) : n;  // tokens past the tables are not appended
    if (usable < n && t == 0) latch_status(A.status, FXPQ_ERR_RANGE);
    if (usable == 0) return;
    const float before = slot0 > 0 ? *scale : 0.0f;
    float top = 0.0f;
    bool bad = false;
    for (int i = t; i < usable * oct; i += TG) {
        const int r = i / oct, o = i - r * oct;
        float a[4], c[4];
        const long long cs = (long long)(from + r) * (rot / 2);
        load_octet(x + (long long)(row0 + r) * ts + (long long)head * hs, o, rot, A.inter, A.vec, A.cos_t + cs, A.sin_t + cs, a, c);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = fabsf(a[e]), w = fabsf(c[e]);
            bad |= !(u <= FLT_MAX) || !(w <= FLT_MAX);
            top = fmaxf(top, fmaxf(u <= FLT_MAX ? u : 0.0f, w <= FLT_MAX ? w : 0.0f));
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if constexpr (TG > 32) {
        __shared__ float part[TG / 32];
        if ((t & 31) == 0) part[t >> 5] = top;
        __syncthreads();
        top = part[0];
#pragma unroll
        for (int w = 1; w < TG / 32; ++w) top = fmaxf(top, part[w]);
    }
    if (bad) latch_status(A.status, FXPQ_ERR_NONFINITE);
    const float after = fmaxf(before, block_scale(top));  // (every thread has read *scale)
    if (t == 0 && after != before) *scale = after;
    if (before > 0.0f && after != before) {  // the block's older codes, rounded again
        const float ratio = __fdiv_rn(before, after);
        for (int i = t; i < slot0 * D / 4; i += TG) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[i];
            int o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = code_of((float)(int8_t)(w >> (8 * e)) * ratio);
            reinterpret_cast<uint32_t*>(codes)[i] = pack_i8(o[0], o[1], o[2], o[3]);
        }
    }
    const Divider over(after);
    for (int i = t; i < usable * oct; i += TG) {
        const int r = i / oct, o = i - r * oct;
        float a[4], c[4];
        int lo, hi, ca[4], cc[4];
        octet_at(o, rot, A.inter, lo, hi);
        const long long cs = (long long)(from + r) * (rot / 2);
        load_octet(x + (long long)(row0 + r) * ts + (long long)head * hs, o, rot, A.inter, A.vec, A.cos_t + cs, A.sin_t + cs, a, c);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ca[e] = fabsf(a[e]) <= FLT_MAX ? code_of(over(a[e])) : 0;
            cc[e] = fabsf(c[e]) <= FLT_MAX ? code_of(over(c[e])) : 0;
        }
        int8_t* dst = codes + (long long)(slot0 + r) * D;
        *reinterpret_cast<uint32_t*>(dst + lo) = pack_i8(ca[0], ca[1], ca[2], ca[3]);
        *reinterpret_cast<uint32_t*>(dst + hi) = pack_i8(cc[0], cc[1], cc[2], cc[3]);
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
void launch_append(const AppendArgs& A, bool wide, cudaStream_t st) {
    const long long units = (long long)A.units * (2 * A.c.heads + A.q_heads);
    if (wide)
        launch_pdl(kv_append_kernel<T, 256>, dim3((unsigned)units), dim3(256), 0, st, A);
    else
        launch_pdl(kv_append_kernel<T, 32>, dim3((unsigned)((units + 3) / 4)), dim3(128), 0, st, A);
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
    if (cands * (2 * cache->heads + A.q_heads) > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    A.units = (int)cands;
    const bool wide = batch->n_tokens >= 8LL * batch->n_seqs;
    const fxpq_kv_rows* rq = has_q ? q : nullptr;
    if (type == FXPQ_FT_F32) {
        A.vec = vec_ok<float>(k) && vec_ok<float>(v) && vec_ok<float>(rq);
        launch_append<float>(A, wide, as_stream(stream));
    } else if (type == FXPQ_FT_F16) {
        A.vec = vec_ok<__half>(k) && vec_ok<__half>(v) && vec_ok<__half>(rq);
        launch_append<__half>(A, wide, as_stream(stream));
    } else {
        A.vec = vec_ok<__nv_bfloat16>(k) && vec_ok<__nv_bfloat16>(v) && vec_ok<__nv_bfloat16>(rq);
        launch_append<__nv_bfloat16>(A, wide, as_stream(stream));
    }
    return after_launch("kv_append");
}

extern "C" fxpq_status fxpq_kv_values(const fxpq_kv_cache* cache, const int32_t* d_list, int32_t n, int32_t type, void* d_k_out,
                                      void* d_v_out, void* stream) {
    if (!cache_ok(cache) || n < 0 || !ftype_ok(type) || (n > 0 && !d_list) || !aligned(d_k_out, 16) || !aligned(d_v_out, 16))
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
