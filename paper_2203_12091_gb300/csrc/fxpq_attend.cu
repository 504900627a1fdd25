// fxpq_attend.cu -- softmax attention over the paged cache of 8-bit keys and values.
#include <cfloat>

#include "fxpq_llm.cuh"

namespace fxpq {
namespace llm {
namespace {

struct AttendArgs {
    Seqs s;
    fxpq_kv_cache c;
    const void* q;
    long long q_token, q_head;
    void* out;
    float* lse;
    int q_heads, causal;
    float scale;
    int* status;
};

// One warp per new token and query head, one key at a time: the running maximum and sum of the softmax.
template <typename T>
__global__ void __launch_bounds__(128) attend_kernel(const AttendArgs A) {
    pdl_wait();
    const long long u = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, D = A.c.dim, E = D / 32;
    if (u >= (long long)A.s.n_tokens * A.q_heads) return;
    const int t = (int)(u / A.q_heads), h = (int)(u - (long long)t * A.q_heads), hk = h / (A.q_heads / A.c.heads);
    int b = A.s.starts ? 0 : t / A.s.each, first = 0, count = 0;
    if (A.s.starts)
        while (b < A.s.n_seqs - 1 && A.s.starts[b + 1] <= t) ++b;
    new_rows(A.s, b, first, count);
    const int len = A.s.lens[b], pos = len - count + (t - first);
    const int end = pos < 0 ? 0 : A.causal ? min(pos + 1, len) : len;
    float q[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0.0f;
    for (int e = 0; e < E; ++e) q[e] = to_f32(static_cast<const T*>(A.q)[t * A.q_token + h * A.q_head + E * lane + e]);
    for (int p = 0; p < end; ++p) {
        const int pi = p / A.c.page, pid = pi < A.s.max_pages ? A.s.pages[b * A.s.pages_stride + pi] : -1;
        if ((unsigned)pid >= (unsigned)A.c.n_pages) {
            if (lane == 0) latch_status(A.status, FXPQ_ERR_RANGE);
            continue;
        }
        const long long block = (long long)pid * A.c.heads + hk, at = (block * A.c.page + p % A.c.page) * D + E * lane;
        float s = 0.0f;
        for (int e = 0; e < E; ++e) s += q[e] * (float)A.c.d_k[at + e];
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= A.c.d_k_scale[block] * A.scale;
        const float top = fmaxf(m, s), f = expf(m - top), w = expf(s - top);
        l = l * f + w;
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * (float)A.c.d_v[at + e] * A.c.d_v_scale[block];
        m = top;
    }
    for (int e = 0; e < E; ++e)
        static_cast<T*>(A.out)[((long long)t * A.q_heads + h) * D + E * lane + e] = from_f32<T>(m > -INFINITY || !(l == 0.0f) ? o[e] / l : 0.0f);
    if (A.lse && lane == 0) A.lse[(long long)t * A.q_heads + h] = !(l == 0.0f) ? m + logf(l) : -INFINITY;
}

}  // namespace
}  // namespace llm
}  // namespace fxpq

using namespace fxpq;
using namespace fxpq::llm;

extern "C" size_t fxpq_kv_attention_workspace(const fxpq_kv_cache* cache, const fxpq_kv_batch* batch, int32_t q_heads) {
    (void)cache, (void)batch, (void)q_heads;
    return 0;
}

extern "C" fxpq_status fxpq_kv_attention(const fxpq_kv_cache* cache, const fxpq_kv_batch* batch, int32_t type, const fxpq_kv_rows* q,
                                         int32_t q_heads, float softmax_scale, int32_t causal, void* d_out, float* d_lse,
                                         void* d_ws, size_t ws_bytes, void* stream) {
    if (!cache_ok(cache) || !batch_ok(batch) || !ftype_ok(type) || q_heads <= 0 || q_heads % cache->heads || !q || causal < 0 ||
        causal > 1 || !(softmax_scale > 0.0f) || !(softmax_scale <= FLT_MAX))
        return FXPQ_ERR_INVALID_ARG;
    if (type == FXPQ_FT_F32) return FXPQ_ERR_UNSUPPORTED;
    if (batch->n_tokens == 0) return FXPQ_OK;
    if (!q->d_x || !aligned(q->d_x, 2) || !d_out || !aligned(d_out, 16) || !aligned(d_lse, 4)) return FXPQ_ERR_INVALID_ARG;
    const size_t need = fxpq_kv_attention_workspace(cache, batch, q_heads);
    if (need && (!d_ws || ws_bytes < need || !aligned(d_ws, 256))) return FXPQ_ERR_WORKSPACE;
    const AttendArgs A = {make_seqs(*batch), *cache, q->d_x, (long long)q->token_stride, (long long)q->head_stride, d_out, d_lse,
                          q_heads, causal, softmax_scale, status_ptr()};
    const long long units = (long long)batch->n_tokens * q_heads;
    if ((units + 3) / 4 > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((units + 3) / 4));
    if (type == FXPQ_FT_F16)
        launch_pdl(attend_kernel<__half>, grid, dim3(128), 0, as_stream(stream), A);
    else
        launch_pdl(attend_kernel<__nv_bfloat16>, grid, dim3(128), 0, as_stream(stream), A);
    return after_launch("kv_attention");
}
