// fxpq_attend.cu -- softmax attention over the paged cache of 8-bit keys and values: checks, choice of kernel.
#include "fxpq_attend.cuh"

using namespace fxpq;
using namespace fxpq::llm;

namespace {

// Codes as [n_pages * heads][page][dim] bytes, boxes of one page's `rows` rows, swizzled by their row size.
bool encode_codes(CUtensorMap* map, const fxpq_kv_cache& c, const int8_t* codes, int rows) {
    EncodeTiledFn enc = encode_tiled();
    const cuuint64_t dims[3] = {(cuuint64_t)c.dim, (cuuint64_t)c.page, (cuuint64_t)c.n_pages * c.heads};
    const cuuint64_t strides[2] = {(cuuint64_t)c.dim, (cuuint64_t)c.dim * c.page};
    const cuuint32_t box[3] = {(cuuint32_t)c.dim, (cuuint32_t)(rows < c.page ? rows : c.page), 1}, es[3] = {1, 1, 1};
    return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<int8_t*>(codes), dims, strides, box, es,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, c.dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a batch is computed.  New tokens per sequence are known on the host only on average.
struct Plan {
    int nt;      // 8 nt query rows share a read of the cache
    bool whole;  // one CTA per unit
    size_t ws;
};
Plan plan(const fxpq_kv_cache& c, const fxpq_kv_batch& b, int q_heads) {
    Plan p;
    const long long group = q_heads / c.heads, seqs = b.n_seqs > 0 ? b.n_seqs : 1;
    p.nt = stream_nt((b.n_tokens * group + seqs - 1) / seqs);
    // A cache of at most 2048 tokens is one CTA's work; longer ones are cut into equal shares for all CTAs.
    p.whole = (long long)b.max_pages * c.page <= 2048;
    p.ws = p.whole ? 0 : (attend_stream_workspace(c.dim, p.nt) + 255) / 256 * 256;
    return p;
}

}  // namespace

extern "C" size_t fxpq_kv_attention_workspace(const fxpq_kv_cache* cache, const fxpq_kv_batch* batch, int32_t q_heads) {
    if (!cache_ok(cache) || !batch_ok(batch) || q_heads <= 0 || q_heads % cache->heads) return 0;
    return plan(*cache, *batch, q_heads).ws;
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
    if ((long long)cache->n_pages * cache->heads > INT32_MAX || (long long)batch->n_tokens * q_heads > INT32_MAX) return FXPQ_ERR_UNSUPPORTED;
    const Plan p = plan(*cache, *batch, q_heads);
    if (p.ws && (!d_ws || ws_bytes < p.ws || !aligned(d_ws, 256))) return FXPQ_ERR_WORKSPACE;
    AttendArgs A;
    if (!encode_codes(&A.tk, *cache, cache->d_k, 32) || !encode_codes(&A.tv, *cache, cache->d_v, 32)) return FXPQ_ERR_CUDA;
    A.s = make_seqs(*batch);
    A.k_scale = cache->d_k_scale, A.v_scale = cache->d_v_scale;
    A.q = q->d_x, A.q_token = q->token_stride, A.q_head = q->head_stride;
    A.out = d_out, A.lse = d_lse, A.part = static_cast<float*>(d_ws);
    A.n_pages = cache->n_pages, A.page = cache->page, A.heads = cache->heads, A.q_heads = q_heads, A.group = q_heads / cache->heads;
    A.q_f16 = type == FXPQ_FT_F16;
    A.q_vec = aligned(q->d_x, 16) && q->token_stride % 8 == 0 && q->head_stride % 8 == 0;
    A.causal = causal;
    A.few = INT32_MAX;
    A.few_only = 0;
    A.scale = softmax_scale;
    A.status = status_ptr();
    return launch_attend_stream(A, cache->dim, p.nt, p.whole, as_stream(stream));
}
