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

// How a batch is computed.  Sequences of at most FEW rows (new tokens x grouped heads) per key head are the stream
// kernel's, the others the tile kernel's; where the counts are only on the device (ragged batches) both are launched
// unless there is but one kind, and each leaves the other's sequences alone.
constexpr int FEW = 32;
constexpr long long EXPAND_ROWS = 2048;
constexpr size_t EXPAND_ROOM = (size_t)1 << 30;

struct Plan {
    bool stream, tile;
    int nt;      // 8 nt query rows share a read of the cache
    bool whole;  // one CTA per unit
    int shares;  // CTAs that share the keys of a block of rows
    bool expand; // the codes are expanded to fp16 once, before the tile kernel
    size_t ws_stream, ws_join, ws;
};
Plan plan(const fxpq_kv_cache& c, const fxpq_kv_batch& b, int q_heads) {
    Plan p;
    const long long group = q_heads / c.heads, seqs = b.n_seqs > 0 ? b.n_seqs : 1;
    const long long mean = (b.n_tokens * group + seqs - 1) / seqs;  // rows of a sequence, the same for all without d_starts
    p.stream = b.d_starts || mean <= FEW;
    // (a ragged batch has a sequence of more than FEW rows only if it has that many rows)
    p.tile = b.d_starts ? b.n_tokens * group > FEW : mean > FEW;
    p.nt = stream_nt(mean);
    // A cache of at most 2048 tokens is one CTA's work; longer ones are cut into equal shares for all CTAs.
    const long long tokens = (long long)b.max_pages * c.page;
    p.whole = tokens <= 2048;
    p.ws_stream = p.stream && !p.whole ? (attend_stream_workspace(c.dim, p.nt) + 255) / 256 * 256 : 0;
    p.shares = 1;
    if (p.tile) {  // as many as fill the SMs, with at least 512 keys each
        const long long units = tile_blocks(b.n_tokens, b.n_seqs, (int)group, false) * c.heads + (b.d_starts ? c.heads : 0);
        while (p.shares < 16 && units * (p.shares + 1) <= num_sms() && tokens >= 512LL * (p.shares + 1)) ++p.shares;
    }
    p.ws_join = p.tile ? (attend_tile_workspace(b.n_tokens, q_heads, c.dim, p.shares) + 255) / 256 * 256 : 0;
    // Expanding costs five bytes of traffic a code and saves every block of 256 rows its own; the room is for max_pages.
    // Both ways measured (us, expanded and not; 65536 rows in all, 8 key heads of 128, groups of 4, causal, 4096 tokens and
    // the new ones): with 1024 rows a key head 1057 and 908, 2048 941 and 925, 4096 903 and 963, 8192 945 and 1051; heads
    // of 64 881 and 804, 839 and 822, 844 and 857, 905 and 940.  Without tokens before, 2048 rows 235 and 231, 4096 267 and 271;
    // behind 12288 2378 and 2332, 2216 and 2365.
    const size_t room = p.tile ? attend_expand_workspace(b.n_seqs, c.heads, c.dim, tokens) : 0;
    p.expand = p.tile && mean > EXPAND_ROWS && tokens > 0 && room <= EXPAND_ROOM && b.n_seqs <= 65535 && c.heads <= 65535 && tokens <= INT32_MAX - 128;
    p.ws = p.ws_stream + p.ws_join + (p.expand ? room : 0);
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
    A.s = make_seqs(*batch);
    A.k_scale = cache->d_k_scale, A.v_scale = cache->d_v_scale;
    A.q = q->d_x, A.q_token = q->token_stride, A.q_head = q->head_stride;
    A.out = d_out, A.lse = d_lse;
    A.n_pages = cache->n_pages, A.page = cache->page, A.heads = cache->heads, A.q_heads = q_heads, A.group = q_heads / cache->heads;
    A.q_f16 = type == FXPQ_FT_F16;
    A.q_vec = aligned(q->d_x, 16) && q->token_stride % 8 == 0 && q->head_stride % 8 == 0;
    A.causal = causal;
    A.few = p.tile ? FEW : INT32_MAX;
    A.few_only = p.stream && p.tile;
    A.scale = softmax_scale;
    A.status = status_ptr();
    cudaStream_t st = as_stream(stream);
    if (p.tile) {  // (first: its CTAs run longest)
        char* ws = static_cast<char*>(d_ws);
        A.part = reinterpret_cast<float*>(ws + p.ws_stream);
        fxpq_status rc;
        if (p.expand) {
            rc = launch_attend_tile_expanded(A, cache->d_k, cache->d_v, cache->dim, ws + p.ws_stream + p.ws_join, p.shares, st);
        } else {
            if (!encode_codes(&A.tk, *cache, cache->d_k, 128) || !encode_codes(&A.tv, *cache, cache->d_v, 128)) return FXPQ_ERR_CUDA;
            rc = launch_attend_tile(A, cache->dim, p.shares, st);
        }
        if (rc != FXPQ_OK || !p.stream) return rc;
    }
    if (!encode_codes(&A.tk, *cache, cache->d_k, 32) || !encode_codes(&A.tv, *cache, cache->d_v, 32)) return FXPQ_ERR_CUDA;
    A.part = static_cast<float*>(d_ws);
    return launch_attend_stream(A, cache->dim, p.nt, p.whole, st);
}
