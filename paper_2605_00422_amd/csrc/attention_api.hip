// C ABI of the cache, the rotary positions, the attention and the eviction: validation on the host, then launches.
// Nothing here allocates device memory, synchronizes or throws.
#include "attention_host.h"

namespace {

// bytes of scratch of an attention call
size_t forward_bytes(const AttArgs& a, bool weights, int dtype) {
    if (a.seqs == 0 || a.max_new == 0) return 0;
    if (bwla_att_is_split(a)) {
        const AttSplit p = bwla_att_split(a, weights);
        return p.part_bytes + p.stat_bytes + p.score_bytes;
    }
    // (the sums of weights, if wanted, use the same memory afterwards)
    const AttSplit p = bwla_att_tile_split(a);
    return std::max(p.part_bytes + p.stat_bytes, weights && a.max_len > 0 ? bwla_att_weights_plan(a, dtype).bytes : 0);
}

// an integer and a place in the list for each token
inline size_t evict_bytes(const bwla_kv_batch_t* b) { return (size_t)b->sequences * ((b->max_len + 3) & ~3) * 8; }

}  // namespace

extern "C" {

bwla_status_t bwla_rope_append(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, const bwla_rope_t* rope,
                               const int32_t* d_position, const void* d_qkv, int x_dtype, int64_t row_stride, int32_t q_heads, void* d_q, float* d_weights,
                               int32_t* d_cache_position, int32_t position_stride, void* stream) {
    RopeArgs a;
    bool idle;
    const bwla_status_t st = rope_args(cache, batch, rope, d_position, d_qkv, x_dtype, row_stride, q_heads, d_q, d_weights, d_cache_position,
                                       position_stride, &a, &idle);
    if (st != BWLA_OK || idle) return st;
    return done(bwla_launch_rope(a, x_dtype, cache->dtype, (hipStream_t)stream));
}

bwla_status_t bwla_attention_workspace_size(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, int32_t q_heads, int weights,
                                            size_t* bytes) {
    if (!bytes) return BWLA_ERR_NULL;
    const bwla_status_t st = check_shapes(cache, batch, q_heads);
    if (st != BWLA_OK) return st;
    *bytes = forward_bytes(shape_args(cache, batch, q_heads), weights != 0, cache->dtype);
    return BWLA_OK;
}

bwla_status_t bwla_attention_forward(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, const bwla_score_t* score,
                                     const void* d_q, int64_t q_stride, int32_t q_heads, void* d_out, float* d_lse, float* d_weights,
                                     void* d_ws, size_t ws_bytes, void* stream) {
    AttArgs a;
    const bwla_status_t st = attention_args(cache, batch, score, d_q, q_stride, q_heads, &a);
    if (st != BWLA_OK) return st;
    if (batch->tokens == 0 || batch->sequences == 0 || a.max_new == 0) return BWLA_OK;
    if (!d_out || (d_weights && !d_lse)) return BWLA_ERR_NULL;
    if (off16(d_out) || off16(d_lse) || off16(d_weights) || off16(d_ws)) return BWLA_ERR_ALIGN;
    const size_t need = forward_bytes(a, d_weights != nullptr, cache->dtype);
    if (need > 0 && !d_ws) return BWLA_ERR_NULL;
    if (ws_bytes < need) return BWLA_ERR_BUFSIZE;
    a.out = (char*)d_out;
    a.lse = d_lse;
    a.weights = d_weights;
    const hipStream_t s = (hipStream_t)stream;
    if (bwla_att_is_split(a)) return done(bwla_launch_attention_split(a, bwla_att_split(a, d_weights != nullptr), cache->dtype, d_ws, s));
    const hipError_t e = bwla_launch_attention_tile(a, bwla_att_tile_split(a), cache->dtype, d_ws, s);
    if (e != hipSuccess || !d_weights || a.max_len == 0) return done(e);
    return done(bwla_launch_attention_weights(a, cache->dtype, d_ws, s));
}

bwla_status_t bwla_attention_weights_workspace_size(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, int32_t q_heads,
                                                    size_t* bytes) {
    if (!bytes) return BWLA_ERR_NULL;
    const bwla_status_t st = check_shapes(cache, batch, q_heads);
    if (st != BWLA_OK) return st;
    const AttArgs a = shape_args(cache, batch, q_heads);
    *bytes = a.seqs == 0 || a.max_len == 0 ? 0 : bwla_att_weights_plan(a, cache->dtype).bytes;
    return BWLA_OK;
}

bwla_status_t bwla_attention_weights(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, const bwla_score_t* score,
                                     const void* d_q, int64_t q_stride, int32_t q_heads, const float* d_lse, float* d_weights, void* d_ws,
                                     size_t ws_bytes, void* stream) {
    AttArgs a;
    const bwla_status_t st = attention_args(cache, batch, score, d_q, q_stride, q_heads, &a);
    if (st != BWLA_OK) return st;
    if (batch->tokens == 0 || batch->sequences == 0 || a.max_new == 0 || a.max_len == 0) return BWLA_OK;
    if (!d_lse || !d_weights) return BWLA_ERR_NULL;
    if (off16(d_weights) || off16(d_ws)) return BWLA_ERR_ALIGN;
    const size_t need = bwla_att_weights_plan(a, cache->dtype).bytes;
    if (need > 0 && !d_ws) return BWLA_ERR_NULL;
    if (ws_bytes < need) return BWLA_ERR_BUFSIZE;
    a.lse = (float*)d_lse;                             // (only read here)
    a.weights = d_weights;
    return done(bwla_launch_attention_weights(a, cache->dtype, d_ws, (hipStream_t)stream));
}

bwla_status_t bwla_cache_evict_workspace_size(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, size_t* bytes) {
    if (!bytes) return BWLA_ERR_NULL;
    const bwla_status_t st = check_shapes(cache, batch, cache ? cache->kv_heads : 1);
    if (st != BWLA_OK) return st;
    *bytes = evict_bytes(batch);
    return BWLA_OK;
}

bwla_status_t bwla_cache_evict(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, const int32_t* d_table_out,
                               int32_t table_out_stride, float* d_weights, int32_t keep, int32_t sinks, int32_t recent, int32_t* d_len_out,
                               int32_t* d_kept, const int32_t* d_position, int32_t position_stride, int32_t* d_position_out, void* d_ws,
                               size_t ws_bytes, void* stream) {
    bwla_status_t st = check_shapes(cache, batch, cache ? cache->kv_heads : 1);
    if (st != BWLA_OK) return st;
    if ((st = check_cache(cache, batch)) != BWLA_OK) return st;
    if (keep < 0 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > keep || table_out_stride < 0) return BWLA_ERR_SHAPE;
    const int64_t most = keep < batch->max_len ? keep : batch->max_len;
    if ((int64_t)table_out_stride * cache->page_size < most) return BWLA_ERR_SHAPE;
    if ((d_position == nullptr) != (d_position_out == nullptr)) return BWLA_ERR_NULL;
    if (d_position && position_stride < batch->max_len) return BWLA_ERR_SHAPE;
    if (batch->sequences == 0) return BWLA_OK;
    if (!d_len_out || !d_weights || (most > 0 && !d_table_out) || (evict_bytes(batch) > 0 && !d_ws)) return BWLA_ERR_NULL;
    if (off16(d_weights) || off16(d_ws)) return BWLA_ERR_ALIGN;
    if (ws_bytes < evict_bytes(batch)) return BWLA_ERR_BUFSIZE;
    EvictArgs a = {};
    const int es = elem_bytes(cache->dtype);
    a.k = (char*)cache->d_k;
    a.v = (char*)cache->d_v;
    a.weights = d_weights;
    a.table = batch->d_table;
    a.len = batch->d_len;
    a.table_out = d_table_out;
    a.pos = d_position;
    a.len_out = d_len_out;
    a.kept = d_kept;
    a.pos_out = d_position_out;
    a.keys = (uint32_t*)d_ws;
    a.list = (int32_t*)d_ws + (size_t)batch->sequences * ((batch->max_len + 3) & ~3);
    a.page_bytes = cache->page_stride * es;
    a.head_bytes = cache->head_stride * es;
    a.slot_bytes = cache->slot_stride * es;
    a.pages = (int32_t)cache->pages;
    a.page_shift = page_shift_of(cache->page_size);
    a.hkv = cache->kv_heads;
    a.row_bytes = cache->head_dim * es;
    a.seqs = batch->sequences;
    a.table_stride = batch->table_stride;
    a.table_out_stride = table_out_stride;
    a.max_len = batch->max_len;
    a.keep = keep;
    a.sinks = sinks;
    a.recent = recent;
    a.pos_stride = position_stride;
    return done(bwla_launch_evict(a, (hipStream_t)stream));
}

}  // extern "C"
