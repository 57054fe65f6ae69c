// C ABI of the normed heads, the cache of 8-bit codes, the attention over it and a step's tables: validation on the host, then launches.
// Nothing here allocates device memory, synchronizes or throws.
#include "attention_host.h"

namespace {

// eps and weights of a norm; *n is filled
bwla_status_t norm_args(const bwla_head_norm_t* h, int32_t head_dim, NormArgs* n) {
    n->normed = h != nullptr;
    if (!h) return BWLA_OK;
    if (!(h->eps > 0.f) || !isnormal(h->eps)) return BWLA_ERR_SHAPE;
    for (const int64_t stride : {h->q_stride, h->k_stride}) {
        if (stride != 0 && stride < head_dim) return BWLA_ERR_SHAPE;
        if (stride % 4 != 0) return BWLA_ERR_ALIGN;
    }
    if (off16(h->d_q) || off16(h->d_k)) return BWLA_ERR_ALIGN;
    n->wq = h->d_q;
    n->wk = h->d_k;
    n->wq_stride = h->q_stride;
    n->wk_stride = h->k_stride;
    n->eps = h->eps;
    n->centered = h->centered != 0;
    return BWLA_OK;
}

// the fields that a cache of codes shares with the others; its strides are bytes
bwla_kv_cache_t like(const bwla_kv_cache8_t* c) {
    return bwla_kv_cache_t{c->d_k, c->d_v, c->page_stride, c->head_stride, c->slot_stride, c->pages, c->page_size, c->kv_heads, c->head_dim, c->dtype};
}
bwla_status_t check_codes(const bwla_kv_cache8_t* c, bool pointers) {
    if (c->code != BWLA_CODE_I8 && c->code != BWLA_CODE_E4M3) return BWLA_ERR_UNSUPPORTED;
    if (c->head_dim % 16 != 0) return BWLA_ERR_UNSUPPORTED;
    if (!pointers) return BWLA_OK;
    if (!c->d_k_scale || !c->d_v_scale) return BWLA_ERR_NULL;
    if (c->scale_stride < c->kv_heads) return BWLA_ERR_SHAPE;
    if (c->page_stride % 16 || c->head_stride % 16 || c->slot_stride % 16 || off16(c->d_k_scale) || off16(c->d_v_scale)) return BWLA_ERR_ALIGN;
    return BWLA_OK;
}

size_t forward8_bytes(const AttArgs& a) {
    if (a.seqs == 0 || a.max_new == 0) return 0;
    const AttSplit p = bwla_att_is_split(a) ? bwla_att_split(a, false) : bwla_att_tile_split(a);
    return p.part_bytes + p.stat_bytes;
}

}  // namespace

extern "C" {

bwla_status_t bwla_norm_rope_append(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, const bwla_rope_t* rope,
                                    const bwla_head_norm_t* norm, const int32_t* d_position, const void* d_qkv, int x_dtype,
                                    int64_t row_stride, int32_t q_heads, void* d_q, float* d_weights, int32_t* d_cache_position,
                                    int32_t position_stride, void* stream) {
    NormArgs n = {};
    bool idle;
    bwla_status_t st = rope_args(cache, batch, rope, d_position, d_qkv, x_dtype, row_stride, q_heads, d_q, d_weights, d_cache_position,
                                 position_stride, &n.r, &idle);
    if (st != BWLA_OK || (st = norm_args(norm, cache->head_dim, &n)) != BWLA_OK || idle) return st;
    if (!norm) return done(bwla_launch_rope(n.r, x_dtype, cache->dtype, (hipStream_t)stream));
    return done(bwla_launch_norm_rope(n, x_dtype, cache->dtype, (hipStream_t)stream));
}

bwla_status_t bwla_norm_rope_append8(const bwla_kv_cache8_t* cache, const bwla_kv_batch_t* batch, const bwla_rope_t* rope,
                                     const bwla_head_norm_t* norm, const int32_t* d_position, const void* d_qkv, int x_dtype,
                                     int64_t row_stride, int32_t q_heads, void* d_q, int32_t* d_cache_position, int32_t position_stride,
                                     void* stream) {
    if (!cache) return BWLA_ERR_NULL;
    const bwla_kv_cache_t c = like(cache);
    NormArgs n = {};
    bool idle;
    bwla_status_t st = check_shapes(&c, batch, q_heads);
    if (st != BWLA_OK || (st = check_codes(cache, false)) != BWLA_OK) return st;
    st = rope_args(&c, batch, rope, d_position, d_qkv, x_dtype, row_stride, q_heads, d_q, nullptr, d_cache_position, position_stride, &n.r, &idle);
    if (st != BWLA_OK || (st = check_codes(cache, true)) != BWLA_OK || (st = norm_args(norm, cache->head_dim, &n)) != BWLA_OK || idle) return st;
    n.k_scale = cache->d_k_scale;
    n.v_scale = cache->d_v_scale;
    n.scale_stride = cache->scale_stride;
    return done(bwla_launch_norm_rope8(n, x_dtype, cache->dtype, cache->code, (hipStream_t)stream));
}

bwla_status_t bwla_cache8_read(const bwla_kv_cache8_t* cache, const bwla_kv_batch_t* batch, void* d_k, void* d_v, int out_dtype, void* stream) {
    if (!cache) return BWLA_ERR_NULL;
    const bwla_kv_cache_t c = like(cache);
    bwla_status_t st = check_shapes(&c, batch, c.kv_heads);
    if (st != BWLA_OK || (st = check_cache(&c, batch)) != BWLA_OK || (st = check_codes(cache, true)) != BWLA_OK) return st;
    if (!known_type(out_dtype)) return BWLA_ERR_UNSUPPORTED;
    if (off16(d_k) || off16(d_v)) return BWLA_ERR_ALIGN;
    if (batch->sequences == 0 || batch->max_len == 0 || (!d_k && !d_v)) return BWLA_OK;
    ReadArgs a = {};
    a.k = (const char*)cache->d_k;
    a.v = (const char*)cache->d_v;
    a.k_scale = cache->d_k_scale;
    a.v_scale = cache->d_v_scale;
    a.k_out = (char*)d_k;
    a.v_out = (char*)d_v;
    a.table = batch->d_table;
    a.len = batch->d_len;
    a.page_bytes = cache->page_stride;
    a.head_bytes = cache->head_stride;
    a.slot_bytes = cache->slot_stride;
    a.scale_stride = cache->scale_stride;
    a.pages = (int32_t)cache->pages;
    a.page_shift = page_shift_of(cache->page_size);
    a.hkv = cache->kv_heads;
    a.d = cache->head_dim;
    a.seqs = batch->sequences;
    a.table_stride = batch->table_stride;
    a.max_len = batch->max_len;
    return done(bwla_launch_cache8_read(a, out_dtype, cache->code, (hipStream_t)stream));
}

bwla_status_t bwla_attention8_workspace_size(const bwla_kv_cache8_t* cache, const bwla_kv_batch_t* batch, int32_t q_heads, size_t* bytes) {
    if (!bytes || !cache) return BWLA_ERR_NULL;
    const bwla_kv_cache_t c = like(cache);
    bwla_status_t st = check_shapes(&c, batch, q_heads);
    if (st != BWLA_OK || (st = check_codes(cache, false)) != BWLA_OK) return st;
    *bytes = forward8_bytes(shape_args(&c, batch, q_heads));
    return BWLA_OK;
}

bwla_status_t bwla_attention8_forward(const bwla_kv_cache8_t* cache, const bwla_kv_batch_t* batch, const bwla_score_t* score, const void* d_q,
                                      int64_t q_stride, int32_t q_heads, void* d_out, float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
    if (!cache) return BWLA_ERR_NULL;
    const bwla_kv_cache_t c = like(cache);
    AttArgs a;
    bwla_status_t st = check_shapes(&c, batch, q_heads);
    if (st != BWLA_OK || (st = check_codes(cache, false)) != BWLA_OK) return st;
    st = attention_args(&c, batch, score, d_q, q_stride, q_heads, &a);
    if (st != BWLA_OK || (st = check_codes(cache, true)) != BWLA_OK) return st;
    if (batch->tokens == 0 || batch->sequences == 0 || a.max_new == 0) return BWLA_OK;
    if (!d_out) return BWLA_ERR_NULL;
    if (off16(d_out) || off16(d_lse) || off16(d_ws)) return BWLA_ERR_ALIGN;
    const size_t need = forward8_bytes(a);
    if (need > 0 && !d_ws) return BWLA_ERR_NULL;
    if (ws_bytes < need) return BWLA_ERR_BUFSIZE;
    a.page_bytes = cache->page_stride;
    a.head_bytes = cache->head_stride;
    a.slot_bytes = cache->slot_stride;
    a.out = (char*)d_out;
    a.lse = d_lse;
    const Att8 e{cache->d_k_scale, cache->d_v_scale, cache->scale_stride, cache->code};
    const hipStream_t s = (hipStream_t)stream;
    if (bwla_att_is_split(a)) return done(bwla_launch_attention8_split(a, e, bwla_att_split(a, false), cache->dtype, d_ws, s));
    return done(bwla_launch_attention8_tile(a, e, bwla_att_tile_split(a), cache->dtype, d_ws, s));
}

bwla_status_t bwla_batch_build_workspace_size(int32_t sequences, int64_t tokens, size_t* bytes) {
    if (!bytes) return BWLA_ERR_NULL;
    if (sequences < 0 || tokens < 0) return BWLA_ERR_SHAPE;
    if (sequences > 65535 || tokens >= 1 << 24) return BWLA_ERR_UNSUPPORTED;
    *bytes = bwla_build_bytes(sequences);
    return BWLA_OK;
}

bwla_status_t bwla_batch_build(const bwla_page_pool_t* pool, const int32_t* d_len, const int32_t* d_new, const int32_t* d_done,
                               const int32_t* d_shift, int32_t* d_table, int32_t table_stride, int32_t sequences, int64_t tokens,
                               int32_t max_len, int32_t* d_len_out, int32_t* d_first, int32_t* d_position, int64_t* d_slot, int32_t* d_sequence,
                               int32_t* d_status, void* d_ws, size_t ws_bytes, void* stream) {
    if (!pool) return BWLA_ERR_NULL;
    if (pool->capacity <= 0 || pool->pages <= 0 || pool->page_size <= 0 || sequences < 0 || tokens < 0 || table_stride < 0 || max_len < 0)
        return BWLA_ERR_SHAPE;
    if ((pool->page_size & (pool->page_size - 1)) != 0 || pool->page_size < 8 || pool->page_size > 65536) return BWLA_ERR_UNSUPPORTED;
    if (pool->pages > INT32_MAX || max_len > BWLA_MAX_CACHE_LEN || sequences > 65535 || tokens >= 1 << 24) return BWLA_ERR_UNSUPPORTED;
    if ((int64_t)table_stride * pool->page_size < max_len) return BWLA_ERR_SHAPE;
    if (!pool->d_ring || !pool->d_state || !pool->d_state_out || !d_first || !d_status) return BWLA_ERR_NULL;
    if (sequences > 0 && (!d_len || !d_new || !d_len_out || (!d_table && max_len > 0))) return BWLA_ERR_NULL;
    const size_t need = bwla_build_bytes(sequences);
    if (!d_ws) return BWLA_ERR_NULL;
    if (off16(d_ws)) return BWLA_ERR_ALIGN;
    if (ws_bytes < need) return BWLA_ERR_BUFSIZE;
    BuildArgs a = {};
    a.ring = pool->d_ring;
    a.state = pool->d_state;
    a.state_out = pool->d_state_out;
    a.len = d_len;
    a.fresh = d_new;
    a.done = d_done;
    a.shift = d_shift;
    a.table = d_table;
    a.len_out = d_len_out;
    a.first = d_first;
    a.position = d_position;
    a.slot = d_slot;
    a.sequence = d_sequence;
    a.status = d_status;
    a.tokens = tokens;
    a.pages = (int32_t)pool->pages;
    a.capacity = pool->capacity;
    a.page_shift = page_shift_of(pool->page_size);
    a.seqs = sequences;
    a.table_stride = table_stride;
    a.max_len = max_len;
    return done(bwla_launch_build(a, d_ws, (hipStream_t)stream));
}

}  // extern "C"
