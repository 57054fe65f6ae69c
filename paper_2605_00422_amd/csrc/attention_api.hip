// C ABI of the cache, the rotary positions, the attention and the eviction: validation on the host, then launches.
// Nothing here allocates device memory, synchronizes or throws.
#include <math.h>
#include <algorithm>

#include "attention.h"

namespace {

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline int elem_bytes(int dtype) { return dtype == BWLA_X_BF16 ? 2 : 4; }
inline bool known_type(int t) { return t == BWLA_X_F32 || t == BWLA_X_BF16; }

int page_shift_of(int32_t page_size) {
    int s = 0;
    while ((1 << s) < page_size) ++s;
    return s;
}

// shapes only: what the workspace sizes depend on
bwla_status_t check_shapes(const bwla_kv_cache_t* c, const bwla_kv_batch_t* b, int32_t q_heads) {
    if (!c || !b) return BWLA_ERR_NULL;
    if (c->pages <= 0 || c->page_size <= 0 || c->kv_heads <= 0 || c->head_dim <= 0 || q_heads <= 0) return BWLA_ERR_SHAPE;
    if (q_heads % c->kv_heads != 0) return BWLA_ERR_SHAPE;
    if (b->sequences < 0 || b->tokens < 0 || b->max_new < 0 || b->max_len < 0 || b->table_stride < 0) return BWLA_ERR_SHAPE;
    if (!known_type(c->dtype)) return BWLA_ERR_UNSUPPORTED;
    if (c->head_dim % 8 != 0 || c->head_dim > BWLA_MAX_HEAD_DIM || q_heads > BWLA_MAX_HEADS) return BWLA_ERR_UNSUPPORTED;
    if ((c->page_size & (c->page_size - 1)) != 0 || c->page_size < 8 || c->page_size > 65536) return BWLA_ERR_UNSUPPORTED;
    if (c->pages > INT32_MAX || b->max_len > BWLA_MAX_CACHE_LEN || b->sequences > 65535 || b->tokens >= 1 << 24) return BWLA_ERR_UNSUPPORTED;
    // (rows of a sequence and key-value head are counted in 32 bits)
    if (std::min<int64_t>(b->max_new, b->tokens) * (q_heads / c->kv_heads) > 1 << 30) return BWLA_ERR_UNSUPPORTED;
    if ((int64_t)b->table_stride * c->page_size < b->max_len) return BWLA_ERR_SHAPE;   // max_len has no room in a row of the table
    return BWLA_OK;
}
bwla_status_t check_cache(const bwla_kv_cache_t* c, const bwla_kv_batch_t* b) {
    if (!c->d_k || !c->d_v) return BWLA_ERR_NULL;
    const int64_t piece = 16 / elem_bytes(c->dtype);
    if (c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < 0) return BWLA_ERR_SHAPE;
    if (c->slot_stride < c->head_dim && c->page_size > 1) return BWLA_ERR_SHAPE;       // slots would overlap
    if (off16(c->d_k) || off16(c->d_v)) return BWLA_ERR_ALIGN;
    if (c->page_stride % piece || c->head_stride % piece || c->slot_stride % piece) return BWLA_ERR_ALIGN;
    if (b->sequences > 0 && (!b->d_len || (!b->d_table && b->max_len > 0))) return BWLA_ERR_NULL;
    return BWLA_OK;
}
// rows of a batch: one a sequence without d_first
bwla_status_t check_rows(const bwla_kv_batch_t* b) {
    if (!b->d_first && b->tokens != b->sequences) return BWLA_ERR_SHAPE;
    return BWLA_OK;
}

AttArgs shape_args(const bwla_kv_cache_t* c, const bwla_kv_batch_t* b, int32_t q_heads) {
    AttArgs a = {};
    const int es = elem_bytes(c->dtype);
    a.k = (const char*)c->d_k;
    a.v = (const char*)c->d_v;
    a.table = b->d_table;
    a.len = b->d_len;
    a.first = b->d_first;
    a.page_bytes = c->page_stride * es;
    a.head_bytes = c->head_stride * es;
    a.slot_bytes = c->slot_stride * es;
    a.tokens = b->tokens;
    a.pages = (int32_t)c->pages;
    a.page_shift = page_shift_of(c->page_size);
    a.hkv = c->kv_heads;
    a.hq = q_heads;
    a.group = q_heads / c->kv_heads;
    a.d = c->head_dim;
    a.seqs = b->sequences;
    a.table_stride = b->table_stride;
    a.max_new = b->d_first ? (int32_t)std::min<int64_t>(b->max_new, b->tokens) : 1;
    a.max_len = b->max_len;
    return a;
}

// all that an attention call checks; *a is filled on success
bwla_status_t attention_args(const bwla_kv_cache_t* c, const bwla_kv_batch_t* b, const bwla_score_t* s, const void* d_q,
                             int64_t q_stride, int32_t q_heads, AttArgs* a) {
    bwla_status_t st = check_shapes(c, b, q_heads);
    if (st != BWLA_OK) return st;
    if (!s) return BWLA_ERR_NULL;
    if ((st = check_cache(c, b)) != BWLA_OK) return st;
    if ((st = check_rows(b)) != BWLA_OK) return st;
    if (!(s->scale > 0.f) || !isfinite(s->scale) || !(s->cap >= 0.f) || !isfinite(s->cap) || s->window < 0) return BWLA_ERR_SHAPE;
    if ((s->d_doc || s->d_position) && s->index_stride < b->max_len) return BWLA_ERR_SHAPE;
    if (b->tokens > 0 && !d_q) return BWLA_ERR_NULL;
    if (q_stride < (int64_t)q_heads * c->head_dim) return BWLA_ERR_SHAPE;
    const int es = elem_bytes(c->dtype);
    if (off16(d_q) || q_stride * es % 16 != 0) return BWLA_ERR_ALIGN;
    *a = shape_args(c, b, q_heads);
    a->q = (const char*)d_q;
    a->q_bytes = q_stride * es;
    a->slopes = s->d_slopes;
    a->prefix = s->d_prefix;
    a->doc = s->d_doc;
    a->pos = s->d_position;
    a->index_stride = s->index_stride;
    a->window = s->window > 0 ? s->window : INT32_MAX;
    a->c1 = s->scale * ATT_LOG2E;
    a->c2 = s->cap > 0.f ? s->scale / s->cap : 0.f;
    a->capped = s->cap * ATT_LOG2E;
    // (what the kernels compute with has to be there in fp32: infinite, or rounded to a few bits, it would make NaN or other scores)
    if (!isnormal(a->c1) || (s->cap > 0.f && (!isnormal(a->c2) || !isnormal(a->capped)))) return BWLA_ERR_UNSUPPORTED;
    return BWLA_OK;
}

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

inline bwla_status_t done(hipError_t e) { return e == hipSuccess ? BWLA_OK : BWLA_ERR_HIP; }

}  // namespace

extern "C" {

bwla_status_t bwla_rope_append(const bwla_kv_cache_t* cache, const bwla_kv_batch_t* batch, const bwla_rope_t* rope,
                               const int32_t* d_position, const void* d_qkv, int x_dtype, int64_t row_stride, int32_t q_heads, void* d_q, float* d_weights,
                               int32_t* d_cache_position, int32_t position_stride, void* stream) {
    bwla_status_t st = check_shapes(cache, batch, q_heads);
    if (st != BWLA_OK) return st;
    if (!rope) return BWLA_ERR_NULL;
    if ((st = check_cache(cache, batch)) != BWLA_OK) return st;
    if ((st = check_rows(batch)) != BWLA_OK) return st;
    if (!known_type(x_dtype)) return BWLA_ERR_UNSUPPORTED;
    if (rope->pairs < 0 || 2 * (int64_t)rope->pairs > cache->head_dim || rope->axes < 1 || rope->axes > 4 || rope->rows < 0) return BWLA_ERR_SHAPE;
    int64_t sum = 0;
    for (int i = 0; i < rope->axes; ++i) {
        if (rope->sections[i] < 0) return BWLA_ERR_SHAPE;
        sum += rope->sections[i];
    }
    if (sum != rope->pairs || (rope->pairs > 0 && rope->rows == 0)) return BWLA_ERR_SHAPE;
    const int64_t width = ((int64_t)q_heads + 2 * (int64_t)cache->kv_heads) * cache->head_dim;
    if (row_stride < width) return BWLA_ERR_SHAPE;
    if (d_cache_position && position_stride < batch->max_len) return BWLA_ERR_SHAPE;
    if (batch->tokens == 0 || batch->sequences == 0) return BWLA_OK;
    if (!d_qkv || !d_q || (rope->pairs > 0 && (!rope->d_cos || !rope->d_sin))) return BWLA_ERR_NULL;
    if ((rope->pairs > 0 || d_cache_position) && !d_position) return BWLA_ERR_NULL;
    if (off16(d_qkv) || off16(d_q) || off16(rope->d_cos) || off16(rope->d_sin) || off16(d_weights)) return BWLA_ERR_ALIGN;
    if (row_stride * elem_bytes(x_dtype) % 16 != 0) return BWLA_ERR_ALIGN;
    RopeArgs a = {};
    a.qkv = (const char*)d_qkv;
    a.k = (char*)cache->d_k;
    a.v = (char*)cache->d_v;
    a.q = (char*)d_q;
    a.cos = rope->d_cos;
    a.sin = rope->d_sin;
    a.pos = d_position;
    a.table = batch->d_table;
    a.len = batch->d_len;
    a.first = batch->d_first;
    a.weights = d_weights;
    a.cache_pos = d_cache_position;
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.slot_stride = cache->slot_stride;
    a.row_stride = row_stride;
    a.tokens = batch->tokens;
    a.pages = (int32_t)cache->pages;
    a.page_shift = page_shift_of(cache->page_size);
    a.hkv = cache->kv_heads;
    a.hq = q_heads;
    a.d = cache->head_dim;
    a.seqs = batch->sequences;
    a.table_stride = batch->table_stride;
    a.max_new = batch->d_first ? batch->max_new : 1;
    a.max_len = batch->max_len;
    a.pos_stride = position_stride;
    a.rows = rope->rows;
    a.pairs = rope->pairs;
    a.axes = rope->axes;
    a.interleaved = rope->interleaved != 0;
    int end = 0;
    for (int i = 0; i < 4; ++i) {
        end += i < rope->axes ? rope->sections[i] : 0;
        a.ends[i] = i < rope->axes - 1 ? end : INT32_MAX;
    }
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
