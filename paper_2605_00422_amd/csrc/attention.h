// What the kernels between the q|k|v and the o projection share: the arguments, where a cached token lies,
// what a query sees, and how a product becomes a score.
//
// Scores are kept in base 2 throughout: y = score * log2(e), weights are exp2(y - m).  With the product
// a = q.k that is y = a * c1 without a cap (c1 = scale log2 e, positive), C tanh(a * c2) with one
// (C = cap log2 e, c2 = scale / cap), minus slope log2(e) |p - r| with a bias.
#pragma once
#include <type_traits>
#include <utility>

#include "bwla_internal.h"

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr float ATT_LOG2E = 1.4426950408889634f;
constexpr float ATT_LN2 = 0.6931471805599453f;

struct AttArgs {
    const char *k, *v;
    const char* q;
    char* out;
    float* lse;
    float* weights;
    const int32_t *table, *len, *first;
    const float* slopes;
    const int32_t *prefix, *doc, *pos;
    int64_t page_bytes, head_bytes, slot_bytes, q_bytes;   // strides of pages, heads, slots; of the rows of q
    int64_t tokens;
    int32_t pages, page_shift, hkv, hq, group, d;
    int32_t seqs, table_stride, max_new, max_len, index_stride;
    int32_t window;                                        // INT32_MAX: none
    float c1, c2, capped;                                  // capped: C, 0: no cap
};

// launchers (attention_tile*.hip, attention_split.hip, attention_weights.hip, attention_rope.hip, cache_evict.hip)

// how a cache's length is split
struct AttSplit {
    int chunk, splits;       // cached tokens of one workgroup; workgroups along the longest sequence
    int rows;                // rows of a sequence and key-value head: new tokens x group
    int row_tiles;           // tiles of 16 rows
    int pitch;               // cached tokens of a row of the scores that the sums of weights read
    size_t part_bytes, stat_bytes, score_bytes;
};
// few rows
AttSplit bwla_att_split(const AttArgs& a, bool weights);
bool bwla_att_is_split(const AttArgs& a);
hipError_t bwla_launch_attention_split(const AttArgs& a, const AttSplit& s, int dtype, void* ws, hipStream_t st);
// many rows
AttSplit bwla_att_tile_split(const AttArgs& a);
hipError_t bwla_launch_attention_tile(const AttArgs& a, const AttSplit& s, int dtype, void* ws, hipStream_t st);
hipError_t bwla_launch_attention_tile_f32(const AttArgs& a, const AttSplit& s, void* ws, hipStream_t st);
// the parts of either added up
hipError_t bwla_launch_attention_join(const AttArgs& a, const AttSplit& s, int dtype, void* ws, hipStream_t st);

struct AttWeightsPlan {
    int parts;               // the rows of a sequence and key-value head are dealt out over this many workgroups
    size_t bytes;            // scratch for their sums (0: one part)
};
AttWeightsPlan bwla_att_weights_plan(const AttArgs& a, int dtype);
hipError_t bwla_launch_attention_weights(const AttArgs& a, int dtype, void* ws, hipStream_t st);

struct RopeArgs {
    const char* qkv;
    char *k, *v, *q;
    const float *cos, *sin;
    const int32_t *pos, *table, *len, *first;
    float* weights;
    int32_t* cache_pos;
    int64_t page_stride, head_stride, slot_stride, row_stride, tokens;    // elements
    int32_t pages, page_shift, hkv, hq, d, seqs, table_stride, max_new, max_len, pos_stride;
    int32_t rows, pairs, axes, interleaved;
    int32_t ends[4];                                       // first pair behind each axis's section
};
hipError_t bwla_launch_rope(const RopeArgs& a, int x_dtype, int dtype, hipStream_t st);

struct EvictArgs {
    char *k, *v;
    float* weights;
    const int32_t *table, *len, *table_out, *pos;
    int32_t *len_out, *kept, *pos_out;
    uint32_t* keys;                                        // scratch: seqs x (max_len, padded to four), weights as ordered integers
    int32_t* list;                                         // scratch: seqs x max_len, kept tokens
    int64_t page_bytes, head_bytes, slot_bytes;
    int32_t pages, page_shift, hkv, row_bytes, seqs, table_stride, table_out_stride, max_len;
    int32_t keep, sinks, recent, pos_stride;
};
hipError_t bwla_launch_evict(const EvictArgs& a, hipStream_t st);

// heads normed, then turned (attention_norm.hip), into a cache as it is or into one of codes
struct NormArgs {
    RopeArgs r;
    const float *wq, *wk;                                  // weights (null: 1)
    int64_t wq_stride, wk_stride;
    float eps;
    int32_t centered, normed;
    float *k_scale, *v_scale;                              // of a cache of codes, whose strides in r are bytes
    int64_t scale_stride;
};
hipError_t bwla_launch_norm_rope(const NormArgs& a, int x_dtype, int dtype, hipStream_t st);
hipError_t bwla_launch_norm_rope8(const NormArgs& a, int x_dtype, int dtype, int code, hipStream_t st);

struct ReadArgs {
    const char *k, *v;
    const float *k_scale, *v_scale;
    char *k_out, *v_out;
    const int32_t *table, *len;
    int64_t page_bytes, head_bytes, slot_bytes, scale_stride;
    int32_t pages, page_shift, hkv, d, seqs, table_stride, max_len;
};
hipError_t bwla_launch_cache8_read(const ReadArgs& a, int out_dtype, int code, hipStream_t st);

// attention over codes (attention8_split*.hip, attention8_tile*.hip): the rules of the other types say how a call is split
struct Att8 {
    const float *k_scale, *v_scale;
    int64_t stride;
    int32_t code;
};
hipError_t bwla_launch_attention8_split(const AttArgs& a, const Att8& e, const AttSplit& s, int dtype, void* ws, hipStream_t st);
hipError_t bwla_launch_attention8_split_f32(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st);
hipError_t bwla_launch_attention8_tile(const AttArgs& a, const Att8& e, const AttSplit& s, int dtype, void* ws, hipStream_t st);
hipError_t bwla_launch_attention8_tile_e4m3(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st);
hipError_t bwla_launch_attention8_tile_f32(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st);
hipError_t bwla_launch_attention8_tile_f32_e4m3(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st);

struct BuildArgs {
    int32_t* ring;
    const int32_t* state;
    int32_t* state_out;
    const int32_t *len, *fresh, *done, *shift;
    int32_t *table, *len_out, *first, *position;
    int64_t* slot;
    int32_t *sequence, *status;
    int64_t tokens;
    int32_t pages, capacity, page_shift, seqs, table_stride, max_len;
};
size_t bwla_build_bytes(int64_t seqs);
hipError_t bwla_launch_build(const BuildArgs& a, void* ws, hipStream_t st);

#ifdef __HIPCC__
// New tokens of a sequence, all of them, as its length is counted from them.  (A length has 2^24 at most, and so have rows: with this
// many all rows lie in front of the cache.)
__device__ __forceinline__ int att_counted(int64_t fresh) { return (int)min(fresh, (int64_t)1 << 25); }
// A sequence as the kernels see it: what lies outside the caller's bounds is cut off here, once.  Of more new tokens than the call takes
// the first remain, at their own indexes.
struct AttSeq {
    int n, fresh, row0;      // cached tokens, new ones among them, first row of q
    int old;                 // the first new one's index (negative: more new tokens than cached ones)
    int prefix;
    const int32_t *table, *doc, *pos;
};
__device__ __forceinline__ AttSeq att_seq(const AttArgs& a, int b) {
    AttSeq s;
    s.n = min(max(a.len[b], 0), a.max_len);
    int64_t row0 = b, fresh = 1;
    if (a.first) {
        row0 = a.first[b];
        fresh = (int64_t)a.first[b + 1] - row0;
    }
    if (row0 < 0 || row0 > a.tokens || fresh < 0) { row0 = 0; fresh = 0; }
    s.old = s.n - att_counted(fresh);
    s.fresh = (int)min(min(fresh, a.tokens - row0), (int64_t)a.max_new);
    s.row0 = (int)row0;
    s.prefix = a.prefix ? min(a.prefix[b], s.n) : 0;
    // (nothing sees the new tokens that are left out, unless they are in the prefix)
    if (s.fresh < fresh) s.n = max(max(s.old + s.fresh, s.prefix), 0);
    s.table = a.table + (int64_t)b * a.table_stride;
    s.doc = a.doc ? a.doc + (int64_t)b * a.index_stride : nullptr;
    s.pos = a.pos ? a.pos + (int64_t)b * a.index_stride : nullptr;
    return s;
}

// A row of the products: new token t of the sequence, as the mask and the bias see it
struct AttRow {
    int i, p, doc;           // index in the cache (-1: the row sees nothing), position, document
};
__device__ __forceinline__ AttRow att_row(const AttSeq& s, int t, bool live) {
    AttRow r;
    r.i = live ? s.old + t : -1;
    if (r.i < 0) { r.i = -1; r.p = 0; r.doc = -2; return r; }
    r.p = s.pos ? max(s.pos[r.i], 0) : r.i;
    r.doc = s.doc ? s.doc[r.i] : 0;
    if (r.doc < 0) r.doc = -2;
    return r;
}
// A cached token: its position, and its document, -1 where it does not exist (doc of a token in none: -1 too)
struct AttKey {
    int p, doc;
};
__device__ __forceinline__ AttKey att_key(const AttArgs& a, const AttSeq& s, int j, bool there) {
    AttKey k;
    const bool ok = there && j < s.n;
    k.p = s.pos && ok ? max(s.pos[j], 0) : j;
    k.doc = ok ? (s.doc ? max(s.doc[j], -1) : 0) : -1;
    return k;
}
// (rows that see nothing have document -2, keys that nothing sees -1; no short cuts: branches would cost more)
__device__ __forceinline__ bool att_sees(const AttRow& r, int prefix, int window, int j, int kp, int kdoc) {
    return (r.doc == kdoc) & ((j < prefix) | ((j <= r.i) & (r.p - kp < window)));
}
// MFMA takes no notice of the execution mask: whatever a branch around one depends on is made a scalar, so that
// the branch is a jump
__device__ __forceinline__ bool att_uniform(bool x) { return __builtin_amdgcn_readfirstlane((int)x) != 0; }
__device__ __forceinline__ int att_wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// tanh to one or two units of the last place: below 0.6 an odd polynomial (degree 11, fitted to tanh(x) / x in
// x^2, relative error 2.5e-9 before rounding), above by the exponential
constexpr float ATT_NEAR = 0.6f;           // ... up to which the polynomial holds
__device__ __forceinline__ float att_tanh_near(float x) {
    const float u = x * x;
    float p = -0.00585642786f;
    p = fmaf(p, u, 0.0207574754f);
    p = fmaf(p, u, -0.0537699218f);
    p = fmaf(p, u, 0.133317047f);
    p = fmaf(p, u, -0.33333284f);
    return fmaf(p * u, x, x);
}
__device__ __forceinline__ float att_tanh(float x) {
    const float p = att_tanh_near(x);
    const float e = __builtin_amdgcn_exp2f(fabsf(x) * (2.f * ATT_LOG2E));
    const float big = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(1.f + e), x);
    return fabsf(x) < ATT_NEAR ? p : big;
}
__device__ __forceinline__ float att_score(const AttArgs& a, float prod) {
    return a.capped != 0.f ? a.capped * att_tanh(prod * a.c2) : prod * a.c1;
}

// What the kernels of many rows make of products, an instance each: nothing but the scale, or a cap or a bias.  In bf16 the latter take
// tanh as 1 - 2 / (1 + exp), whose error is one of the cap, 1.2e-7 of it, and not of the score: up to ATT_SHORT_CAP (128, in base 2)
// at most 1.5e-5 of a weight, a hundredth of what rounding a weight to bf16 costs.  Above it they take att_tanh, as fp32 does always.
enum AttForm { ATT_PLAIN, ATT_SHORT, ATT_LONG };
constexpr float ATT_SHORT_CAP = 128.f * ATT_LOG2E;
inline AttForm att_form(const AttArgs& a, bool bf) {
    if (a.capped == 0.f && !a.slopes) return ATT_PLAIN;
    return bf && a.capped <= ATT_SHORT_CAP ? ATT_SHORT : ATT_LONG;
}

// Products of 32 keys (rows of the tile) and 32 rows (lanes, in both halves alike) into scores: cap and bias.  (Without either they
// stay products until their weights are taken.)  The tile's keys are number 32 k .. of those behind j0, of which lane i knows the
// position of key i; mp: the row's position.
template <int FORM>
__device__ __forceinline__ void att_transform(const AttArgs& a, v16f& sc, int mp, float slope, int j0, int k, int kp, bool moved) {
    const int hf = (threadIdx.x >> 5) & 1;
    if (a.capped != 0.f) {
        const float C = a.capped, c3 = a.c2 * (2.f * ATT_LOG2E);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if constexpr (FORM == ATT_SHORT)
                sc[r] = fmaf(-2.f * C, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(sc[r] * c3)), C);
            else
                sc[r] = C * att_tanh(sc[r] * a.c2);
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] *= a.c1;
    }
    if (a.slopes && moved) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
            sc[r] = fmaf(-slope, fabsf((float)(mp - __shfl(kp, k * 32 + (r & 3) + 8 * (r >> 2) + 4 * hf, 64))), sc[r]);
    } else if (a.slopes) {
        const float away = (float)(mp - j0 - k * 32 - 4 * hf);
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = fmaf(-slope, fabsf(away - (float)((r & 3) + 8 * (r >> 2))), sc[r]);
    }
}
// What rows (lane i: row i & 31) see of 64 keys (lane i: key j0 + i, and its position and document): a bit for each key
__device__ __forceinline__ uint64_t att_seen(const AttArgs& a, const AttSeq& s, const AttRow& me, int j0, int kp, int kdoc) {
    const int lane = threadIdx.x & 63;
    uint64_t ok = 0;
    if (s.pos && a.window != INT32_MAX) {
        for (int r = 0; r < 32; ++r) {
            const AttRow row{__builtin_amdgcn_readlane(me.i, r), __builtin_amdgcn_readlane(me.p, r), __builtin_amdgcn_readlane(me.doc, r)};
            const uint64_t bits = __ballot(att_sees(row, s.prefix, a.window, j0 + lane, kp, kdoc));
            ok = (lane & 31) == r ? bits : ok;
        }
        return ok;
    }
    for (uint64_t left = __ballot(kdoc >= 0); left;) { // a step for each of the keys' documents, of which there are few
        const int one = __builtin_amdgcn_readlane(kdoc, __builtin_ctzll(left));
        const uint64_t bits = __ballot(kdoc == one);
        ok = me.doc == one ? bits : ok;
        left &= ~bits;
    }
    const int up = me.i - j0, from = up >= a.window ? up - a.window + 1 : 0, pre = s.prefix - j0;
    uint64_t reach = up >= 63 ? ~0ull : up < 0 ? 0 : (2ull << up) - 1;
    reach = from > 63 ? 0 : reach >> from << from;
    reach |= pre > 63 ? ~0ull : pre <= 0 ? 0 : (1ull << pre) - 1;
    return ok & reach;
}
// bits of any of the wavefront's rows (lane i has those of row i & 31), a scalar
__device__ __forceinline__ uint64_t att_rows_or(uint64_t bits) {
    uint32_t w[2] = {(uint32_t)bits, (uint32_t)(bits >> 32)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[i] |= __builtin_amdgcn_mov_dpp(w[i], 0x128, 0xf, 0xf, true);         // 16 lanes turned by 8, 4, 2, 1
        w[i] |= __builtin_amdgcn_mov_dpp(w[i], 0x124, 0xf, 0xf, true);
        w[i] |= __builtin_amdgcn_mov_dpp(w[i], 0x122, 0xf, 0xf, true);
        w[i] |= __builtin_amdgcn_mov_dpp(w[i], 0x121, 0xf, 0xf, true);
        const auto r = __builtin_amdgcn_permlane16_swap(w[i], w[i], false, false);
        w[i] = __builtin_amdgcn_readfirstlane(r[0] | r[1]);
    }
    return ((uint64_t)w[1] << 32) | w[0];
}


// 16 bytes a lane from memory to LDS: lane i's go to dst + 16 i (dst is uniform).  In assembly, since the compiler lets the
// transposing LDS reads wait for every such copy on the way, also those to other buffers (vmcnt(0) in front of each block's second
// product: 954 us for a prompt of 8192 with 32 heads).  The caller waits (vmcnt) before the barrier behind which the copy is read;
// nothing is returned in registers.
// dst: att_lds_address of where the first copy goes, ofs: bytes from there
__device__ __forceinline__ uint32_t att_lds_address(const char* p) {
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p);
}
template <int OFS>
__device__ __forceinline__ void att_copy16(const char* src, uint32_t dst) {
    asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(dst), "i"(OFS) : "memory", "m0", "scc");
}
template <int... I, typename F>
__device__ __forceinline__ void att_each(std::integer_sequence<int, I...>, F f) {
    (f(std::integral_constant<int, I>{}), ...);
}

__device__ __forceinline__ uint32_t att_pack_bf16(float lo, float hi) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    v2bf r;
    r[0] = (__bf16)lo;
    r[1] = (__bf16)hi;
    return __builtin_bit_cast(uint32_t, r);
}
// c plus both bf16 halves of x.  Outputs are divided by the sum of the weights as they enter the second product,
// rounded to bf16, so that a row of one key is that key's value, and of equal values that value; lse is of the fp32 sum.
__device__ __forceinline__ float att_add_bf16(uint32_t x, float c) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, x), __builtin_bit_cast(v2bf, 0x3f803f80u), c, false);
}
// A row's end.  l: the sum of its weights, 0 where it sees nothing, NaN where a score was (as its output then is: such a row is not
// taken for one that sees nothing); lr: the sum as above; at: its place, tokens and heads counted through.
__device__ __forceinline__ float att_over(float l, float lr) { return l == 0.f ? 0.f : 1.f / lr; }
template <bool BF>
__device__ __forceinline__ void att_put(const AttArgs& a, int64_t at, int c, float4 v, float over) {
    const int64_t to = at * a.d + c;
    if constexpr (BF) *(uint2*)(a.out + to * 2) = make_uint2(att_pack_bf16(v.x * over, v.y * over), att_pack_bf16(v.z * over, v.w * over));
    else *(float4*)(a.out + to * 4) = make_float4(v.x * over, v.y * over, v.z * over, v.w * over);
}
__device__ __forceinline__ void att_put_lse(const AttArgs& a, int64_t at, float m, float l) {
    if (a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m + __log2f(l)) * ATT_LN2;
}
// The maximum that stands for a part whose weights add up to l when parts are joined: fmaxf drops NaN, so that a part of nothing else
// would have -inf, as one of which nothing is seen.
__device__ __forceinline__ float att_part_max(float m, float l) { return l != l ? l : m; }
#endif
