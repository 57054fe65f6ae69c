// Norms of the heads of a merged projection's rows, their rotary positions, and the rows' way into the cache, in one pass; into a
// cache of 8-bit codes as well, whose scales belong to a page and head.  And the codes' values read back.
//
//   y = (x - mu) w rsqrt(mean((x - mu)^2) + eps),  (a, b) -> (a cos - b sin, a sin + b cos),  in fp32
//   codes: scale = A / top of the largest magnitude A, or the page's old scale doubled until A fits;  code = nearest(value / scale)
//
// A head of a row belongs to a group of 4 to 64 lanes, which hold it in registers from load to store: an item is VEC pairs to turn, or
// 2 VEC columns that stay, and the sums of a norm are exchanges between a group's lanes.  Codes: a workgroup has the new tokens
// of a page and head, of keys or of values, one for each of its groups in registers (in pages of more tokens than that the others are
// read and computed twice); the largest magnitude goes through LDS, and older codes of the page follow where its scale grew.
//
// Bound by memory, or, with few rows, by the launch and a chain of loads (row, table, angles; in 8 bits the page's scale too).  A prompt of 4096
// rows, 32 query heads and 8 key-value heads of 128, fp32 in, bf16 queries and e4m3 codes out: 32 us, 4.5 TB/s; as it is, 1001 rows in three chunks,
// 17.5 us; sixteen rows 4.0 us, 64 into codes 10.8 with their values read back (5).  A page's tokens by a workgroup that reads them once, in up to
// 1024 threads: with 256, which read most of them twice, that prompt with its reading back takes 51.1 us instead of 44.9 (other inputs each time).
#include <algorithm>

#include "code8.h"

namespace {

template <typename T, int N>
struct __align__(sizeof(T) * N) Vec {
    T v[N];
};
template <int N>
__device__ __forceinline__ void load(const char* base, bool bf, int64_t at, float* x) {
    if (bf) {
        const Vec<uint16_t, N> r = *(const Vec<uint16_t, N>*)(base + at * 2);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = bwla_bf16_to_f32(r.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += N < 4 ? N : 4) {
            constexpr int W = N < 4 ? N : 4;
            const Vec<float, W> r = *(const Vec<float, W>*)(base + (at + i) * 4);
#pragma unroll
            for (int e = 0; e < W; ++e) x[i + e] = r.v[e];
        }
    }
}
template <int N>
__device__ __forceinline__ void store(char* base, bool bf, int64_t at, const float* x) {
    if (bf) {
        Vec<uint16_t, N> r;
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
        *(Vec<uint16_t, N>*)(base + at * 2) = r;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += N < 4 ? N : 4) {
            constexpr int W = N < 4 ? N : 4;
            Vec<float, W> r;
#pragma unroll
            for (int e = 0; e < W; ++e) r.v[e] = x[i + e];
            *(Vec<float, W>*)(base + (at + i) * 4) = r;
        }
    }
}

// items of a head: `turned` of VEC pairs, then those of 2 VEC columns, the last of which may have VEC
struct Items {
    int lanes, items;                    // lanes of a group, a power of two
};
template <int VEC>
constexpr int items_a_lane() { return VEC == 1 ? 2 : 1; }            // (d / 2 items of single pairs at most: 128)

// where the two runs of VEC columns of an item lie; hi < 0: there is none
__device__ __forceinline__ void item_columns(const RopeArgs& a, int vec, int item, bool turns, int& lo, int& hi) {
    const int pairs = turns ? a.pairs : 0, turned = pairs / vec;
    if (item < turned) {
        lo = a.interleaved ? 2 * item * vec : item * vec;
        hi = a.interleaved ? lo + vec : a.pairs + lo;
    } else {
        lo = 2 * pairs + 2 * vec * (item - turned);
        hi = lo + vec < a.d ? lo + vec : -1;
        if (lo >= a.d) lo = -1;
    }
}

__device__ __forceinline__ float group_sum(float v, int lanes) {
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// A row's head, normed and turned: x[it][0 .. VEC) and x[it][VEC .. 2 VEC) are the runs of item lane + lanes * it.  kind 0: query,
// 1: key, 2: value.  All lanes of a wavefront come here (live: whether there is such a head).
template <int VEC, bool XBF>
__device__ __forceinline__ void head_values(const NormArgs& n, Items it, int64_t row, int head, int kind, bool live, int lane, float (&x)[items_a_lane<VEC>()][2 * VEC]) {
    constexpr int IT = items_a_lane<VEC>();
    const RopeArgs& a = n.r;
    const int64_t src = row * a.row_stride + (int64_t)(head + (kind == 0 ? 0 : kind == 1 ? a.hq : a.hq + a.hkv)) * a.d;
    int lo[IT], hi[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        item_columns(a, VEC, lane + i * it.lanes, kind != 2, lo[i], hi[i]);
        if (!live || lane + i * it.lanes >= it.items) lo[i] = hi[i] = -1;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) x[i][e] = 0.f;
        if (lo[i] >= 0) load<VEC>(a.qkv, XBF, src + lo[i], x[i]);
        if (hi[i] >= 0) load<VEC>(a.qkv, XBF, src + hi[i], x[i] + VEC);
    }
    if (kind == 2) return;
    // the angles do not wait for the norm
    const int turned = a.pairs / VEC;
    float co[IT][VEC], si[IT][VEC];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int item = lane + i * it.lanes, p = item * VEC;
        if (lo[i] < 0 || item >= turned) continue;
        const int first = (p >= a.ends[0]) + (p >= a.ends[1]) + (p >= a.ends[2]);
        const int last = (p + VEC - 1 >= a.ends[0]) + (p + VEC - 1 >= a.ends[1]) + (p + VEC - 1 >= a.ends[2]);
        const int at = min(max(a.pos[first * a.tokens + row], 0), a.rows - 1);
        if (first == last) {
            load<VEC>((const char*)a.cos, false, (int64_t)at * a.pairs + p, co[i]);
            load<VEC>((const char*)a.sin, false, (int64_t)at * a.pairs + p, si[i]);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int axis = (p + e >= a.ends[0]) + (p + e >= a.ends[1]) + (p + e >= a.ends[2]);
                const int64_t to = (int64_t)min(max(a.pos[axis * a.tokens + row], 0), a.rows - 1) * a.pairs + p + e;
                co[i][e] = a.cos[to];
                si[i][e] = a.sin[to];
            }
        }
    }
    if (n.normed) {
        const float over = 1.f / (float)a.d;
        float mu = 0.f;
        if (n.centered) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < IT; ++i)
#pragma unroll
                for (int e = 0; e < 2 * VEC; ++e) s += x[i][e] * over;
            mu = group_sum(s, it.lanes);
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
            for (int e = 0; e < 2 * VEC; ++e) {
                x[i][e] -= (e < VEC ? lo[i] : hi[i]) >= 0 ? mu : 0.f;
                s = fmaf(x[i][e], x[i][e], s);
            }
        s = group_sum(s, it.lanes);
        float f = rsqrtf(fmaf(s, over, n.eps));
        // squares beyond fp32's range: those of 2^-70 of the numbers (eps is nothing beside them)
        if (__builtin_expect(__any(s > 3.0e38f), 0)) {
            constexpr float DOWN = 0x1p-70f;
            float t = 0.f;
#pragma unroll
            for (int i = 0; i < IT; ++i)
#pragma unroll
                for (int e = 0; e < 2 * VEC; ++e) t = fmaf(x[i][e] * DOWN, x[i][e] * DOWN, t);
            t = group_sum(t, it.lanes);
            if (s > 3.0e38f) f = rsqrtf(t * over) * DOWN;
        }
        const float* w = kind == 0 ? n.wq : n.wk;
        if (w) w += head * (kind == 0 ? n.wq_stride : n.wk_stride);
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            float g[2 * VEC];
#pragma unroll
            for (int e = 0; e < 2 * VEC; ++e) g[e] = 1.f;
            if (w && lo[i] >= 0) load<VEC>((const char*)w, false, lo[i], g);
            if (w && hi[i] >= 0) load<VEC>((const char*)w, false, hi[i], g + VEC);
#pragma unroll
            for (int e = 0; e < 2 * VEC; ++e) x[i][e] = x[i][e] * f * g[e];
        }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        if (lo[i] < 0 || lane + i * it.lanes >= turned) continue;
        float y[2 * VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int u = a.interleaved ? 2 * e : e, v = a.interleaved ? 2 * e + 1 : VEC + e;
            y[u] = x[i][u] * co[i][e] - x[i][v] * si[i][e];
            y[v] = x[i][u] * si[i][e] + x[i][v] * co[i][e];
        }
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) x[i][e] = y[e];
    }
}
// where the runs of that head's items are stored
template <int VEC, bool BF>
__device__ __forceinline__ void put_head(const NormArgs& n, Items it, char* base, int64_t dst, int kind, int lane, const float (&x)[items_a_lane<VEC>()][2 * VEC]) {
#pragma unroll
    for (int i = 0; i < items_a_lane<VEC>(); ++i) {
        int lo, hi;
        item_columns(n.r, VEC, lane + i * it.lanes, kind != 2, lo, hi);
        if (lane + i * it.lanes >= it.items) continue;
        if (lo >= 0) store<VEC>(base, BF, dst + lo, x[i]);
        if (hi >= 0) store<VEC>(base, BF, dst + hi, x[i] + VEC);
    }
}

// A row of the call: its sequence, its number among all of the sequence's new tokens, and whether it is one of those that are taken
struct RowOf {
    int b, t, j;                         // j: its index in the cache
    bool live;
};
__device__ __forceinline__ RowOf row_of(const RopeArgs& a, int64_t row) {
    RowOf r;
    r.b = (int)row;
    int64_t r0 = row;
    int fresh = 1, counted = 1;
    r.live = row < a.tokens;
    if (a.first) {
        int lo = 0, up = a.seqs;                       // first[lo] <= row < first[up], if any
        while (up - lo > 1) {
            const int mid = (lo + up) >> 1;
            if (a.first[mid] <= row) lo = mid;
            else up = mid;
        }
        r.b = lo;
        r0 = a.first[lo];
        const int64_t f = (int64_t)a.first[lo + 1] - r0;
        r.live = r.live && r0 >= 0 && row >= r0 && row < r0 + f;         // (else a row of no sequence)
        fresh = (int)min(max(f, (int64_t)0), (int64_t)a.max_new);
        counted = att_counted(f);
    } else {
        r.live = r.live && row < a.seqs;
    }
    r.t = (int)(row - r0);
    r.live = r.live && r.t < fresh;
    r.j = 0;
    if (r.live) r.j = min(max(a.len[r.b], 0), a.max_len) - counted + r.t;
    return r;
}

template <int VEC, bool XBF, bool BF>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormArgs n, Items it) {
    const RopeArgs& a = n.r;
    const int64_t row = blockIdx.x;
    const int job = blockIdx.y * (256 / it.lanes) + threadIdx.x / it.lanes, lane = threadIdx.x & (it.lanes - 1);
    const RowOf r = row_of(a, row);
    if (!r.live) return;
    int page = -1;
    if (r.j >= 0) page = a.table[(int64_t)r.b * a.table_stride + (r.j >> a.page_shift)];
    const bool there = (unsigned)page < (unsigned)a.pages;
    const int slot = r.j & ((1 << a.page_shift) - 1);
    if (job == 0 && lane == 0 && a.cache_pos && r.j >= 0) a.cache_pos[(int64_t)r.b * a.pos_stride + r.j] = a.pos[row];
    const int kind = job < a.hq ? 0 : job < a.hq + a.hkv ? 1 : 2, head = job - (kind == 0 ? 0 : kind == 1 ? a.hq : a.hq + a.hkv);
    const bool live = job < a.hq + 2 * a.hkv && (kind == 0 || there);
    if (kind == 1 && lane == 0 && a.weights && there) a.weights[(((int64_t)page * a.hkv + head) << a.page_shift) + slot] = 0.f;
    float x[items_a_lane<VEC>()][2 * VEC];
    head_values<VEC, XBF>(n, it, row, head, job < a.hq + 2 * a.hkv ? kind : 2, live, lane, x);
    if (!live) return;
    if (kind == 0)
        put_head<VEC, BF>(n, it, a.q, (row * a.hq + head) * a.d, kind, lane, x);
    else
        put_head<VEC, BF>(n, it, kind == 1 ? a.k : a.v, page * a.page_stride + head * a.head_stride + slot * a.slot_stride, kind, lane, x);
}

// finite magnitudes only
__device__ __forceinline__ float magnitude(float v) {
    const float m = fabsf(v);
    return m <= 3.402823466e38f ? m : 0.f;
}
// the largest over a workgroup
__device__ __forceinline__ float block_max(float v, float* words) {
    v = bwla_wave_max(v);
    if ((threadIdx.x & 63) == 0) words[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < (int)blockDim.x / 64; ++w) v = fmaxf(v, words[w]);
    return v;
}
// x / scale, to the last bit but for a few: with the reciprocal alone quotients that lie in the middle of two codes, as those of bf16 values
// often do, would go either way.
template <bool I8, int VEC>
__device__ __forceinline__ void put_codes(uint8_t* dst, const float* x, float scale, float over) {
    constexpr float top = code_top<I8>();
    float y[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const float q = x[e] * over, better = fmaf(fmaf(-q, scale, x[e]), over, q);
        const float v = fminf(fmaxf(fabsf(x[e]) <= 3.402823466e38f ? better : q, -top), top);
        y[e] = q == q ? v : 0.f;                       // (over is 0 where the scale is: infinities become 0 there)
    }
    if constexpr (VEC >= 4) {
        Vec<uint32_t, VEC / 4> w;
#pragma unroll
        for (int e = 0; e < VEC / 4; ++e) w.v[e] = code_of4<I8>(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
        *(Vec<uint32_t, VEC / 4>*)dst = w;
    } else {
        dst[0] = code_of<I8>(y[0]);
    }
}

// The first query_blocks workgroups write queries, of `rows` rows each or of a part of one's heads; of the others each has a page's new
// tokens, of one key-value head's keys or values.
// Page number u of the call: those that sequence b touches begin at first[b] / page + 2 b, which leaves room for each one's.
// ONCE: no page has more new tokens than a workgroup has groups.  (Without the loops over the others' tokens 61 registers
// instead of 101, and twice the wavefronts: 49.8 -> 44.9 us of the prompt named at the top.)
template <int VEC, bool XBF, bool BF, bool I8, bool ONCE>
__global__ __launch_bounds__(1024, (ONCE ? 8 : 4)) void norm_rope8_kernel(NormArgs n, Items it, int64_t query_blocks, int rows) {
    constexpr int IT = items_a_lane<VEC>();
    __shared__ float words[16];
    const RopeArgs& a = n.r;
    const int groups = blockDim.x / it.lanes, group = threadIdx.x / it.lanes, lane = threadIdx.x & (it.lanes - 1);
    if (blockIdx.x < query_blocks) {
        int64_t row;
        int head;
        bool live;
        if (rows > 0) {
            const int r = group / a.hq;
            row = blockIdx.x * (int64_t)rows + r;
            head = group - r * a.hq;
            live = r < rows && row < a.tokens;
        } else {
            const int per = (a.hq + groups - 1) / groups;
            row = blockIdx.x / per;
            head = (int)(blockIdx.x % per) * groups + group;
            live = head < a.hq;
        }
        const RowOf r = row_of(a, live ? row : 0);
        live = live && r.live;
        if (live && head == 0 && lane == 0 && a.cache_pos && r.j >= 0) a.cache_pos[(int64_t)r.b * a.pos_stride + r.j] = a.pos[row];
        float x[IT][2 * VEC];
        head_values<VEC, XBF>(n, it, row, head, 0, live, lane, x);
        if (live) put_head<VEC, BF>(n, it, a.q, (row * a.hq + head) * a.d, 0, lane, x);
        return;
    }
    const int64_t id = blockIdx.x - query_blocks;
    const int job = (int)(id % (2 * a.hkv)), kind = job < a.hkv ? 1 : 2, head = kind == 1 ? job : job - a.hkv;
    const int64_t u = id / (2 * a.hkv);
    // the sequence: the last one whose pages begin at or before u
    int b = (int)u;
    int64_t r0 = u, fresh = 1, behind = 0;
    if (a.first) {
        int lo = 0, up = a.seqs;
        while (up - lo > 1) {
            const int mid = (lo + up) >> 1;
            if ((a.first[mid] >> a.page_shift) + 2ll * mid <= u) lo = mid;
            else up = mid;
        }
        b = lo;
        r0 = a.first[b];
        fresh = (int64_t)a.first[b + 1] - r0;
        behind = u - ((r0 >> a.page_shift) + 2ll * b);
        if (r0 < 0 || r0 > a.tokens || fresh < 0 || behind < 0) return;
    }
    const int len = min(max(a.len[b], 0), a.max_len), start = len - att_counted(fresh);
    fresh = min(min(fresh, a.tokens - r0), (int64_t)a.max_new);
    const int size = 1 << a.page_shift, end = start + (int)fresh;        // new tokens start .. end - 1
    const int64_t e = (max(start, 0) >> a.page_shift) + behind;
    if (end <= 0 || e << a.page_shift >= end) return;
    const int from = max(max(start, 0), (int)e << a.page_shift), to = (int)min((int64_t)end, (e + 1) << a.page_shift);
    const int page = a.table[(int64_t)b * a.table_stride + e];
    if (to <= from || (unsigned)page >= (unsigned)a.pages) return;
    const int inside = from & (size - 1);              // older tokens of the page
    char* const base = (kind == 1 ? a.k : a.v) + page * a.page_stride + head * a.head_stride;
    float* const scale_at = (kind == 1 ? n.k_scale : n.v_scale) + page * n.scale_stride + head;
    const int64_t row_from = r0 + (from - start);
    const int count = to - from;
    float x[IT][2 * VEC];                              // the first token of this group
    float most = 0.f;
    auto values = [&](int t, float (&y)[IT][2 * VEC]) {
        head_values<VEC, XBF>(n, it, row_from + min(t, count - 1), head, kind, t < count, lane, y);
    };
    auto watch = [&](const float (&y)[IT][2 * VEC]) {
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
            for (int c = 0; c < 2 * VEC; ++c) most = fmaxf(most, magnitude(y[i][c]));
    };
    const float was = inside > 0 ? *scale_at : 0.f;
    values(group, x);
    watch(x);
    if constexpr (!ONCE) {
        for (int t = groups; t < count; t += groups) {
            float y[IT][2 * VEC];
            values(t + group, y);
            watch(y);
        }
    }
    most = block_max(most, words);                     // (everyone has read the scale in front of it)
    constexpr float top = code_top<I8>();
    float scale = was;
    int doubled = 0;
    if (!(was > 0.f)) {
        scale = most > 0.f ? fmaxf(most / top, 0x1p-126f) : 0.f;
        doubled = inside > 0 && scale > 0.f ? 1000 : 0;                  // (older codes stood for 0)
    } else {
        // the least number of doublings with most <= (top * was) 2^n
        const float room = top * was;
        if (most > room) {
            doubled = ilogbf(most) - ilogbf(room);
            if (most > ldexpf(room, doubled)) ++doubled;
        }
        if (most > 0.f && ldexpf(was, doubled) < 0x1p-126f) doubled = -126 - ilogbf(was);    // (of which there is no reciprocal)
        scale = ldexpf(was, doubled);
    }
    if (threadIdx.x == 0) *scale_at = scale;
    if (doubled > 0) {
        const int pieces = a.d / 16;
        for (int i = threadIdx.x; i < inside * pieces; i += blockDim.x) {
            c8_v4u* at = (c8_v4u*)(base + (int64_t)(i / pieces) * a.slot_stride + i % pieces * 16);
            c8_v4u w = *at;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[q] = code_of4<I8>(ldexpf(code_value<I8, 0>(w[q]), -doubled), ldexpf(code_value<I8, 1>(w[q]), -doubled),
                                    ldexpf(code_value<I8, 2>(w[q]), -doubled), ldexpf(code_value<I8, 3>(w[q]), -doubled));
            *at = w;
        }
    }
    // (a scale below 2^-126: nothing finite but zeros)
    const float over = scale >= 0x1p-126f ? 1.f / scale : scale > 0.f ? 1.f : 0.f;
    auto put = [&](int t, const float (&y)[IT][2 * VEC]) {
        if (t >= count) return;
        uint8_t* const dst = (uint8_t*)base + (int64_t)((from + t) & (size - 1)) * a.slot_stride;
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            int lo, hi;
            item_columns(a, VEC, lane + i * it.lanes, kind != 2, lo, hi);
            if (lane + i * it.lanes >= it.items) continue;
            if (lo >= 0) put_codes<I8, VEC>(dst + lo, y[i], scale, over);
            if (hi >= 0) put_codes<I8, VEC>(dst + hi, y[i] + VEC, scale, over);
        }
    };
    put(group, x);
    if constexpr (!ONCE) {
        for (int t = groups; t < count; t += groups) {
            float y[IT][2 * VEC];
            values(t + group, y);
            put(t + group, y);
        }
    }
}

// 16 columns of a cached token's key or value a thread
template <bool BF, bool I8>
__global__ __launch_bounds__(256) void cache8_read_kernel(ReadArgs a, int jobs) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int pieces = a.d / 16, b = blockIdx.y;
    const int64_t token = id / (jobs * a.hkv * pieces);
    if (token >= a.max_len) return;
    const int rest = (int)(id - token * (jobs * a.hkv * pieces)), job = rest / (a.hkv * pieces), at = rest - job * a.hkv * pieces;
    const int head = at / pieces, c = (at - head * pieces) * 16, j = (int)token;
    const bool key = jobs == 2 ? job == 0 : a.k_out != nullptr;
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = 0.f;
    if (j < min(max(a.len[b], 0), a.max_len)) {
        const int page = a.table[(int64_t)b * a.table_stride + (j >> a.page_shift)];
        if ((unsigned)page < (unsigned)a.pages) {
            const c8_v4u w = *(const c8_v4u*)((key ? a.k : a.v) + page * a.page_bytes + head * a.head_bytes +
                                        (int64_t)(j & ((1 << a.page_shift) - 1)) * a.slot_bytes + c);
            const float s = (key ? a.k_scale : a.v_scale)[page * a.scale_stride + head];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[4 * i] = code_value<I8, 0>(w[i]) * s;
                y[4 * i + 1] = code_value<I8, 1>(w[i]) * s;
                y[4 * i + 2] = code_value<I8, 2>(w[i]) * s;
                y[4 * i + 3] = code_value<I8, 3>(w[i]) * s;
            }
        }
    }
    const int64_t to = (((int64_t)b * a.max_len + j) * a.hkv + head) * a.d + c;
    store<8>(key ? a.k_out : a.v_out, BF, to, y);
    store<8>(key ? a.k_out : a.v_out, BF, to + 8, y + 8);
}

template <int VEC>
Items items_of(const RopeArgs& a) {
    const int still = a.d - 2 * a.pairs, columns = (a.d + 2 * VEC - 1) / (2 * VEC);
    Items it;
    it.items = a.pairs / VEC + (still + 2 * VEC - 1) / (2 * VEC);
    if (it.items < columns) it.items = columns;        // (values: all columns stay)
    it.lanes = 4;
    while (it.lanes < it.items && it.lanes < 64) it.lanes *= 2;
    return it;
}
// Eight pairs a thread where they come in eights (heads and rows are 16-byte aligned), else four, else one.  (Four instead of eight: that prompt
// 44.9 -> 55.5 us, the chunks 18.3 -> 19.6, 64 rows into codes 10.8 -> 10.6.)
template <typename F>
hipError_t by_pairs(const RopeArgs& a, F go) {
    if ((a.pairs & 7) == 0) return go(std::integral_constant<int, 8>{});
    if ((a.pairs & 3) == 0) return go(std::integral_constant<int, 4>{});
    return go(std::integral_constant<int, 1>{});
}
template <typename F>
hipError_t by_types(bool x, bool y, F go) {
    if (x && y) return go(std::true_type{}, std::true_type{});
    if (x) return go(std::true_type{}, std::false_type{});
    if (y) return go(std::false_type{}, std::true_type{});
    return go(std::false_type{}, std::false_type{});
}

}  // namespace

hipError_t bwla_launch_norm_rope(const NormArgs& n, int x_dtype, int dtype, hipStream_t st) {
    return by_pairs(n.r, [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        const Items it = items_of<V>(n.r);
        const int jobs = n.r.hq + 2 * n.r.hkv, per = 256 / it.lanes;
        const dim3 grid((unsigned)n.r.tokens, (jobs + per - 1) / per);
        return by_types(x_dtype == BWLA_X_BF16, dtype == BWLA_X_BF16, [&](auto x, auto y) {
            norm_rope_kernel<V, decltype(x)::value, decltype(y)::value><<<grid, 256, 0, st>>>(n, it);
            return hipGetLastError();
        });
    });
}

hipError_t bwla_launch_norm_rope8(const NormArgs& n, int x_dtype, int dtype, int code, hipStream_t st) {
    return by_pairs(n.r, [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        const RopeArgs& a = n.r;
        const Items it = items_of<V>(a);
        // as many threads as a page's new tokens have work for, so that each is read once (figures at the top)
        int threads = 64;
        while (threads < 1024 && (int64_t)threads < (int64_t)it.lanes * std::min(a.max_new, 1 << a.page_shift)) threads *= 2;
        const int groups = threads / it.lanes, rows = groups / a.hq;
        const int64_t queries = rows > 0 ? (a.tokens + rows - 1) / rows : a.tokens * ((a.hq + groups - 1) / groups);
        const int64_t units = a.first ? (a.tokens >> a.page_shift) + 2ll * a.seqs : a.seqs;
        const int64_t blocks = queries + units * 2 * a.hkv;
        if (blocks * threads >= 1ll << 32) return hipErrorInvalidConfiguration;       // (a grid has fewer than 2^32 threads)
        return by_types(x_dtype == BWLA_X_BF16, dtype == BWLA_X_BF16, [&](auto x, auto y) {
            constexpr bool X = decltype(x)::value, Y = decltype(y)::value;
            auto go = [&](auto i8, auto once) {
                norm_rope8_kernel<V, X, Y, decltype(i8)::value, decltype(once)::value><<<(unsigned)blocks, threads, 0, st>>>(n, it, queries, rows);
                return hipGetLastError();
            };
            return by_types(code == BWLA_CODE_I8, std::min(a.max_new, 1 << a.page_shift) <= groups, go);
        });
    });
}

hipError_t bwla_launch_cache8_read(const ReadArgs& a, int out_dtype, int code, hipStream_t st) {
    const int jobs = (a.k_out != nullptr) + (a.v_out != nullptr);
    const int64_t blocks = ((int64_t)a.max_len * jobs * a.hkv * (a.d / 16) + 255) / 256;
    if (blocks >= 1ll << 24) return hipErrorInvalidConfiguration;
    return by_types(out_dtype == BWLA_X_BF16, code == BWLA_CODE_I8, [&](auto y, auto i8) {
        cache8_read_kernel<decltype(y)::value, decltype(i8)::value><<<dim3((unsigned)blocks, a.seqs), 256, 0, st>>>(a, jobs);
        return hipGetLastError();
    });
}
