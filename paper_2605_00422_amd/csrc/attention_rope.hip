// Rotary positions of a merged projection's rows, and the rows' way into the cache.
//
//   (a, b) -> (a cos - b sin, a sin + b cos)  for each pair of columns, in fp32, rounded once to the cache's type
//
// One pass: each value is read once and written once.  A thread takes VEC pairs of one head (or VEC columns that stay);
// the row of the tables that a pair needs follows from its axis.  The work is bound by memory, and by the chain
// position -> table row and sequence -> page where there are few rows: a row's heads are dealt out over workgroups.
// 4096 rows of 64 + 8 heads on three axes, fp32 to bf16: 52.7 us, 4.8 TB/s, what a large copy reaches; 16 rows of 40 + 8: 3.7 us.
#include "attention.h"

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

template <int VEC, bool XBF, bool BF>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeArgs a, int items) {
    const int64_t row = blockIdx.x;
    const int item = blockIdx.y * 256 + threadIdx.x;
    // the row's sequence: the last one that starts at or before it
    int b = (int)row;
    int64_t r0 = row;
    int fresh = 1, counted = 1;
    if (a.first) {
        int lo = 0, up = a.seqs;                       // first[lo] <= row < first[up], if any
        while (up - lo > 1) {
            const int mid = (lo + up) >> 1;
            if (a.first[mid] <= row) lo = mid;
            else up = mid;
        }
        b = lo;
        r0 = a.first[b];
        const int64_t f = (int64_t)a.first[b + 1] - r0;
        if (r0 < 0 || row < r0 || row >= r0 + f) return;                 // a row of no sequence
        fresh = (int)min(f, (int64_t)a.max_new);
        counted = att_counted(f);
    } else if (b >= a.seqs) {
        return;
    }
    const int t = (int)(row - r0);
    if (t >= fresh) return;
    const int n = min(max(a.len[b], 0), a.max_len);
    const int j = n - counted + t;                       // its index in the cache
    int page = -1;
    if (j >= 0) page = a.table[(int64_t)b * a.table_stride + (j >> a.page_shift)];
    const bool there = (unsigned)page < (unsigned)a.pages;
    const int slot = j & ((1 << a.page_shift) - 1);

    if (item == 0 && a.cache_pos && j >= 0) a.cache_pos[(int64_t)b * a.pos_stride + j] = a.pos[row];
    if (item < a.hkv && a.weights && there) a.weights[(((int64_t)page * a.hkv + item) << a.page_shift) + slot] = 0.f;
    if (item >= items) return;

    const int groups = a.pairs / VEC, still = (a.d - 2 * a.pairs) / VEC, turned = groups + still, plain = a.d / VEC;
    const int turned_items = (a.hq + a.hkv) * turned;
    int head, g;
    if (item < turned_items) {
        head = item / turned;
        g = item - head * turned;
    } else {
        head = (item - turned_items) / plain;
        g = item - turned_items - head * plain;
        head += a.hq + a.hkv;
    }
    const int64_t src = row * a.row_stride + (int64_t)head * a.d;
    char* base;
    int64_t dst;
    if (head < a.hq) {
        base = a.q;
        dst = (row * a.hq + head) * a.d;
    } else {
        if (!there) return;
        const bool key = head < a.hq + a.hkv;
        base = key ? a.k : a.v;
        dst = page * a.page_stride + (int64_t)(head - a.hq - (key ? 0 : a.hkv)) * a.head_stride + slot * a.slot_stride;
    }
    if (head >= a.hq + a.hkv || g >= groups) {
        const int c = head >= a.hq + a.hkv ? g * VEC : 2 * a.pairs + (g - groups) * VEC;
        float x[VEC];
        load<VEC>(a.qkv, XBF, src + c, x);
        store<VEC>(base, BF, dst + c, x);
        return;
    }
    const int p = g * VEC;
    float co[VEC], si[VEC], x[VEC], y[VEC];
    if (a.interleaved) {
        float z[2 * VEC];
        load<VEC>(a.qkv, XBF, src + 2 * p, z);
        load<VEC>(a.qkv, XBF, src + 2 * p + VEC, z + VEC);
#pragma unroll
        for (int i = 0; i < VEC; ++i) { x[i] = z[2 * i]; y[i] = z[2 * i + 1]; }
    } else {
        load<VEC>(a.qkv, XBF, src + p, x);
        load<VEC>(a.qkv, XBF, src + a.pairs + p, y);
    }
    const int axis_a = (p >= a.ends[0]) + (p >= a.ends[1]) + (p >= a.ends[2]);
    const int axis_b = (p + VEC - 1 >= a.ends[0]) + (p + VEC - 1 >= a.ends[1]) + (p + VEC - 1 >= a.ends[2]);
    const int at_a = min(max(a.pos[axis_a * a.tokens + row], 0), a.rows - 1);
    if (axis_a == axis_b) {
        load<VEC>((const char*)a.cos, false, (int64_t)at_a * a.pairs + p, co);
        load<VEC>((const char*)a.sin, false, (int64_t)at_a * a.pairs + p, si);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int axis = (p + i >= a.ends[0]) + (p + i >= a.ends[1]) + (p + i >= a.ends[2]);
            const int64_t at = (int64_t)min(max(a.pos[axis * a.tokens + row], 0), a.rows - 1) * a.pairs + p + i;
            co[i] = a.cos[at];
            si[i] = a.sin[at];
        }
    }
    float u[2 * VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float ru = x[i] * co[i] - y[i] * si[i], rv = x[i] * si[i] + y[i] * co[i];
        if (a.interleaved) { u[2 * i] = ru; u[2 * i + 1] = rv; }
        else { u[i] = ru; u[VEC + i] = rv; }
    }
    store<VEC>(base, BF, a.interleaved ? dst + 2 * p : dst + p, u);
    store<VEC>(base, BF, a.interleaved ? dst + 2 * p + VEC : dst + a.pairs + p, u + VEC);
}

}  // namespace

hipError_t bwla_launch_rope(const RopeArgs& a, int x_dtype, int dtype, hipStream_t st) {
    const bool xbf = x_dtype == BWLA_X_BF16, bf = dtype == BWLA_X_BF16;
    auto go = [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        const int items = (a.hq + a.hkv) * (a.pairs / V + (a.d - 2 * a.pairs) / V) + a.hkv * (a.d / V);
        const dim3 grid((unsigned)a.tokens, (items + 255) / 256);
        if (xbf && bf) rope_append_kernel<V, true, true><<<grid, 256, 0, st>>>(a, items);
        else if (xbf) rope_append_kernel<V, true, false><<<grid, 256, 0, st>>>(a, items);
        else if (bf) rope_append_kernel<V, false, true><<<grid, 256, 0, st>>>(a, items);
        else rope_append_kernel<V, false, false><<<grid, 256, 0, st>>>(a, items);
        return hipGetLastError();
    };
    // eight pairs a thread where they come in eights (heads and rows are 16-byte aligned), else four, else one
    if ((a.pairs & 7) == 0) return go(std::integral_constant<int, 8>{});
    if ((a.pairs & 3) == 0) return go(std::integral_constant<int, 4>{});
    return go(std::integral_constant<int, 1>{});
}
