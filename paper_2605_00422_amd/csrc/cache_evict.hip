// Eviction: each sequence's heaviest tokens, moved in order to pages of their own.
//
// Three launches: the tokens' weights as integers of the same order (sum over the heads in 64 bits, rounded once);
// per sequence the keep-th largest of them by a radix selection, eight bits a pass over counts in LDS, and the kept
// tokens' list by prefix sums in index order, so that ties fall to the lowest index; the copy of keys, values and sums,
// one thread 16 bytes, from anywhere to anywhere, since the pages written are no others' pages.
#include "attention.h"

namespace {

__global__ __launch_bounds__(256) void evict_keys_kernel(EvictArgs a) {
    const int b = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
    const int n = min(max(a.len[b], 0), a.max_len);
    if (j >= n) return;
    const int p = a.table[(int64_t)b * a.table_stride + (j >> a.page_shift)];
    uint32_t key = 0;                                  // below every weight: the page does not exist
    if ((unsigned)p < (unsigned)a.pages) {
        const float* w = a.weights + (((int64_t)p * a.hkv) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        double sum = 0.0;
        for (int h = 0; h < a.hkv; ++h) sum += (double)w[(int64_t)h << a.page_shift];
        const float f = sum != sum ? -INFINITY : (float)sum + 0.f;     // (+ 0: one zero)
        const uint32_t u = __float_as_uint(f);
        key = u >> 31 ? ~u : u | 0x80000000u;
        if (j < a.sinks || j >= n - a.recent) key = 0xffffffffu;
    }
    a.keys[(int64_t)b * a.max_len + j] = key;
}

constexpr int EV_T = 1024;

// sum of v over the threads before this one, and over all of them; red: 17 words of LDS
__device__ __forceinline__ int scan(int v, int* red, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) red[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < EV_T / 64; ++w) {
        if (w < wave) before += red[w];
        total += red[w];
    }
    return before + x - v;
}

__global__ __launch_bounds__(EV_T) void evict_pick_kernel(EvictArgs a) {
    __shared__ int hist[256];
    __shared__ int red[EV_T / 64];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int n = min(max(a.len[b], 0), a.max_len);
    const uint32_t* keys = a.keys + (int64_t)b * a.max_len;
    int* list = a.list + (int64_t)b * a.max_len;

    int mine = 0, exist;
    for (int j = tid; j < n; j += EV_T) mine += keys[j] != 0;
    scan(mine, red, exist);
    const int kept = min(exist, a.keep);
    // the kept-th largest key, and how many of its equals belong to the kept
    uint32_t limit = 1;
    int equals = 0;                                    // with exist <= keep: all above 0
    if (exist > a.keep) {
        if (tid == 0) { s_prefix = 0; s_need = a.keep; }
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            const uint32_t prefix = s_prefix;
            for (int j = tid; j < n; j += EV_T) {
                const uint32_t k = keys[j];
                if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&hist[(k >> shift) & 255], 1);
            }
            __syncthreads();
            // digits from the largest down: the one in which the count reaches what is needed
            const int c = tid < 256 ? hist[255 - tid] : 0;
            int total;
            const int before = scan(c, red, total);
            const int need = s_need;
            __syncthreads();
            if (tid < 256 && before < need && before + c >= need) {
                s_prefix = prefix | (uint32_t)(255 - tid) << shift;
                s_need = need - before;
            }
            __syncthreads();
        }
        limit = s_prefix;
        equals = s_need;
    }
    int out = 0, same = 0;                             // kept so far, equals so far
    for (int j0 = 0; j0 < n; j0 += EV_T) {
        const int j = j0 + tid;
        const uint32_t k = j < n ? keys[j] : 0;
        bool take = k > limit || (equals == 0 && k == limit);
        if (equals > 0) {
            int total;
            const int before = same + scan(k == limit, red, total);
            take = k > limit || (k == limit && before < equals);
            same += total;
        }
        int total;
        const int at = out + scan(take, red, total);
        if (take) {
            list[at] = j;
            if (a.kept) a.kept[(int64_t)b * a.keep + at] = j;
            if (a.pos) a.pos_out[(int64_t)b * a.keep + at] = a.pos[(int64_t)b * a.pos_stride + j];
        }
        out += total;
    }
    for (int i = kept + tid; i < a.keep; i += EV_T) {
        if (a.kept) a.kept[(int64_t)b * a.keep + i] = -1;
        if (a.pos) a.pos_out[(int64_t)b * a.keep + i] = -1;
    }
    if (tid == 0) a.len_out[b] = kept;
}

// A thread moves 16 bytes of a key and of its value; pieces of a row are neighbours.
__global__ __launch_bounds__(256) void evict_copy_kernel(EvictArgs a, int pieces) {
    const int b = blockIdx.z, h = blockIdx.y;
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int i = (int)(idx / pieces), piece = (int)(idx - (int64_t)i * pieces);
    if (i >= a.len_out[b]) return;
    const int j = a.list[(int64_t)b * a.max_len + i], mask = (1 << a.page_shift) - 1;
    const int from = a.table[(int64_t)b * a.table_stride + (j >> a.page_shift)];
    const int to = a.table_out[(int64_t)b * a.table_out_stride + (i >> a.page_shift)];
    if ((unsigned)to >= (unsigned)a.pages || (unsigned)from >= (unsigned)a.pages) return;
    const int64_t src = (int64_t)from * a.page_bytes + (int64_t)h * a.head_bytes + (int64_t)(j & mask) * a.slot_bytes + piece * 16;
    const int64_t dst = (int64_t)to * a.page_bytes + (int64_t)h * a.head_bytes + (int64_t)(i & mask) * a.slot_bytes + piece * 16;
    const uint4 x = *(const uint4*)(a.k + src), y = *(const uint4*)(a.v + src);
    *(uint4*)(a.k + dst) = x;
    *(uint4*)(a.v + dst) = y;
    if (piece == 0)
        a.weights[(((int64_t)to * a.hkv + h) << a.page_shift) + (i & mask)] = a.weights[(((int64_t)from * a.hkv + h) << a.page_shift) + (j & mask)];
}

}  // namespace

hipError_t bwla_launch_evict(const EvictArgs& a, hipStream_t st) {
    if (a.max_len > 0) evict_keys_kernel<<<dim3((a.max_len + 255) / 256, a.seqs), 256, 0, st>>>(a);
    evict_pick_kernel<<<a.seqs, EV_T, 0, st>>>(a);
    const int pieces = a.row_bytes / 16;
    const int64_t work = (int64_t)(a.keep < a.max_len ? a.keep : a.max_len) * pieces;
    if (work > 0) evict_copy_kernel<<<dim3((unsigned)((work + 255) / 256), a.hkv, a.seqs), 256, 0, st>>>(a, pieces);
    return hipGetLastError();
}
