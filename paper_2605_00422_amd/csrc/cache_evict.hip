// Eviction: each sequence's heaviest tokens, moved in order to pages of their own.
//
// Three launches: the tokens' weights as integers of the same order (sum over the heads in 64 bits, rounded once);
// per sequence the keep-th largest of them by a radix selection (11, 11 and 10 bits a pass over counts in LDS: the first digit
// holds the exponent and two bits more, so that a pass's additions spread over many words), and the kept tokens' list
// by prefix sums in index order, so that ties fall to the lowest index; the copy of keys, values and sums, one thread
// 16 bytes, from anywhere to anywhere, since the pages written are no others' pages.  In the second launch a thread
// has a run of neighbouring tokens, whose integers stay in registers up to 32 of them.  Short sequences (EV_SHORT) have
// their integers made there, too, which spares a launch.
// 16 sequences of 9000 to 16384 tokens, 8 heads of 128 bf16 columns, cut to 4096: integers 5 us, selection 24 (one workgroup a
// sequence), copy 112, 4.8 TB/s, what a large copy reaches.  Three of 300 to 601: 8 and 3 us.
#include "attention.h"

namespace {

constexpr int EV_T = 1024;
constexpr int EV_SHORT = 2 * EV_T;

// a token's weight as an integer of the same order: 0 where its page does not exist, all ones where it stays anyway
__device__ __forceinline__ uint32_t evict_key(const EvictArgs& a, int b, int n, int j) {
    const int p = a.table[(int64_t)b * a.table_stride + (j >> a.page_shift)];
    if ((unsigned)p >= (unsigned)a.pages) return 0;
    if (j < a.sinks || j >= n - a.recent) return 0xffffffffu;
    const float* w = a.weights + (((int64_t)p * a.hkv) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
    double sum = 0.0;
#pragma unroll 4
    for (int h = 0; h < a.hkv; ++h) sum += (double)w[(int64_t)h << a.page_shift];
    const float f = sum != sum ? -INFINITY : (float)sum + 0.f;         // (+ 0: one zero)
    const uint32_t u = __float_as_uint(f);
    return u >> 31 ? ~u : u | 0x80000000u;             // (-inf: 0x007fffff, +inf: 0xff800000)
}

__global__ __launch_bounds__(256) void evict_keys_kernel(EvictArgs a) {
    const int b = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
    const int n = min(max(a.len[b], 0), a.max_len);
    if (j < n) a.keys[(int64_t)b * ((a.max_len + 3) & ~3) + j] = evict_key(a, b, n, j);
}

// sum of v over the threads before this one, and over all of them; red: a word of LDS for each wavefront
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

// RUN: integers that a thread holds in registers, 0: none, they are read each time
template <int RUN>
__global__ __launch_bounds__(EV_T) void evict_pick_kernel(EvictArgs a) {
    __shared__ int hist[4][2048];                      // four copies: neighbouring lanes mostly have the same first digit
    __shared__ int red[EV_T / 64];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int n = min(max(a.len[b], 0), a.max_len);
    const uint32_t* keys = a.keys + (int64_t)b * ((a.max_len + 3) & ~3);
    int* list = a.list + (int64_t)b * a.max_len;
    const int run = RUN ? RUN : (n + EV_T - 1) / EV_T, j0 = min(tid * run, n), len = min(run, n - j0);

    uint32_t own[RUN ? RUN : 1];
    if constexpr (RUN != 0) {
#pragma unroll
        for (int i = 0; i < RUN; ++i) own[i] = 0;
        if constexpr (RUN * EV_T <= EV_SHORT) {
#pragma unroll
            for (int i = 0; i < RUN; ++i)
                if (i < len) own[i] = evict_key(a, b, n, j0 + i);
        } else {
#pragma unroll
            for (int i = 0; i < RUN; i += 4)
                if (i < len) {                         // (rows are padded to four)
                    const uint4 x = *(const uint4*)(keys + j0 + i);
                    own[i] = x.x;
                    own[i + 1] = i + 1 < len ? x.y : 0;
                    own[i + 2] = i + 2 < len ? x.z : 0;
                    own[i + 3] = i + 3 < len ? x.w : 0;
                }
        }
    }
    auto each = [&](auto f) {                          // f(key, token) in order; tokens that do not exist have key 0
        if constexpr (RUN != 0) {
#pragma unroll
            for (int i = 0; i < RUN; ++i) f(own[i], j0 + i);
        } else {
            for (int i = 0; i < len; ++i) f(keys[j0 + i], j0 + i);
        }
    };

    int mine = 0, exist;
    each([&](uint32_t k, int) { mine += k != 0; });
    scan(mine, red, exist);
    const int kept = min(exist, a.keep);
    // the kept-th largest integer, and how many of its equals are kept
    uint32_t limit = 1;
    int equals = 0;                                    // exist <= keep: all that is above 0
    if (exist > a.keep && a.keep > 0) {
        if (tid == 0) { s_prefix = 0; s_need = a.keep; }
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
            for (int i = tid; i < 4 * 2048; i += EV_T) (&hist[0][0])[i] = 0;
            __syncthreads();
            const uint32_t prefix = s_prefix;
            each([&](uint32_t k, int) {
                if (k != 0 && (pass == 0 || (k ^ prefix) >> (pass == 1 ? 21 : 10) == 0)) atomicAdd(&hist[tid & 3][(k >> shift) & (bins - 1)], 1);
            });
            __syncthreads();
            // digits from the largest down, two a thread: the one in which the count reaches what is needed
            const int hi = bins - 1 - 2 * tid;
            int c0 = 0, c1 = 0;
            if (hi >= 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) { c0 += hist[i][hi]; c1 += hist[i][hi - 1]; }
            }
            int total;
            const int before = scan(c0 + c1, red, total), need = s_need;
            __syncthreads();
            if (before < need && before + c0 + c1 >= need) {
                const bool second = before + c0 < need;
                s_prefix = prefix | (uint32_t)(hi - second) << shift;
                s_need = need - before - (second ? c0 : 0);
            }
            __syncthreads();
        }
        limit = s_prefix;
        equals = s_need;
    }
    if (a.keep == 0) limit = 0xffffffffu, equals = -1;
    // this thread's part: what lies above, and of the equals those that come first
    int above = 0, same = 0, total;
    each([&](uint32_t k, int) { above += k > limit; same += k == limit; });
    int left = 0;                                      // equals that are still to take when this thread's turn comes
    if (equals > 0) left = equals - scan(same, red, total);
    else if (equals == 0) left = 1 << 30;
    else above = 0;
    int at = scan(above + min(same, max(left, 0)), red, total);
    each([&](uint32_t k, int j) {
        const bool take = equals >= 0 && (k > limit || (k == limit && left-- > 0));
        if (take) {
            list[at] = j;
            if (a.kept) a.kept[(int64_t)b * a.keep + at] = j;
            if (a.pos) a.pos_out[(int64_t)b * a.keep + at] = a.pos[(int64_t)b * a.pos_stride + j];
            ++at;
        }
    });
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
    hipError_t e = hipSuccess;
    if (a.max_len > EV_SHORT) {
        evict_keys_kernel<<<dim3((a.max_len + 255) / 256, a.seqs), 256, 0, st>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (a.max_len <= EV_SHORT) evict_pick_kernel<2><<<a.seqs, EV_T, 0, st>>>(a);
    else if (a.max_len <= 4 * EV_T) evict_pick_kernel<4><<<a.seqs, EV_T, 0, st>>>(a);
    else if (a.max_len <= 8 * EV_T) evict_pick_kernel<8><<<a.seqs, EV_T, 0, st>>>(a);
    else if (a.max_len <= 16 * EV_T) evict_pick_kernel<16><<<a.seqs, EV_T, 0, st>>>(a);
    else if (a.max_len <= 32 * EV_T) evict_pick_kernel<32><<<a.seqs, EV_T, 0, st>>>(a);
    else evict_pick_kernel<0><<<a.seqs, EV_T, 0, st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;                   // (a list that was not made is not followed)
    const int pieces = a.row_bytes / 16;
    const int64_t work = (int64_t)(a.keep < a.max_len ? a.keep : a.max_len) * pieces;
    if (work > 0) evict_copy_kernel<<<dim3((unsigned)((work + 255) / 256), a.hkv, a.seqs), 256, 0, st>>>(a, pieces);
    return hipGetLastError();
}
