// A step's tables from its requests' lengths: pages given back to and taken from a ring of free ones, row offsets, positions and slots.
//
// With n_b cached tokens (0 for a request that starts), m_b new ones and pages of p:  take_b = ceil((n_b + m_b) / p) - ceil(n_b / p).
// Sums over the requests in front (of take_b, of the pages that done requests name, of m_b) say where in the ring and in the rows
// each request's share lies, so that everything else is independent: no atomics, and the same answer for the same arguments.
// Integer work of a few bytes an entry, bound by launches and chains of loads.  Two kernels: requests' shares, added up over groups of 64 (a
// wavefront each, which also counts the pages that are given back); then, for each group, the sums in front of it, its entries of table
// and ring, and its rows, dealt out over as many workgroups as there are rows for: 4096 requests of a token each 7.0 us, of 24 8.0 us; a fortieth
// of them done and prompts in their place, 2 x 10^5 rows, 13.9 us.  (One workgroup for all sums in between, and rows by
// bisection of all offsets: 21.9 us for 4096 requests with 10^5 rows.)  Few requests and rows: all of it by one workgroup, in one launch, 3.6
// us for 64 requests of a token each and 3.8 for 256 (two launches: 6.2 and 6.8); with 1024 rows 6.0 to 7.1 either way, with 4096 18.3
// where two take 7.6.
#include <algorithm>

#include "attention.h"

namespace {

constexpr int BB_FEW = 256;              // requests and rows that one workgroup takes in a launch of its own
constexpr int BB_FEW_ROWS = 1024;

// entry number `at` of a ring behind its front: both below the ring's size
__device__ __forceinline__ int ring_at(int front, int at, int capacity) {
    const uint32_t x = (uint32_t)front + (uint32_t)at;
    return (int)(x >= (uint32_t)capacity ? x - capacity : x);
}
__device__ __forceinline__ int cut(int v, int most) { return min(max(v, 0), most); }
__device__ __forceinline__ int up(int n, int shift) { return (int)(((int64_t)n + (1 << shift) - 1) >> shift); }

// A request: its cached tokens before the call and those that stay, and what it takes, adds and gives back.
struct Share {
    uint32_t take, rows, back, beyond;   // beyond: whether it would be too long
    int32_t old, n;
};
// (old: a.len[b] cut, wherever it stands)
__device__ __forceinline__ Share share_of(const BuildArgs& a, int b, int old, uint32_t back) {
    Share s;
    s.back = back;
    s.old = old;
    s.n = a.done && a.done[b] != 0 ? 0 : old;
    s.rows = max(a.fresh[b], 0);
    const uint32_t size = 1u << a.page_shift;          // (2^31 + 2^24 + 2^16 at most)
    s.take = ((s.n + s.rows + size - 1) >> a.page_shift) - ((s.n + size - 1) >> a.page_shift);
    s.beyond = s.n + s.rows > (uint32_t)a.max_len;
    return s;
}
// pages that request b, which is done, gives back: by a wavefront
__device__ __forceinline__ uint32_t given_back(const BuildArgs& a, int b, int old) {
    const int lane = threadIdx.x & 63, held = up(old, a.page_shift);
    const int32_t* row = a.table + (int64_t)b * a.table_stride;
    uint32_t sum = 0;
    for (int e = 0; e < held; e += 64) sum += __popcll(__ballot(e + lane < held && (uint32_t)row[min(e + lane, held - 1)] < (uint32_t)a.pages));
    return sum;
}
// what a lane's request gives back, 64 of them from b0 on
__device__ __forceinline__ uint32_t all_given_back(const BuildArgs& a, int b0, bool done, int old) {
    const int lane = threadIdx.x & 63;
    uint32_t mine = 0;
    for (uint64_t left = __ballot(done); left; left &= left - 1) {
        const int i = __builtin_ctzll(left);
        const uint32_t k = given_back(a, b0 + i, __builtin_amdgcn_readlane(old, i));
        if (lane == i) mine = k;
    }
    return mine;
}

// Sums that stay at the largest 32-bit number: more than that fits no pool and no batch.
struct Sums {
    uint32_t take, rows, back, beyond;
};
__device__ __forceinline__ uint32_t add(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y) {
    return Sums{add(x.take, y.take), add(x.rows, y.rows), add(x.back, y.back), add(x.beyond, y.beyond)};
}
// over the lanes up to each
__device__ __forceinline__ Sums sums_to(Sums x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const Sums y{__shfl_up(x.take, o, 64), __shfl_up(x.rows, o, 64), __shfl_up(x.back, o, 64), __shfl_up(x.beyond, o, 64)};
        if (lane >= o) x = x + y;
    }
    return x;
}
__device__ __forceinline__ Sums of_lane(const Sums& x, int lane) {
    return Sums{__shfl(x.take, lane, 64), __shfl(x.rows, lane, 64), __shfl(x.back, lane, 64), __shfl(x.beyond, lane, 64)};
}

struct Head {
    int32_t ok, front, count, rows;      // rows: given out in all
};
// (a state that is none: what the ring can hold)
__device__ __forceinline__ int front_of(const BuildArgs& a) { return (int)((uint32_t)a.state[0] % (uint32_t)a.capacity); }
__device__ __forceinline__ int count_of(const BuildArgs& a) { return cut(a.state[1], a.capacity); }
__device__ __forceinline__ Head head_of(const BuildArgs& a, const Sums& all, int front, int count) {
    const bool ok = all.take <= (uint32_t)count && all.rows <= (uint32_t)a.tokens && all.beyond == 0;
    return Head{ok, front, count, ok ? (int)all.rows : 0};
}
__device__ void put_status(const BuildArgs& a, const Sums& all, const Head& h) {
    const auto word = [](uint32_t v) { return (int32_t)min(v, (uint32_t)INT32_MAX); };
    const auto less = [](uint32_t x, uint32_t y) { return x > y ? x - y : 0; };
    a.status[0] = word(less(all.take, h.count));
    a.status[1] = word(all.beyond);
    a.status[2] = word(less(all.rows, (uint32_t)a.tokens));
    a.status[3] = word(all.rows);
    const int taken = h.ok ? (int)all.take : 0;
    a.state_out[0] = ring_at(h.front, taken, a.capacity);
    a.state_out[1] = h.count - taken + (int)min(all.back, (uint32_t)(a.capacity - h.count));
    a.first[0] = 0;
}

// a request's entries of the ring and the table, by a wavefront.  before: what the requests in front of it come to
__device__ void entries(const BuildArgs& a, const Head& h, int b, int old, bool done, uint32_t rows, uint32_t take, uint32_t back) {
    const int lane = threadIdx.x & 63;
    int32_t* row = a.table + (int64_t)b * a.table_stride;
    if (done) {
        const int held = up(old, a.page_shift);
        int64_t at = back;
        for (int e = 0; e < held; e += 64) {
            const int page = e + lane < held ? row[e + lane] : -1;
            const uint64_t there = __ballot((uint32_t)page < (uint32_t)a.pages);
            const int64_t k = at + __popcll(there & ((1ull << lane) - 1));
            // (a pool that has more pages given back than it holds keeps the first)
            if ((uint32_t)page < (uint32_t)a.pages && k < a.capacity - h.count) a.ring[ring_at(h.front, h.count + (int)k, a.capacity)] = page;
            at += __popcll(there);
        }
    }
    if (!h.ok) return;
    const int n = done ? 0 : old, base = up(n, a.page_shift), want = up(n + (int)rows, a.page_shift);
    for (int e = base + lane; e < want; e += 64) row[e] = a.ring[ring_at(h.front, (int)take + e - base, a.capacity)];
}
// Those of the 64 requests from b0 on, a lane each.  A running request takes a page now and then, all of them at once; those that are done
// or take more are done in turn, every `parts`-th here.
__device__ __forceinline__ void group_entries(const BuildArgs& a, const Head& h, int b0, const Share& s, bool done, const Sums& before, int part,
                                              int parts) {
    const int lane = threadIdx.x & 63;
    const bool one = h.ok && !done && s.take == 1;
    if (one && part == 0)
        a.table[(int64_t)(b0 + lane) * a.table_stride + up(s.n, a.page_shift)] = a.ring[ring_at(h.front, (int)before.take, a.capacity)];
    int turn = 0;
    for (uint64_t left = __ballot(done || (h.ok && s.take > 1)); left; left &= left - 1, ++turn) {
        if (turn % parts != part) continue;
        const int i = __builtin_ctzll(left);
        entries(a, h, b0 + i, __builtin_amdgcn_readlane(s.old, i), __builtin_amdgcn_readlane((int)done, i) != 0, __builtin_amdgcn_readlane(s.rows, i),
                __builtin_amdgcn_readlane(before.take, i), __builtin_amdgcn_readlane(before.back, i));
    }
}

// row t of request b, its new token i, behind n tokens that stay; take: pages that the requests in front of it take.  b < 0: of none
__device__ __forceinline__ void one_row(const BuildArgs& a, const Head& h, int t, int b, int i, int n, int take) {
    int64_t slot = -1;
    int at = -1;
    if (b >= 0) {
        const int base = up(n, a.page_shift), j = n + i, e = j >> a.page_shift;
        at = j + (a.shift ? a.shift[b] : 0);
        if (a.slot) {
            // (a page in front of the new ones stands in the table, where this call enters nothing)
            const int page = e >= base ? a.ring[ring_at(h.front, take + e - base, a.capacity)] : a.table[(int64_t)b * a.table_stride + e];
            if ((uint32_t)page < (uint32_t)a.pages) slot = ((int64_t)page << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        }
    }
    if (a.position) a.position[t] = at;
    if (a.slot) a.slot[t] = slot;
    if (a.sequence) a.sequence[t] = b;
}
// the last i with first[i] <= t, of i < n; first[0] <= t
__device__ __forceinline__ int below(const int32_t* first, int n, int t) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(BB_FEW) void build_few_kernel(BuildArgs a) {
    __shared__ int32_t s_n[BB_FEW], s_take[BB_FEW], s_first[BB_FEW + 1];
    __shared__ Sums words[BB_FEW / 64];
    const int b = threadIdx.x, lane = threadIdx.x & 63, wave = att_wave();
    const bool in = b < a.seqs, done = in && a.done && a.done[b] != 0;
    const int old = in ? cut(a.len[b], a.max_len) : 0, front = front_of(a), count = count_of(a);
    const uint32_t back = a.done ? all_given_back(a, wave * 64, done, old) : 0;
    Share s{0, 0, 0, 0, 0, 0};
    if (in) s = share_of(a, b, old, back);
    const Sums to = sums_to(Sums{s.take, s.rows, s.back, s.beyond});
    if (lane == 63) words[wave] = to;
    __syncthreads();                     // (everyone has read lengths and state)
    Sums before{__shfl_up(to.take, 1, 64), __shfl_up(to.rows, 1, 64), __shfl_up(to.back, 1, 64), 0}, all{0, 0, 0, 0};
    if (lane == 0) before = all;
#pragma unroll
    for (int w = 0; w < BB_FEW / 64; ++w) {
        if (w < wave) before = before + words[w];
        all = all + words[w];
    }
    const Head h = head_of(a, all, front, count);
    if (b == 0) put_status(a, all, h);
    const int end = h.ok ? (int)(before.rows + s.rows) : 0;
    s_n[b] = s.n;
    s_take[b] = (int)before.take;
    s_first[b + 1] = end;
    if (b == 0) s_first[0] = 0;
    if (in) {
        a.len_out[b] = s.n + (h.ok ? (int)s.rows : 0);
        a.first[b + 1] = end;
    }
    __syncthreads();
    if (a.position || a.slot || a.sequence)
        for (int t = threadIdx.x; t < a.tokens; t += BB_FEW) {
            const int r = t < h.rows ? below(s_first, a.seqs + 1, t) : -1;
            if (r < 0) one_row(a, h, t, -1, 0, 0, 0);
            else one_row(a, h, t, r, t - s_first[r], s_n[r], s_take[r]);
        }
    group_entries(a, h, wave * 64, s, done, before, 0, 1);
}

// what the first launch leaves
struct Found {
    int32_t *old, *back;                 // of each request
    Sums* group;                         // of each 64 requests
    int32_t* state;                      // front and count
};

__global__ __launch_bounds__(256) void build_sums_kernel(BuildArgs a, Found f) {
    const int g = blockIdx.x * 4 + att_wave(), lane = threadIdx.x & 63, b = g * 64 + lane;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        f.state[0] = front_of(a);
        f.state[1] = count_of(a);
    }
    if (g > 0 && g * 64 >= a.seqs) return;
    const bool in = b < a.seqs, done = in && a.done && a.done[b] != 0;
    const int old = in ? cut(a.len[b], a.max_len) : 0;
    const uint32_t back = a.done ? all_given_back(a, g * 64, done, old) : 0;
    Share s{0, 0, 0, 0, 0, 0};
    if (in) {
        s = share_of(a, b, old, back);
        f.old[b] = old;
        f.back[b] = (int)back;
    }
    const Sums to = sums_to(Sums{s.take, s.rows, s.back, s.beyond});
    if (lane == 63) f.group[g] = to;
}

// Workgroup (group, part): the group's entries and rows, every parts-th of them
__global__ __launch_bounds__(256) void build_apply_kernel(BuildArgs a, Found f, int groups, int parts) {
    __shared__ int32_t s_n[64], s_take[64], s_first[65];
    __shared__ Sums s_front[4], s_all[4];
    const int g = blockIdx.x / parts, part = blockIdx.x - g * parts, lane = threadIdx.x & 63, wave = att_wave();
    const int b = g * 64 + lane;
    const bool in = b < a.seqs, done = in && a.done && a.done[b] != 0;
    Share s{0, 0, 0, 0, 0, 0};
    if (in) s = share_of(a, b, f.old[b], (uint32_t)f.back[b]);
    Sums front{0, 0, 0, 0}, all{0, 0, 0, 0};
    for (int i = threadIdx.x; i < groups; i += 256) {
        const Sums x = f.group[i];
        if (i < g) front = front + x;
        all = all + x;
    }
    front = sums_to(front);
    all = sums_to(all);
    if (lane == 63) {
        s_front[wave] = front;
        s_all[wave] = all;
    }
    __syncthreads();
    front = all = Sums{0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        front = front + s_front[w];
        all = all + s_all[w];
    }
    const Head h = head_of(a, all, f.state[0], f.state[1]);
    const Sums to = sums_to(Sums{s.take, s.rows, s.back, 0});
    Sums before{__shfl_up(to.take, 1, 64), __shfl_up(to.rows, 1, 64), __shfl_up(to.back, 1, 64), 0};
    if (lane == 0) before = Sums{0, 0, 0, 0};
    before = before + front;
    const int end = h.ok ? (int)(before.rows + s.rows) : 0;
    if (wave == 0) {
        s_n[lane] = s.n;
        s_take[lane] = (int)before.take;
        s_first[lane + 1] = end;
        if (lane == 0) s_first[0] = h.ok ? (int)front.rows : 0;
        if (part == 0 && in) {
            a.len_out[b] = s.n + (h.ok ? (int)s.rows : 0);
            a.first[b + 1] = end;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) put_status(a, all, h);
    __syncthreads();
    if (a.position || a.slot || a.sequence) {
        const int here = min(64, a.seqs - g * 64);
        for (int t = s_first[0] + part * 256 + threadIdx.x; t < s_first[64]; t += parts * 256) {
            const int r = below(s_first, here, t);
            one_row(a, h, t, g * 64 + r, t - s_first[r], s_n[r], s_take[r]);
        }
        for (int64_t t = h.rows + (int64_t)blockIdx.x * 256 + threadIdx.x; t < a.tokens; t += (int64_t)gridDim.x * 256) one_row(a, h, (int)t, -1, 0, 0, 0);
    }
    group_entries(a, h, g * 64, s, done, before, part * 4 + wave, parts * 4);
}

}  // namespace

size_t bwla_build_bytes(int64_t seqs) { return (size_t)bwla_align256((uint64_t)seqs * 8 + (uint64_t)((seqs + 63) / 64 + 2) * 16); }

hipError_t bwla_launch_build(const BuildArgs& a, void* ws, hipStream_t st) {
    if (a.seqs <= BB_FEW && a.tokens <= BB_FEW_ROWS) {
        build_few_kernel<<<1, BB_FEW, 0, st>>>(a);
        return hipGetLastError();
    }
    const int groups = a.seqs > 0 ? (a.seqs + 63) / 64 : 1;
    Sums* group = (Sums*)((char*)ws + 16);
    int32_t* old = (int32_t*)(group + groups);
    const Found f{old, old + a.seqs, group, (int32_t*)ws};
    build_sums_kernel<<<(groups + 3) / 4, 256, 0, st>>>(a, f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // A row a thread, up to two workgroups for each compute unit.  (64 requests of 64 rows, 512 and 2048 rows a workgroup: 6.9, 7.7 and 10.1
    // us.  One workgroup a compute unit at most, and two: 1024 of 100 rows 11.6 and 12.3, 2 x 10^5 rows of uneven requests 15.9 and 13.9.)
    const int64_t rows = a.position || a.slot || a.sequence ? a.tokens / 256 / groups + 1 : 1;
    const int parts = (int)std::min<int64_t>(rows, std::max(1, 512 / groups));
    build_apply_kernel<<<groups * parts, 256, 0, st>>>(a, f, groups, parts);
    return hipGetLastError();
}
