// A step's tables from its requests' lengths: pages given back to and taken from a ring of free ones, row offsets, positions and slots.
//
// With n_b cached tokens (0 for a request that starts), m_b new ones and pages of p:  take_b = ceil((n_b + m_b) / p) - ceil(n_b / p).
// Sums over the requests in front (of take_b, of the pages that done requests name, of m_b) say where in the ring and in the rows
// each request's share lies, so that everything else is independent: no atomics, and the same answer for the same arguments.
// Integer work of a few bytes an entry, bound by launches and chains of loads.  Three kernels: pages that are given back counted (a
// wavefront a request; not without d_done), the sums (one workgroup), then entries (a wavefront a request) and rows (a thread each,
// whose request is found by bisection of the offsets in LDS).  Few requests and rows: all of it by one workgroup, in one launch.
#include "attention.h"

namespace {

constexpr int BB_THREADS = 1024;
constexpr int BB_WAVES = BB_THREADS / 64;
constexpr int BB_FEW = 1024;             // requests that one workgroup takes in a launch of its own
constexpr int BB_FEW_ROWS = 8192;
constexpr int BB_STEPS = 2048;           // row offsets that a workgroup of rows keeps

// what the sums leave for each request: its cached tokens before the call, the first of its pages among those taken, and among those
// given back
struct Plan {
    int32_t *old, *take, *back;
};
struct Head {
    int32_t ok, front, count, rows;      // rows: given out in all
};

__device__ __forceinline__ int cut(int v, int most) { return min(max(v, 0), most); }
__device__ __forceinline__ int up(int n, int shift) { return (int)(((int64_t)n + (1 << shift) - 1) >> shift); }

// pages that request b gives back
__device__ int given_back(const BuildArgs& a, int b) {
    if (!a.done || a.done[b] == 0) return 0;
    const int lane = threadIdx.x & 63, held = up(cut(a.len[b], a.max_len), a.page_shift);
    const int32_t* row = a.table + (int64_t)b * a.table_stride;
    int sum = 0;
    for (int e = 0; e < held; e += 64) sum += __popcll(__ballot(e + lane < held && (uint32_t)row[min(e + lane, held - 1)] < (uint32_t)a.pages));
    return sum;
}

struct Share {
    int64_t take, rows;
    int32_t back, beyond;                // beyond: whether the request would be too long
};
__device__ __forceinline__ Share share_of(const BuildArgs& a, int b, const int32_t* back) {
    const int n = a.done && a.done[b] != 0 ? 0 : cut(a.len[b], a.max_len);
    const int64_t m = max(a.fresh[b], 0);
    Share s;
    s.rows = m;
    s.take = ((n + m + (1 << a.page_shift) - 1) >> a.page_shift) - up(n, a.page_shift);
    s.back = back[b];
    s.beyond = n + m > a.max_len;
    return s;
}
__device__ __forceinline__ int64_t shfl_up(int64_t v, int o) {
    const int lo = __shfl_up((int)v, o, 64), hi = __shfl_up((int)(v >> 32), o, 64);
    return ((int64_t)hi << 32) | (uint32_t)lo;
}
// sums over the workgroup's threads in front of each, and over all
__device__ __forceinline__ void scan(int64_t v, int64_t* words, int64_t& before, int64_t& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = shfl_up(x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) words[wave] = x;
    __syncthreads();
    int64_t front = 0;
    all = 0;
    for (int w = 0; w < BB_WAVES; ++w) {
        if (w < wave) front += words[w];
        all += words[w];
    }
    before = front + x - v;
}

// The sums, by one workgroup of BB_THREADS.  back: what given_back said; first: written as a.first is.
__device__ void plan_all(const BuildArgs& a, const Plan& p, const int32_t* back, int32_t* first, Head* head, int64_t* words) {
    int64_t take = 0, rows = 0, freed = 0, beyond = 0;
    for (int b = threadIdx.x; b < a.seqs; b += BB_THREADS) {
        const Share s = share_of(a, b, back);
        take += s.take;
        rows += s.rows;
        freed += s.back;
        beyond += s.beyond;
    }
    int64_t none, t_take, t_rows, t_back, t_beyond;
    scan(take, words, none, t_take);
    scan(rows, words, none, t_rows);
    scan(freed, words, none, t_back);
    scan(beyond, words, none, t_beyond);
    // (a state that is none: what the ring can hold)
    const int front = (int)((uint32_t)a.state[0] % (uint32_t)a.capacity), count = cut(a.state[1], a.capacity);
    const int64_t missing = max(t_take - count, (int64_t)0), lost = max(t_rows - a.tokens, (int64_t)0);
    const bool ok = missing == 0 && lost == 0 && t_beyond == 0;
    __syncthreads();                     // (everyone has read the state)
    if (threadIdx.x == 0) {
        const auto word = [](int64_t v) { return (int32_t)min(v, (int64_t)INT32_MAX); };
        a.status[0] = word(missing);
        a.status[1] = word(t_beyond);
        a.status[2] = word(lost);
        a.status[3] = word(t_rows);
        const int taken = ok ? (int)t_take : 0;
        a.state_out[0] = (int)(((int64_t)front + taken) % a.capacity);
        a.state_out[1] = count - taken + (int)min(t_back, (int64_t)a.capacity - count);
        *head = Head{ok, front, count, ok ? (int)t_rows : 0};
        first[0] = 0;
        if (first != a.first) a.first[0] = 0;
    }
    int64_t c_take = 0, c_rows = 0, c_back = 0;
    for (int b0 = 0; b0 < a.seqs; b0 += BB_THREADS) {
        const int b = b0 + threadIdx.x;
        const bool in = b < a.seqs;
        Share s{0, 0, 0, 0};
        if (in) s = share_of(a, b, back);
        int64_t x_take, x_rows, x_back, n_take, n_rows, n_back;
        scan(s.take, words, x_take, n_take);
        scan(s.rows, words, x_rows, n_rows);
        scan(s.back, words, x_back, n_back);
        if (in) {
            const int old = cut(a.len[b], a.max_len), n = a.done && a.done[b] != 0 ? 0 : old;
            const int end = ok ? (int)(c_rows + x_rows + s.rows) : 0;
            p.old[b] = old;
            p.take[b] = ok ? (int)(c_take + x_take) : 0;
            p.back[b] = (int)min(c_back + x_back, (int64_t)INT32_MAX);
            a.len_out[b] = n + (ok ? (int)s.rows : 0);
            first[b + 1] = end;
            if (first != a.first) a.first[b + 1] = end;
        }
        c_take += n_take;
        c_rows += n_rows;
        c_back += n_back;
    }
}

// a request's entries of the table and the ring, by a wavefront
__device__ void entries(const BuildArgs& a, const Plan& p, const Head& h, int b) {
    const int lane = threadIdx.x & 63, old = p.old[b];
    const bool done = a.done && a.done[b] != 0;
    int32_t* row = a.table + (int64_t)b * a.table_stride;
    if (done) {
        const int held = up(old, a.page_shift);
        int at = p.back[b];
        for (int e = 0; e < held; e += 64) {
            const int page = e + lane < held ? row[e + lane] : -1;
            const uint64_t there = __ballot((uint32_t)page < (uint32_t)a.pages);
            const int k = at + __popcll(there & ((1ull << lane) - 1));
            // (a pool that has more pages given back than it holds keeps the first)
            if ((uint32_t)page < (uint32_t)a.pages && k < a.capacity - h.count)
                a.ring[(int)(((int64_t)h.front + h.count + k) % a.capacity)] = page;
            at += __popcll(there);
        }
    }
    if (!h.ok) return;
    const int n = done ? 0 : old, base = up(n, a.page_shift), want = up(n + max(a.fresh[b], 0), a.page_shift);
    for (int e = base + lane; e < want; e += 64) row[e] = a.ring[(int)(((int64_t)h.front + p.take[b] + e - base) % a.capacity)];
}

// row t of request b, its new token i
__device__ __forceinline__ void one_row(const BuildArgs& a, const Plan& p, const Head& h, int t, int b, int i) {
    const bool live = b >= 0;
    int64_t slot = -1;
    int at = -1;
    if (live) {
        const int n = a.done && a.done[b] != 0 ? 0 : p.old[b], base = up(n, a.page_shift), j = n + i, e = j >> a.page_shift;
        at = j + (a.shift ? a.shift[b] : 0);
        if (a.slot) {
            const int page = e >= base ? a.ring[(int)(((int64_t)h.front + p.take[b] + e - base) % a.capacity)]
                                       : a.table[(int64_t)b * a.table_stride + e];
            if ((uint32_t)page < (uint32_t)a.pages) slot = ((int64_t)page << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        }
    }
    if (a.position) a.position[t] = at;
    if (a.slot) a.slot[t] = slot;
    if (a.sequence) a.sequence[t] = b;
}
// the last b with first[b * step] <= t, of b <= most
__device__ __forceinline__ int below(const int32_t* first, int step, int most, int t) {
    int lo = 0, hi = most + 1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid * step] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(BB_THREADS) void build_few_kernel(BuildArgs a) {
    __shared__ int32_t s_old[BB_FEW], s_take[BB_FEW], s_back[BB_FEW], s_first[BB_FEW + 1];
    __shared__ int64_t words[BB_WAVES];
    __shared__ Head s_head;
    const Plan p{s_old, s_take, s_back};
    const int wave = att_wave();
    if (a.done) {
        for (int b = wave; b < a.seqs; b += BB_WAVES) {
            const int k = given_back(a, b);
            if ((threadIdx.x & 63) == 0) s_old[b] = k;
        }
    } else {
        for (int b = threadIdx.x; b < a.seqs; b += BB_THREADS) s_old[b] = 0;
    }
    __syncthreads();
    // (each thread reads what was given back of its own requests before it writes their lengths there)
    plan_all(a, p, s_old, s_first, &s_head, words);
    __syncthreads();
    const Head h = s_head;
    // rows first: a page in front of the new ones is read from the table, where no entry of theirs is written
    const int total = h.rows;
    if (a.position || a.slot || a.sequence)
        for (int t = threadIdx.x; t < a.tokens; t += BB_THREADS) {
            const int b = t < total ? below(s_first, 1, a.seqs, t) : -1;
            one_row(a, p, h, t, b, b < 0 ? 0 : t - s_first[b]);
        }
    for (int b = wave; b < a.seqs; b += BB_WAVES) entries(a, p, h, b);
}

__global__ __launch_bounds__(256) void build_count_kernel(BuildArgs a, int32_t* back) {
    const int b = blockIdx.x * 4 + att_wave();
    if (b >= a.seqs) return;
    const int k = given_back(a, b);
    if ((threadIdx.x & 63) == 0) back[b] = k;
}
__global__ __launch_bounds__(BB_THREADS) void build_plan_kernel(BuildArgs a, Plan p, Head* head, bool counted) {
    __shared__ int64_t words[BB_WAVES];
    if (!counted) {
        for (int b = threadIdx.x; b < a.seqs; b += BB_THREADS) p.old[b] = 0;
        __syncthreads();
    }
    plan_all(a, p, p.old, a.first, head, words);
}
__global__ __launch_bounds__(256) void build_apply_kernel(BuildArgs a, Plan p, const Head* head, int row_blocks) {
    __shared__ int32_t s_first[BB_STEPS];
    const Head h = *head;
    if ((int)blockIdx.x >= row_blocks) {
        const int b = (blockIdx.x - row_blocks) * 4 + att_wave();
        if (b < a.seqs) entries(a, p, h, b);
        return;
    }
    const int t0 = blockIdx.x * 1024;
    const int step = (a.seqs + 1 + BB_STEPS - 1) / BB_STEPS, held = a.seqs / step;     // offsets 0, step, .. held * step
    if (t0 < h.rows) {
        for (int i = threadIdx.x; i <= held; i += 256) s_first[i] = a.first[i * step];
        __syncthreads();
    }
    for (int t = t0 + threadIdx.x; t < min(t0 + 1024, (int)a.tokens); t += 256) {
        int b = -1, i = 0;
        if (t < h.rows) {
            const int lo = below(s_first, 1, held, t) * step;
            b = step == 1 ? lo : lo + below(a.first + lo, 1, min(step - 1, a.seqs - lo), t);
            i = t - a.first[b];
        }
        one_row(a, p, h, t, b, i);
    }
}

}  // namespace

size_t bwla_build_bytes(int64_t seqs) { return (size_t)bwla_align256((uint64_t)seqs * 12 + 16); }

hipError_t bwla_launch_build(const BuildArgs& a, void* ws, hipStream_t st) {
    if (a.seqs <= BB_FEW && a.tokens <= BB_FEW_ROWS) {
        build_few_kernel<<<1, BB_THREADS, 0, st>>>(a);
        return hipGetLastError();
    }
    Head* head = (Head*)ws;
    int32_t* at = (int32_t*)((char*)ws + 16);
    const Plan p{at, at + a.seqs, at + 2 * a.seqs};
    hipError_t e = hipSuccess;
    if (a.done && a.seqs > 0) {
        build_count_kernel<<<(a.seqs + 3) / 4, 256, 0, st>>>(a, p.old);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    build_plan_kernel<<<1, BB_THREADS, 0, st>>>(a, p, head, a.done != nullptr);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int row_blocks = a.position || a.slot || a.sequence ? (int)((a.tokens + 1023) / 1024) : 0;
    if (row_blocks + a.seqs == 0) return hipSuccess;
    build_apply_kernel<<<row_blocks + (a.seqs + 3) / 4, 256, 0, st>>>(a, p, head, row_blocks);
    return hipGetLastError();
}
