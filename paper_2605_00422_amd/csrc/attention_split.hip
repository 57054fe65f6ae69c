// Attention of few rows over a long cache (decoding): the cache's length is split over workgroups, and a
// second launch joins their parts.
//
// The products' rows are the new tokens times the query heads of one key-value head, 16 to a tile, so that a
// group of heads reads its keys and values once.  A wavefront takes 32 cached tokens a step and keeps them in
// registers from load to use, with no LDS: S^T = K Q^T on 16x16 MFMA has the keys as rows, read as they lie
// (64 bytes of 16 keys an instruction), and leaves lane (row r = lane & 15, g = lane >> 4) the scores of keys 4g
// to 4g + 3, which is the order in which the second product O^T = V^T P^T contracts.  Its operand V^T is
// gathered from rows of V by byte permutes: lane m reads columns 8m to 8m + 7 of its four keys, whole rows of
// 256 bytes side by side, and tile c of the result holds columns 8m + c.
// Softmax: running maximum and sum in fp32 per wavefront, joined over the four wavefronts in LDS and over the
// splits in att_join_kernel, in a fixed order.  Weights enter the second product in the cache's type: bf16 ones rounded (by 2^-9 of
// each at most), as the instruction takes them, and divided by their sum as rounded, rows of few keys as well.
// Bound by the reads of keys and values: one token behind 32768, 64 heads of 8 groups of 128 columns 25 us, 5.3 TB/s, what a large
// read reaches, and 5 us for the join; 64 sequences of 500 to 8192 238 us, 4.8 TB/s, with the sums of weights 302 us (the
// scores, 71 MB, are written here and read again).  Three such sequences of 37 fp32 tokens and 8 heads of 64: 6.5 us, a chain of loads.
#include "attention.h"

namespace {

constexpr int SP_WAVES = 4;
constexpr int SP_STEP = 32;                    // cached tokens of a step of one wavefront
constexpr int SP_MAX_CHUNK = 1024;

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float xor16(float v, bool max_of) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
    return max_of ? fmaxf(a, b) : a + b;
}
__device__ __forceinline__ float xor32(float v, bool max_of) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
    return max_of ? fmaxf(a, b) : a + b;
}

// BF: bf16 (else fp32); DP: columns, 64, 128 or 256; EXACT: d == DP (else columns from d on count as zero)
template <bool BF, int DP, bool EXACT>
__global__ __launch_bounds__(64 * SP_WAVES) void att_split_kernel(AttArgs a, AttSplit sp, float* __restrict__ part,
                                                                 float4* __restrict__ stat, float* __restrict__ scores) {
    constexpr int ES = BF ? 2 : 4;
    constexpr int KS = DP * ES / 64;           // 64-byte steps along a row of K
    constexpr int CW = DP >= 128 ? 8 : DP / 16;  // columns of a lane side by side
    constexpr int U = DP / 16 / CW;
    constexpr int NT = U * CW;                 // column tiles of the result
    constexpr int VB = CW * ES;                // bytes of those columns
    constexpr int VD = VB / 4;                 // ... in dwords
    __shared__ int tab[SP_MAX_CHUNK + 8];
    __shared__ float s_m[SP_WAVES][16], s_l[SP_WAVES][16], s_lr[SP_WAVES][16], s_mm[16], s_ll[16], s_llr[16];
    __shared__ __align__(16) float s_o[SP_WAVES][16][DP + 4];

    const int lane = threadIdx.x & 63, wave = att_wave(), li = lane & 15, g = lane >> 4;
    // units (sequence, key-value head, rows) before splits: workgroups are dealt round-robin to the 8 XCDs, and sequences
    // of different lengths have their last splits in different numbers (8 splits side by side gave one XCD all the
    // first ones: 64 sequences of 500 to 8192 tokens 300 us, 5320 GB/s only where all were of one length)
    const int units = a.seqs * a.hkv * sp.row_tiles;
    const int split = blockIdx.x / units, unit = blockIdx.x - split * units;
    const int bh = unit / sp.row_tiles, rt = unit - bh * sp.row_tiles, b = bh / a.hkv, h = bh - b * a.hkv;
    const AttSeq s = att_seq(a, b);
    const int rows = s.fresh * a.group, row = rt * 16 + li;
    const bool parts = s.n > sp.chunk;         // (a sequence of one part is done here)
    if (rt * 16 >= rows || (!parts && split > 0)) return;
    const int64_t at_part = (int64_t)unit * sp.splits + split;
    const int c0 = split * sp.chunk, c1 = min(c0 + sp.chunk, s.n);
    // where no position and no row count says otherwise, keys in front of the first row's window are not read
    const int i_first = max(s.old + rt * 16 / a.group, 0);
    const int skip_to = (s.pos || a.window == INT32_MAX) ? 0 : i_first - a.window + 1;
    const bool none = c0 >= c1 || (c1 <= skip_to && c0 >= s.prefix);
    if (none && parts) {
        if (threadIdx.x < 16) stat[at_part * 16 + threadIdx.x] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
        if (scores) {                          // (what the sums of weights read of it)
            for (int r = 0; r < 16 && rt * 16 + r < rows; ++r)
                for (int j = c0 + threadIdx.x; j < c1; j += 64 * SP_WAVES)
                    scores[((int64_t)(b * a.hkv + h) * sp.rows + rt * 16 + r) * sp.pitch + j] = -INFINITY;
        }
        return;
    }
    const int e0 = c0 >> a.page_shift;
    const int entries = c1 > c0 ? ((c1 - 1) >> a.page_shift) - e0 + 1 : 0;
    for (int e = threadIdx.x; e < entries; e += 64 * SP_WAVES) {
        const int p = s.table[e0 + e];
        tab[e] = (unsigned)p < (unsigned)a.pages ? p : -1;
    }
    // this lane's row
    const int tok = row / a.group, head = h * a.group + row - tok * a.group;
    const AttRow me = att_row(s, tok, row < rows);
    const float slope = a.slopes && row < rows ? a.slopes[head] * ATT_LOG2E : 0.f;
    v4u qf[KS];
    {
        const char* qp = a.q + (int64_t)(s.row0 + (row < rows ? tok : 0)) * a.q_bytes +
                         (int64_t)(row < rows ? head : 0) * a.d * ES + 16 * g;
#pragma unroll
        for (int t = 0; t < KS; ++t) {
            const bool in = row < rows && (EXACT || 64 * t + 16 * g < a.d * ES);
            qf[t] = in ? *(const v4u*)(qp + 64 * t) : v4u{0, 0, 0, 0};
        }
    }
    __syncthreads();

    v4f o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = v4f{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f, lr = 0.f;    // l: sum of the weights, lr: as the second product takes them
    const char* kh = a.k + (int64_t)h * a.head_bytes;
    const char* vh = a.v + (int64_t)h * a.head_bytes;
    const int slot_mask = (1 << a.page_shift) - 1;

    // The keys of the next step are asked for as soon as this one's scores are there, its values as soon as this one's have
    // been used: a wavefront always has 8 KiB on the way.  Pages hold 8 tokens at least, so a lane's four keys of V lie in
    // one; tokens from c1 on read the last one's row.
    v4u kf[2][KS];
    uint32_t vf[2][4][U][VD];
    int page_v[2];
    auto load_keys = [&](int j0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int j = min(j0 + 16 * t + li, c1 - 1);
            const int p = max(tab[(j >> a.page_shift) - e0], 0);
            const char* src = kh + (int64_t)p * a.page_bytes + (int64_t)(j & slot_mask) * a.slot_bytes + 16 * g;
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                if (EXACT || 64 * u + 16 * g < a.d * ES) kf[t][u] = *(const v4u*)(src + 64 * u);
                else kf[t][u] = v4u{0, 0, 0, 0};
            }
        }
    };
    auto load_values = [&](int j0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int jv = j0 + 16 * t + 4 * g;
            page_v[t] = tab[(min(jv, c1 - 1) >> a.page_shift) - e0];
            const char* src = vh + (int64_t)max(page_v[t], 0) * a.page_bytes;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const char* rowp = src + (int64_t)(min(jv + r, c1 - 1) & slot_mask) * a.slot_bytes + li * VB;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool in = EXACT || u * 16 * VB + li * VB < a.d * ES;
                    if constexpr (VD >= 4) {
#pragma unroll
                        for (int w = 0; w < VD / 4; ++w) {
                            const v4u x = in ? *(const v4u*)(rowp + u * 16 * VB + 16 * w) : v4u{0, 0, 0, 0};
#pragma unroll
                            for (int e = 0; e < 4; ++e) vf[t][r][u][4 * w + e] = x[e];
                        }
                    } else {
                        const v2u x = in ? *(const v2u*)(rowp + u * 16 * VB) : v2u{0, 0};
                        vf[t][r][u][0] = x[0];
                        vf[t][r][u][1] = x[1];
                    }
                }
            }
        }
    };
    constexpr int STRIDE = SP_WAVES * SP_STEP;
    if (c0 + wave * SP_STEP < c1) {
        load_keys(c0 + wave * SP_STEP);
        load_values(c0 + wave * SP_STEP);
    }
    for (int j0 = c0 + wave * SP_STEP; j0 < c1; j0 += STRIDE) {
        float y[2][4];
        bool used[2][4];                       // whether any row sees the key: what an unseen one holds stays out
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            v4f acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                if constexpr (BF) {
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, kf[t][u]),
                                                                  __builtin_bit_cast(v8bf, qf[u]), acc, 0, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[t][u][e]), __uint_as_float(qf[u][e]),
                                                                   acc, 0, 0, 0);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = j0 + 16 * t + 4 * g + r;
                const AttKey key = att_key(a, s, j, page_v[t] >= 0 && j < c1);
                const bool seen = att_sees(me, s.prefix, a.window, j, key.p, key.doc);
                float v = att_score(a, acc[r]);
                if (a.slopes) v -= slope * fabsf((float)(me.p - key.p));
                y[t][r] = seen ? v : -INFINITY;
                used[t][r] = ((__ballot(seen) >> (16 * g)) & 0xffffull) != 0;
                top = fmaxf(top, y[t][r]);
            }
            if (scores && row < rows) {
                const int j = j0 + 16 * t + 4 * g;
                if (j < c1) {
                    float* dst = scores + ((int64_t)(b * a.hkv + h) * sp.rows + row) * sp.pitch + j;
                    *(float4*)dst = make_float4(y[t][0], y[t][1], y[t][2], y[t][3]);
                }
            }
        }
        if (j0 + STRIDE < c1) load_keys(j0 + STRIDE);
        top = xor32(xor16(top, true), true);
        if (__any(top > m)) {
            const float now = fmaxf(m, top);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
            l *= f;
            lr *= f;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t] *= f;
            m = now;
        }
        const float base = m == -INFINITY ? 0.f : m;
        float w[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                w[t][r] = __builtin_amdgcn_exp2f(y[t][r] - base);
                l += w[t][r];
            }
        if constexpr (BF) {
            const v4u pf = {att_pack_bf16(w[0][0], w[0][1]), att_pack_bf16(w[0][2], w[0][3]),
                            att_pack_bf16(w[1][0], w[1][1]), att_pack_bf16(w[1][2], w[1][3])};
#pragma unroll
            for (int e = 0; e < 4; ++e) lr = att_add_bf16(pf[e], lr);
            uint32_t keep[4];                  // halves of the operand that hold a key in use
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    keep[2 * t + r] = (used[t][2 * r] ? 0xffffu : 0u) | (used[t][2 * r + 1] ? 0xffff0000u : 0u);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int c = 0; c < CW; ++c) {
                    const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
                    v4u x;
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            x[2 * t + r] = __builtin_amdgcn_perm(vf[t][2 * r + 1][u][c / 2], vf[t][2 * r][u][c / 2], sel) &
                                           keep[2 * t + r];
                    o[u * CW + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, pf), o[u * CW + c], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int c = 0; c < CW; ++c) {
                            const float x = used[t][r] ? __uint_as_float(vf[t][r][u][c]) : 0.f;
                            o[u * CW + c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, w[t][r], o[u * CW + c], 0, 0, 0);
                        }
        }
        if (j0 + STRIDE < c1) load_values(j0 + STRIDE);
    }
    // ---- the four wavefronts' parts, in their order
    l = xor32(xor16(l, false), false);
    lr = BF ? xor32(xor16(lr, false), false) : l;
    m = att_part_max(m, l);
    if (g == 0) {
        s_m[wave][li] = m;
        s_l[wave][li] = l;
        s_lr[wave][li] = lr;
    }
    __syncthreads();
    float mm = -INFINITY, ll = 0.f, llr = 0.f;
#pragma unroll
    for (int w = 0; w < SP_WAVES; ++w) mm = fmaxf(mm, s_m[w][li]);
#pragma unroll
    for (int w = 0; w < SP_WAVES; ++w)
        if (s_m[w][li] != -INFINITY) {
            const float e = __builtin_amdgcn_exp2f(s_m[w][li] - mm);
            ll += s_l[w][li] * e;
            llr += s_lr[w][li] * e;
        }
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mm);
    // lane (row li, g) holds columns 128 u + 4 CW g + CW r + c
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < CW; c += 4)
                *(float4*)&s_o[wave][li][u * 16 * CW + 4 * CW * g + CW * r + c] =
                    make_float4(o[u * CW + c][r] * f, o[u * CW + c + 1][r] * f, o[u * CW + c + 2][r] * f, o[u * CW + c + 3][r] * f);
    if (wave == 0 && g == 0) {
        if (parts) stat[at_part * 16 + li] = make_float4(att_part_max(mm, ll), ll, llr, 0.f);
        s_mm[li] = mm;
        s_ll[li] = ll;
        s_llr[li] = llr;
    }
    __syncthreads();
    constexpr int PER = 16 * DP / 4 / (64 * SP_WAVES);
#pragma unroll
    for (int it = 0; it < PER; ++it) {
        const int idx = it * 64 * SP_WAVES + threadIdx.x, r = idx / (DP / 4), c = idx % (DP / 4) * 4;
        float4 v = *(const float4*)&s_o[0][r][c];
#pragma unroll
        for (int w = 1; w < SP_WAVES; ++w) {
            const float4 x = *(const float4*)&s_o[w][r][c];
            v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        }
        if (parts) {
            if (rt * 16 + r < rows) *(float4*)(part + (at_part * 16 + r) * DP + c) = v;
        } else if (rt * 16 + r < rows && c < a.d) {
            const int t = (rt * 16 + r) / a.group, hd = h * a.group + rt * 16 + r - t * a.group;
            const int64_t at = (int64_t)(s.row0 + t) * a.hq + hd;
            att_put<BF>(a, at, c, v, att_over(s_ll[r], s_llr[r]));
            if (c == 0) att_put_lse(a, at, s_mm[r], s_ll[r]);
        }
    }
}

// One row's parts added up.  GROUPS groups of threads take every GROUPS-th split, four columns a thread, with two of their
// loads in flight; the splits' factors are computed once, in LDS.
template <bool BF, int DP, int GROUPS>
__global__ __launch_bounds__(GROUPS * DP / 4) void att_join_kernel(AttArgs a, AttSplit sp, const float* __restrict__ part,
                                                                   const float4* __restrict__ stat) {
    constexpr int LANES = DP / 4, THREADS = GROUPS * LANES, WAVES = THREADS / 64;
    constexpr int MOST = 512;                          // splits whose factors fit
    __shared__ float red[3 * WAVES], s_f[MOST];
    __shared__ __align__(16) float s_o[GROUPS][DP];
    const int h = blockIdx.y, b = blockIdx.z, row = blockIdx.x, tid = threadIdx.x;
    const AttSeq s = att_seq(a, b);
    if (row >= s.fresh * a.group) return;
    const int rt = row >> 4, r = row & 15;
    const int64_t unit = ((int64_t)b * a.hkv + h) * sp.row_tiles + rt;
    if (s.n <= sp.chunk) return;                       // (one part: written by its workgroup)
    const int used = (s.n + sp.chunk - 1) / sp.chunk;
    const float4* st = stat + unit * sp.splits * 16 + r;
    float m = -INFINITY;
    for (int i = tid; i < used; i += THREADS) m = fmaxf(m, st[i * 16].x);
    m = bwla_wave_max(m);
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, red[w]);
    const int grp = tid / LANES, c = tid % LANES * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f, lr = 0.f;
    for (int i0 = 0; i0 < used; i0 += MOST) {
        const int up = min(used - i0, MOST);
        __syncthreads();
        for (int i = tid; i < up; i += THREADS) {
            const float4 x = st[(i0 + i) * 16];
            const float f = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - m);
            s_f[i] = f;
            l += x.y * f;
            lr += x.z * f;
        }
        __syncthreads();
        const float* src = part + ((unit * sp.splits + i0) * 16 + r) * DP + c;
#pragma unroll 2
        for (int i = grp; i < up; i += GROUPS) {
            const float f = s_f[i];
            if (f == 0.f) continue;                    // (nothing was written where nothing is seen)
            const float4 p = *(const float4*)(src + (int64_t)i * 16 * DP);
            v.x += p.x * f; v.y += p.y * f; v.z += p.z * f; v.w += p.w * f;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        l += __shfl_xor(l, o, 64);
        lr += __shfl_xor(lr, o, 64);
    }
    if ((tid & 63) == 0) {
        red[WAVES + (tid >> 6)] = l;
        red[2 * WAVES + (tid >> 6)] = lr;
    }
    *(float4*)&s_o[grp][c] = v;
    __syncthreads();
    if (grp != 0 || c >= a.d) return;
    l = lr = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        l += red[WAVES + w];
        lr += red[2 * WAVES + w];
    }
    v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        const float4 p = *(const float4*)&s_o[i][c];
        v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
    }
    const int t = row / a.group, hd = h * a.group + row - t * a.group;
    const int64_t at = (int64_t)(s.row0 + t) * a.hq + hd;
    att_put<BF>(a, at, c, v, att_over(l, lr));
    if (c == 0) att_put_lse(a, at, m, l);
}

// The same where rows are many and splits few: DP / 4 threads a row, which take the splits in turn.
template <bool BF, int DP>
__global__ __launch_bounds__(256) void att_join_rows_kernel(AttArgs a, AttSplit sp, const float* __restrict__ part,
                                                            const float4* __restrict__ stat) {
    constexpr int LANES = DP / 4, ROWS = 256 / LANES;
    const int h = blockIdx.y, b = blockIdx.z, row = blockIdx.x * ROWS + threadIdx.x / LANES, c = threadIdx.x % LANES * 4;
    const AttSeq s = att_seq(a, b);
    if (row >= s.fresh * a.group || s.n <= sp.chunk || c >= a.d) return;
    const int used = (s.n + sp.chunk - 1) / sp.chunk;
    const int64_t at = (((int64_t)b * a.hkv + h) * sp.row_tiles + (row >> 4)) * sp.splits * 16 + (row & 15);
    float m = -INFINITY;
#pragma unroll 4
    for (int i = 0; i < used; ++i) m = fmaxf(m, stat[at + i * 16].x);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f, lr = 0.f;
#pragma unroll 4
    for (int i = 0; i < used; ++i) {
        const float4 x = stat[at + i * 16];
        if (x.x == -INFINITY) continue;                // (nothing was written where nothing is seen)
        const float f = __builtin_amdgcn_exp2f(x.x - m);
        const float4 p = *(const float4*)(part + (at + i * 16) * DP + c);
        l += x.y * f;
        lr += x.z * f;
        v.x += p.x * f; v.y += p.y * f; v.z += p.z * f; v.w += p.w * f;
    }
    const int t = row / a.group, hd = h * a.group + row - t * a.group;
    const int64_t to = (int64_t)(s.row0 + t) * a.hq + hd;
    att_put<BF>(a, to, c, v, att_over(l, lr));
    if (c == 0) att_put_lse(a, to, m, l);
}

// The rows' weights of each cached token, from the scores that the first launch left, added to the token's sum.  A thread
// takes four tokens, which lie in one page.
__global__ __launch_bounds__(256) void att_sum_kernel(AttArgs a, AttSplit sp, const float* __restrict__ scores) {
    const int j = (blockIdx.x * 256 + threadIdx.x) * 4, h = blockIdx.y, b = blockIdx.z;
    const AttSeq s = att_seq(a, b);
    if (j >= s.n) return;
    const int p = s.table[j >> a.page_shift];
    if ((unsigned)p >= (unsigned)a.pages) return;
    const float* src = scores + (int64_t)(b * a.hkv + h) * sp.rows * sp.pitch + j;
    const int rows = s.fresh * a.group;
    float4* const w = (float4*)(a.weights + (((int64_t)p * a.hkv + h) << a.page_shift) + (j & ((1 << a.page_shift) - 1)));
    float4 sum = *w;
    float4 add = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* lse = a.lse + (int64_t)s.row0 * a.hq + h * a.group;
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
        const int t = r / a.group;
        const float l = lse[(int64_t)t * a.hq + r - t * a.group] * ATT_LOG2E;
        const float4 y = *(const float4*)(src + (int64_t)r * sp.pitch);
        // (a row that sees nothing has scores of -inf only; behind the sequence's last token lie none)
        add.x += y.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y.x - l);
        add.y += y.y == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y.y - l);
        add.z += y.z == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y.z - l);
        add.w += y.w == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y.w - l);
    }
    sum.x += add.x;
    if (j + 1 < s.n) sum.y += add.y;
    if (j + 2 < s.n) sum.z += add.z;
    if (j + 3 < s.n) sum.w += add.w;
    *w = sum;
}

template <bool BF, int DP>
hipError_t join(const AttArgs& a, const AttSplit& s, void* ws, hipStream_t st) {
    const float* part = (const float*)ws;
    const float4* stat = (const float4*)((const char*)ws + s.part_bytes);
    // Many rows: a few threads each (53280 rows of up to 4 splits 35 -> 16 us, but 4096 rows 7.6 -> 9.0 us).  Few rows of many splits
    // (long caches of few sequences): more threads (128 splits of 64 rows 13.2 -> 7.2 us, but 4 splits of 4096 rows 8.8 -> 16.3 us)
    constexpr int FEW = 4, MANY = DP == 256 ? 8 : 16, ROWS = 1024 / DP;
    const dim3 rows(s.rows, a.hkv, a.seqs);
    if ((int64_t)s.rows * a.hkv * a.seqs >= 8192)
        att_join_rows_kernel<BF, DP><<<dim3((s.rows + ROWS - 1) / ROWS, a.hkv, a.seqs), 256, 0, st>>>(a, s, part, stat);
    else if (s.splits > 16) att_join_kernel<BF, DP, MANY><<<rows, MANY * DP / 4, 0, st>>>(a, s, part, stat);
    else att_join_kernel<BF, DP, FEW><<<rows, FEW * DP / 4, 0, st>>>(a, s, part, stat);
    return hipGetLastError();
}

template <bool BF, int DP>
hipError_t launch(const AttArgs& a, const AttSplit& s, void* ws, hipStream_t st) {
    float* part = (float*)ws;
    float4* stat = (float4*)((char*)ws + s.part_bytes);
    float* scores = a.weights ? (float*)((char*)ws + s.part_bytes + s.stat_bytes) : nullptr;
    const int64_t groups = (int64_t)s.splits * a.seqs * a.hkv * s.row_tiles;
    if (groups >= 1 << 24) return hipErrorInvalidConfiguration;        // (a grid has fewer than 2^32 threads)
    const dim3 grid((unsigned)groups);
    if (a.d == DP) att_split_kernel<BF, DP, true><<<grid, 64 * SP_WAVES, 0, st>>>(a, s, part, stat, scores);
    else att_split_kernel<BF, DP, false><<<grid, 64 * SP_WAVES, 0, st>>>(a, s, part, stat, scores);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && s.splits > 1) e = join<BF, DP>(a, s, ws, st);
    if (e != hipSuccess || !scores || a.max_len == 0) return e;            // (what is not there is not added to the sums)
    att_sum_kernel<<<dim3((a.max_len + 1023) / 1024, a.hkv, a.seqs), 256, 0, st>>>(a, s, scores);
    return hipGetLastError();
}

}  // namespace

// Up to 64 rows of a sequence and key-value head are split over the cache's length here, more go to the tiles.  Up to 16 rows read
// each key once.  17 to 64 rows read it for each 16, which the tiles do not, but these start later; 64 heads of 8, "/": here, tiles:
// one sequence of 1024, 4 and 8 new tokens 12.9 / 15.5 and 13.2 / 16.3 us; behind 8192 21.5 / 17.9 and 31 / 20, behind 32768 49 / 32 and 87 /
// 36; 16 sequences of 8192 161 / 102 and 310 / 107.  Of the tiles' time that is, over 1 to 32 sequences of 64 to 16384 tokens, 0.7 to 3.0
// in bf16, less than 1 where few sequences have up to 1024; 0.35 to 1 in fp32, but up to 1.3 behind 4096 and more, and up to 2.8 where 32
// sequences bring 64 rows to each of 32 heads.  (128 rows, one sequence: 14.7 / 18.4, 49 / 24 and 159 / 45 us.)
bool bwla_att_is_split(const AttArgs& a) { return (int64_t)a.max_new * a.group <= 64; }

AttSplit bwla_att_split(const AttArgs& a, bool weights) {
    AttSplit s;
    s.rows = a.max_new * a.group;
    s.row_tiles = (s.rows + 15) / 16;
    const int64_t units = (int64_t)a.seqs * a.hkv * s.row_tiles;
    const int64_t step = SP_WAVES * SP_STEP;
    int64_t chunk = (units * a.max_len + 511) / 512;
    chunk = (chunk + step - 1) / step * step;
    s.chunk = (int)(chunk < 2 * step ? 2 * step : chunk > SP_MAX_CHUNK ? SP_MAX_CHUNK : chunk);
    s.splits = a.max_len > 0 ? (a.max_len + s.chunk - 1) / s.chunk : 1;
    s.pitch = (a.max_len + 31) & ~31;
    const int dp = a.d <= 64 ? 64 : a.d <= 128 ? 128 : 256;
    s.part_bytes = s.splits > 1 ? (size_t)units * s.splits * 16 * dp * 4 : 0;
    s.stat_bytes = s.splits > 1 ? (size_t)bwla_align256((uint64_t)units * s.splits * 16 * 16) : 0;
    s.score_bytes = weights ? (size_t)a.seqs * a.hkv * s.rows * s.pitch * 4 : 0;
    return s;
}

hipError_t bwla_launch_attention_split(const AttArgs& a, const AttSplit& s, int dtype, void* ws, hipStream_t st) {
    if (dtype == BWLA_X_BF16) {
        if (a.d <= 64) return launch<true, 64>(a, s, ws, st);
        if (a.d <= 128) return launch<true, 128>(a, s, ws, st);
        return launch<true, 256>(a, s, ws, st);
    }
    if (a.d <= 64) return launch<false, 64>(a, s, ws, st);
    if (a.d <= 128) return launch<false, 128>(a, s, ws, st);
    return launch<false, 256>(a, s, ws, st);
}

hipError_t bwla_launch_attention_join(const AttArgs& a, const AttSplit& s, int dtype, void* ws, hipStream_t st) {
    if (dtype == BWLA_X_BF16) {
        if (a.d <= 64) return join<true, 64>(a, s, ws, st);
        if (a.d <= 128) return join<true, 128>(a, s, ws, st);
        return join<true, 256>(a, s, ws, st);
    }
    if (a.d <= 64) return join<false, 64>(a, s, ws, st);
    if (a.d <= 128) return join<false, 128>(a, s, ws, st);
    return join<false, 256>(a, s, ws, st);
}
