// Attention of few rows over a long cache of 8-bit codes (decoding): the cache's length is split over workgroups, as for the other
// types, and the same second launch joins their parts.
//
//   y = c1 (q . code) ks(page),  w = 2^(y - m),  o = S sum_j [w vs(page) / S] code_j,  S the largest vs seen so far
//
// Codes are numbers of fp16 exactly, so the products run on its 16x16 MFMA with codes as they are: a scale multiplies four scores (a
// lane's four keys lie in one page) or four weights, never a code.  Queries: each row times the power of two that brings its largest
// element to [2^14, 2^15), in one term for bf16 (which fp16 holds exactly down to 2^-24 of that) and two for fp32.  Weights times
// vs / S <= 1 times 2^15, in one term (11 bits, against the output's 8) or two: what is smaller than 2^-39 of the largest is lost.
// The rest is as in the split kernel of the other types: S^T = K Q^T has keys as rows and leaves each lane the scores of the keys that
// its operand of O^T = V^T P^T needs; a lane gathers that operand from rows of codes by byte permutes, two columns at a time.
// Codes of unseen keys are finite or cleared (e4m3 has NaN), their pages' scales count as 0.
//
// Bound by memory, and for short caches by the chain from length and table to keys, softmax and values (6.4 us).  64 sequences of 500 to 8192
// tokens, 64 heads of 8 groups of 128 columns, e4m3, capped: 124 us, 4.6 TB/s, and 7 for the join; the same in bf16 233 in all.  One token
// behind 32768: 16.5 us and 5.4 for the join; parts of 512 tokens, as in the other types, where 384, 768 and 1024 take 1.7 to 2.9 more.
// The next step's keys are asked for behind this one's scores and its values behind this one's products, and a step that every row sees
// in full tests nothing: 156 -> 124 us.
#pragma once
#include "code8.h"

namespace {

constexpr int SP_WAVES = 4;
constexpr int SP_STEP = 32;                    // cached tokens of a step of one wavefront
constexpr int SP_MAX_CHUNK = 1024;
constexpr int SP_PAGES = SP_MAX_CHUNK / 8 + 8;

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

// BF: bf16 queries and outputs (else fp32); I8: integers (else e4m3); DP: columns, 64, 128 or 256; EXACT: d == DP;
// FORM: ATT_PLAIN, nothing but the scale, or ATT_LONG, a cap or a bias
template <bool BF, bool I8, int DP, bool EXACT, int FORM>
__global__ __launch_bounds__(64 * SP_WAVES, (DP == 256 ? 1 : 2)) void att8_split_kernel(AttArgs a, Att8 sc, AttSplit sp, float* __restrict__ part,
                                                                  float4* __restrict__ stat) {
    constexpr int ES = BF ? 2 : 4, T = BF ? 1 : 2;
    constexpr int KS = DP / 64;                // 64-byte steps along a row of K
    constexpr int CW = DP >= 128 ? 8 : DP / 16;  // columns of a lane side by side
    constexpr int U = DP / 16 / CW;
    constexpr int NT = U * CW;                 // column tiles of the result
    constexpr int VD = CW / 4;                 // words of those columns
    __shared__ int tab[SP_PAGES];
    __shared__ float s_ks[SP_PAGES], s_vs[SP_PAGES];
    __shared__ float s_m[SP_WAVES][16], s_l[SP_WAVES][16], s_mm[16], s_ll[16];
    __shared__ __align__(16) float s_o[SP_WAVES][16][DP + 4];

    const int lane = threadIdx.x & 63, wave = att_wave(), li = lane & 15, g = lane >> 4;
    const int units = a.seqs * a.hkv * sp.row_tiles;   // (units before splits: as in the other types' kernel)
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
        return;
    }
    const int e0 = c0 >> a.page_shift;
    const int entries = c1 > c0 ? ((c1 - 1) >> a.page_shift) - e0 + 1 : 0;
    for (int e = threadIdx.x; e < entries; e += 64 * SP_WAVES) {
        const int p = s.table[e0 + e];
        const bool there = (unsigned)p < (unsigned)a.pages;
        const int64_t at = (there ? p : 0) * sc.stride + h;
        tab[e] = there ? p : -1;
        s_ks[e] = sc.k_scale[at];
        s_vs[e] = sc.v_scale[at];
    }
    // this lane's row
    const int tok = row / a.group, head = h * a.group + row - tok * a.group;
    const AttRow me = att_row(s, tok, row < rows);
    [[maybe_unused]] const float slope = FORM != ATT_PLAIN && a.slopes && row < rows ? a.slopes[head] * ATT_LOG2E : 0.f;
    Terms<T> qf[KS][2];
    int q_exponent;                            // ... of the power of two that was taken out of the row
    {
        const char* qp = a.q + (int64_t)(s.row0 + (row < rows ? tok : 0)) * a.q_bytes + (int64_t)(row < rows ? head : 0) * a.d * ES;
        float x[KS][16], most = 0.f;
#pragma unroll
        for (int u = 0; u < KS; ++u) {
            const bool in = row < rows && (EXACT || 64 * u + 16 * g < a.d);
            const char* at = qp + (64 * u + 16 * g) * ES;
#pragma unroll
            for (int i = 0; i < ES; ++i) {
                const v4u w = in ? *(const v4u*)(at + 16 * i) : v4u{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (BF) {
                        x[u][8 * i + 2 * e] = __uint_as_float(w[e] << 16);
                        x[u][8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                    } else {
                        x[u][4 * i + e] = __uint_as_float(w[e]);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float v = fabsf(x[u][e]);
                most = fmaxf(most, v <= 3.402823466e38f ? v : 0.f);    // (what is not finite makes its row's scores so)
            }
        }
        most = xor32(xor16(most, true), true);
        const int up = max((int)((__float_as_uint(most) >> 23) & 255) - 127, -100);
#pragma unroll
        for (int u = 0; u < KS; ++u) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[u][e] = ldexpf(x[u][e], 14 - up);
            qf[u][0] = terms_of<T>(x[u]);
            qf[u][1] = terms_of<T>(x[u] + 8);
        }
        q_exponent = up - 14;
    }
    __syncthreads();

    v4f o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = v4f{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    float S = 0.f, down = 0.f;                 // the largest scale of values so far, and 2^15 / S
    const char* kh = a.k + (int64_t)h * a.head_bytes;
    const char* vh = a.v + (int64_t)h * a.head_bytes;
    const int slot_mask = (1 << a.page_shift) - 1;

    // The keys of the next step are asked for as soon as this one's scores are there, its values as soon as this one's have been
    // used.  Pages hold 8 tokens at least, so a lane's four keys of V lie in one; tokens from c1 on read the last one's row.
    v4u kf[2][KS];
    uint32_t vf[2][4][U][VD];
    int page_v[2];
    float ks_v[2], vs_v[2];
    auto load_keys = [&](int j0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int j = min(j0 + 16 * t + li, c1 - 1);
            const int p = max(tab[(j >> a.page_shift) - e0], 0);
            const char* src = kh + (int64_t)p * a.page_bytes + (int64_t)(j & slot_mask) * a.slot_bytes + 16 * g;
#pragma unroll
            for (int u = 0; u < KS; ++u) {
                if (EXACT || 64 * u + 16 * g < a.d) kf[t][u] = *(const v4u*)(src + 64 * u);
                else kf[t][u] = v4u{0, 0, 0, 0};
            }
        }
    };
    auto load_values = [&](int j0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int jv = j0 + 16 * t + 4 * g, e = (min(jv, c1 - 1) >> a.page_shift) - e0;
            page_v[t] = tab[e];
            ks_v[t] = s_ks[e];
            vs_v[t] = s_vs[e];
            const char* src = vh + (int64_t)max(page_v[t], 0) * a.page_bytes;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const char* rowp = src + (int64_t)(min(jv + r, c1 - 1) & slot_mask) * a.slot_bytes + li * CW;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool in = EXACT || u * 16 * CW + li * CW < a.d;
                    if constexpr (VD == 2) {
                        const v2u x = in ? *(const v2u*)(rowp + u * 16 * CW) : v2u{0, 0};
                        vf[t][r][u][0] = x[0];
                        vf[t][r][u][1] = x[1];
                    } else {
                        vf[t][r][u][0] = in ? *(const uint32_t*)(rowp + u * 16 * CW) : 0u;
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
    // keys in front of this index are seen by every row, where nothing but the index counts
    const int seen_to = s.doc || s.pos || a.window != INT32_MAX ? 0 : min(c1, max(s.old + rt * 16 / a.group, -1) + 1);
    for (int j0 = c0 + wave * SP_STEP; j0 < c1; j0 += STRIDE) {
        // Every row sees every key of the step, as when one token follows a cache without windows and documents: nothing is tested then.  (One
        // body for both: two of them took 189 registers instead of 128.)
        const bool whole = j0 + SP_STEP <= seen_to && att_uniform(__all((page_v[0] >= 0) & (page_v[1] >= 0)));
        float y[8];
        uint32_t used[2] = {15u, 15u};         // of a lane's four keys those that any row sees
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            v4f acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < KS; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const Halves x0 = code_halves<I8>(kf[t][u][2 * i]), x1 = code_halves<I8>(kf[t][u][2 * i + 1]);
                    const v4u x{x0.lo, x0.hi, x1.lo, x1.hi};
#pragma unroll
                    for (int n = 0; n < T; ++n)
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x), qf[u][i].t[n], acc, 0, 0, 0);
                }
            const float kq = ldexpf(ks_v[t], q_exponent) * (FORM != ATT_PLAIN && a.capped != 0.f ? 1.f : a.c1);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[4 * t + r] = acc[r] * kq;
        }
        if constexpr (FORM != ATT_PLAIN) {
            if (a.capped != 0.f) capped_scores<8>(a, y);
        }
        if (__builtin_expect(whole, 1)) {
            if constexpr (FORM != ATT_PLAIN) {
                if (a.slopes) {
                    const float away = (float)(me.p - j0 - 4 * g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] -= slope * fabsf(away - (float)(16 * (i / 4) + i % 4));
                }
            }
        } else {
            const int last = c1 - 1;
            used[0] = used[1] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = j0 + 16 * (i / 4) + 4 * g + i % 4, in = min(j, last);
                const int kp = s.pos ? max(s.pos[in], 0) : j;
                const int kd = page_v[i / 4] >= 0 && j <= last ? (s.doc ? max(s.doc[in], -1) : 0) : -1;
                const bool seen = att_sees(me, s.prefix, a.window, j, kp, kd);
                if constexpr (FORM != ATT_PLAIN) {
                    if (a.slopes) y[i] -= slope * fabsf((float)(me.p - kp));
                }
                y[i] = seen ? y[i] : -INFINITY;
                used[i / 4] |= ((__ballot(seen) >> (16 * g)) & 0xffffull) != 0 ? 1u << (i % 4) : 0u;
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, y[i]);
        float now_s = fmaxf(used[0] ? vs_v[0] : 0.f, used[1] ? vs_v[1] : 0.f);
        // as the values' scales stand for this step: nothing of what no row sees
        float over[2] = {used[0] ? vs_v[0] : 0.f, used[1] ? vs_v[1] : 0.f};
        if (j0 + STRIDE < c1) load_keys(j0 + STRIDE);
        if (att_uniform(__any(now_s > S))) {
            now_s = fmaxf(fmaxf(S, xor32(xor16(now_s, true), true)), 0x1p-126f);    // (a reciprocal has to be there)
            const float f = S / now_s;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t] *= f;
            S = now_s;
            down = 1.f / S;
        }
        top = xor32(xor16(top, true), true);
        if (__any(top > m)) {
            const float now = fmaxf(m, top);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
            l *= f;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t] *= f;
            m = now;
        }
        const float base = m == -INFINITY ? 0.f : m;
        float w[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            over[t] = over[t] * down * 32768.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float e = __builtin_amdgcn_exp2f(y[4 * t + r] - base);
                l += e;
                w[4 * t + r] = e * over[t];
            }
        }
        const Terms<T> pf = terms_of<T>(w);
        uint32_t keep[4];                      // bytes of a pair of keys in use
        if constexpr (!I8) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    keep[2 * t + p] = ((used[t] >> (2 * p)) & 1 ? 0x00ff00ffu : 0u) | ((used[t] >> (2 * p)) & 2 ? 0xff00ff00u : 0u);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < CW; c += 2) {
                v4u x0, x1;                    // operands of columns c and c + 1
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        uint32_t two = __builtin_amdgcn_perm(vf[t][2 * p + 1][u][c / 4], vf[t][2 * p][u][c / 4], c & 2 ? 0x07030602u : 0x05010400u);
                        if constexpr (!I8) two &= keep[2 * t + p];
                        const Halves x = code_halves<I8>(two);
                        x0[2 * t + p] = x.lo;
                        x1[2 * t + p] = x.hi;
                    }
#pragma unroll
                for (int n = 0; n < T; ++n) {
                    o[u * CW + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x0), pf.t[n], o[u * CW + c], 0, 0, 0);
                    o[u * CW + c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x1), pf.t[n], o[u * CW + c + 1], 0, 0, 0);
                }
            }
        if (j0 + STRIDE < c1) load_values(j0 + STRIDE);
    }
    // ---- the four wavefronts' parts, in their order
    l = xor32(xor16(l, false), false);
    m = att_part_max(m, l);
    if (g == 0) {
        s_m[wave][li] = m;
        s_l[wave][li] = l;
    }
    __syncthreads();
    float mm = -INFINITY, ll = 0.f;
#pragma unroll
    for (int w = 0; w < SP_WAVES; ++w) mm = fmaxf(mm, s_m[w][li]);
#pragma unroll
    for (int w = 0; w < SP_WAVES; ++w)
        if (s_m[w][li] != -INFINITY) ll += s_l[w][li] * __builtin_amdgcn_exp2f(s_m[w][li] - mm);
    // (one after the other: their product may have few bits)
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mm), back = S * 0x1p-15f;
    // lane (row li, g) holds columns 128 u + 4 CW g + CW r + c
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < CW; c += 4)
                *(float4*)&s_o[wave][li][u * 16 * CW + 4 * CW * g + CW * r + c] =
                    make_float4(o[u * CW + c][r] * f * back, o[u * CW + c + 1][r] * f * back, o[u * CW + c + 2][r] * f * back, o[u * CW + c + 3][r] * f * back);
    if (wave == 0 && g == 0) {
        if (parts) stat[at_part * 16 + li] = make_float4(att_part_max(mm, ll), ll, ll, 0.f);
        s_mm[li] = mm;
        s_ll[li] = ll;
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
            att_put<BF>(a, at, c, v, att_over(s_ll[r], s_ll[r]));
            if (c == 0) att_put_lse(a, at, s_mm[r], s_ll[r]);
        }
    }
}

template <bool BF, int DP>
hipError_t launch8(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st) {
    float* part = (float*)ws;
    float4* stat = (float4*)((char*)ws + s.part_bytes);
    const int64_t groups = (int64_t)s.splits * a.seqs * a.hkv * s.row_tiles;
    if (groups >= 1 << 24) return hipErrorInvalidConfiguration;        // (a grid has fewer than 2^32 threads)
    const dim3 grid((unsigned)groups);
    auto go = [&](auto kernel) {
        kernel<<<grid, 64 * SP_WAVES, 0, st>>>(a, e, s, part, stat);
        return hipGetLastError();
    };
    auto columns = [&](auto i8, auto form) {
        constexpr bool I8 = decltype(i8)::value;
        constexpr int FORM = decltype(form)::value;
        return a.d == DP ? go(att8_split_kernel<BF, I8, DP, true, FORM>) : go(att8_split_kernel<BF, I8, DP, false, FORM>);
    };
    auto codes = [&](auto form) { return e.code == BWLA_CODE_I8 ? columns(std::true_type{}, form) : columns(std::false_type{}, form); };
    const hipError_t r = att_form(a, BF) == ATT_PLAIN ? codes(std::integral_constant<int, ATT_PLAIN>{}) : codes(std::integral_constant<int, ATT_LONG>{});
    if (r != hipSuccess || s.splits == 1) return r;
    return bwla_launch_attention_join(a, s, BF ? BWLA_X_BF16 : BWLA_X_F32, ws, st);
}
template <bool BF>
hipError_t launch8_columns(const AttArgs& a, const Att8& e, const AttSplit& s, void* ws, hipStream_t st) {
    if (a.d <= 64) return launch8<BF, 64>(a, e, s, ws, st);
    if (a.d <= 128) return launch8<BF, 128>(a, e, s, ws, st);
    return launch8<BF, 256>(a, e, s, ws, st);
}

}  // namespace
