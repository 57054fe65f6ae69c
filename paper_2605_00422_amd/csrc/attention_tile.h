// Attention of many rows (prompts, chunks): a workgroup of four wavefronts holds 128 rows of the products -- new
// tokens times the query heads of one key-value head, tokens major, so that a group of heads shares what is read --
// and walks over the cache in blocks of keys.
//
// S^T = K Q^T on 32x32 MFMA: keys are the rows of the result, so that a lane has the scores of one row (lane & 31)
// and the softmax needs one exchange between the wavefront's halves; its queries stay in registers.  Lane half h
// holds keys 8 g + 4 h + 0..3 of the tile, and the second product O^T = V^T P^T contracts in that very order: the
// weights go from accumulators to operand without leaving the lane.  Its operand V^T comes out of LDS by transposing
// reads (bf16), or one value a lane (fp32 MFMA contracts two keys an instruction).
// Keys and values come by asynchronous copies to LDS, one block ahead, 16 bytes a lane, in an order (XOR with the key)
// that keeps the reads off each other's banks.
#pragma once
#include "attention.h"

namespace {

constexpr int AT_WAVES = 4;
constexpr int AT_ROWS = 32 * AT_WAVES;
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <bool BF, int DP>
struct AtShape {
    static constexpr int ES = BF ? 2 : 4;
    static constexpr int BK = BF ? 64 : 32;            // keys of a block
    static constexpr int ROWB = DP * ES;               // bytes of a row in LDS
    static constexpr int CH = ROWB / 16;               // 16-byte pieces of a row
    static constexpr int TILE = BK * ROWB;             // bytes of a block of keys, and of values
    static constexpr int COPIES = BK * CH / (64 * AT_WAVES);
    static constexpr int LDS = 4 * TILE + 2 * (2 * BK + 4) * 4;
};

// BF: bf16 (else fp32); DP: columns, 64, 128 or 256; EXACT: d == DP; GENERAL: a cap or a bias
template <bool BF, int DP, bool EXACT, bool GENERAL>
__global__ __launch_bounds__(64 * AT_WAVES, DP == 256 ? 1 : 2) void att_tile_kernel(AttArgs a, int tiles, int units) {
    using S = AtShape<BF, DP>;
    constexpr int ES = S::ES, BK = S::BK, ROWB = S::ROWB, CH = S::CH, KT = BK / 32, DT = DP / 32;
    extern __shared__ __align__(16) char smem[];
    char* const ks = smem;                             // [2][BK][ROWB]
    char* const vs = smem + 2 * S::TILE;
    int* const info = (int*)(smem + 4 * S::TILE);      // [2][BK positions, BK documents, flag]
    constexpr int INFO = 2 * BK + 4;

    // workgroups are dealt round-robin to the 8 XCDs: each takes whole (sequence, key-value head) units, whose
    // keys and values then stay in its own L2, the longest rows first
    int unit, tile;
    if (units % 8 == 0 || units >= 32) {
        const int x = blockIdx.x & 7, k = blockIdx.x >> 3;
        unit = k / tiles * 8 + x;
        tile = tiles - 1 - k % tiles;
    } else {
        unit = blockIdx.x % units;
        tile = tiles - 1 - blockIdx.x / units;
    }
    if (unit >= units || tile < 0) return;
    const int b = unit / a.hkv, h = unit - b * a.hkv;
    const AttSeq s = att_seq(a, b);
    const int rows = s.fresh * a.group;
    if (tile * AT_ROWS >= rows) return;

    const int tid = threadIdx.x, lane = tid & 63, wave = att_wave(), l32 = lane & 31, hf = lane >> 5;
    const int row = tile * AT_ROWS + wave * 32 + l32;
    const bool live = row < rows;
    const int tok = live ? row / a.group : 0, head = h * a.group + (live ? row - tok * a.group : 0);
    const AttRow me = att_row(s, tok, live);
    const float slope = GENERAL && a.slopes ? a.slopes[head] * ATT_LOG2E : 0.f;
    // indexes of the first and last row of this wavefront, and of the workgroup
    const int old = s.n - s.fresh;
    const int w_first = old + min(tile * AT_ROWS + wave * 32, rows - 1) / a.group;
    const int w_last = old + min(tile * AT_ROWS + wave * 32 + 31, rows - 1) / a.group;
    const int g_first = max(old + tile * AT_ROWS / a.group, 0);
    const int g_last = old + min(tile * AT_ROWS + AT_ROWS - 1, rows - 1) / a.group;

    // blocks of keys: those of the prefix, then from the first row's window to the last row's index
    const int hi = max((g_last + BK) / BK, 0);
    const int pb = min((max(s.prefix, 0) + BK - 1) / BK, (s.n + BK - 1) / BK);
    int lo = s.pos || a.window == INT32_MAX ? 0 : max(g_first - a.window + 1, 0) / BK;
    if (lo < pb) lo = pb;
    const int blocks = pb + max(hi - lo, 0);

    v4u qf[CH / 2];
    {
        const char* qp = a.q + (int64_t)(s.row0 + tok) * a.q_bytes + (int64_t)head * a.d * ES;
#pragma unroll
        for (int t = 0; t < CH / 2; ++t) {
            const int c = (2 * t + hf) * 16;
            qf[t] = live && (EXACT || c < a.d * ES) ? *(const v4u*)(qp + c) : v4u{0, 0, 0, 0};
        }
    }
    const char* const kh = a.k + (int64_t)h * a.head_bytes;
    const char* const vh = a.v + (int64_t)h * a.head_bytes;
    const int slot_mask = (1 << a.page_shift) - 1;
    auto first_of = [&](int t) { return (t < pb ? t : lo + t - pb) * BK; };

    // ---- copies of a block: thread's piece i is piece (i 4 + wave) 64 + lane of the tile
    constexpr int KSW = (CH < 16 ? CH : 16) - 1;                             // keys: piece ^ (key & KSW)
    constexpr int VSW = BF ? (CH < 16 ? 3 : 7) : 0;                          // values: piece ^ (key & VSW) * 2
    int page[S::COPIES];
    auto key_of = [&](int i) { return ((i * AT_WAVES + wave) * 64 + lane) / CH; };
    auto find_pages = [&](int t) {
#pragma unroll
        for (int i = 0; i < S::COPIES; ++i) {
            const int j = min(first_of(t) + key_of(i), s.n - 1);
            const int p = s.table[j >> a.page_shift];
            page[i] = (unsigned)p < (unsigned)a.pages ? p : 0;               // (read, and not used)
        }
    };
    auto copy_block = [&](int t, int buf) {
#pragma unroll
        for (int i = 0; i < S::COPIES; ++i) {
            const int key = key_of(i), piece = ((i * AT_WAVES + wave) * 64 + lane) % CH;
            const int j = min(first_of(t) + key, s.n - 1);
            const int64_t at = (int64_t)page[i] * a.page_bytes + (int64_t)(j & slot_mask) * a.slot_bytes;
            const int pk = piece ^ (key & KSW), pv = piece ^ (key & VSW) * 2;
            const int dst = buf * S::TILE + (i * AT_WAVES + wave) * 1024;
            if (EXACT || pk * 16 < a.d * ES)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(kh + at + pk * 16),
                                                 (__attribute__((address_space(3))) void*)(ks + dst), 16, 0, 0);
            if (EXACT || pv * 16 < a.d * ES)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(vh + at + pv * 16),
                                                 (__attribute__((address_space(3))) void*)(vs + dst), 16, 0, 0);
        }
    };
    // position and document of the block's keys, by the first BK threads
    // (looked up in front of the copies that are issued after it, and waited for behind the block's products)
    int key_page = 0, key_pos = 0, key_doc = 0;
    auto find_key = [&](int t) {
        if (tid < BK) {
            const int j = first_of(t) + tid, in = min(j, s.n - 1);
            key_page = j < s.n ? s.table[in >> a.page_shift] : -1;
            key_pos = s.pos ? s.pos[in] : j;
            key_doc = s.doc ? s.doc[in] : 0;
        }
    };
    auto put_key = [&](int buf) {
        if (tid < BK) {
            const bool there = (unsigned)key_page < (unsigned)a.pages;
            info[buf * INFO + tid] = max(key_pos, 0);
            info[buf * INFO + BK + tid] = there ? max(key_doc, -1) : -1;
            const bool gone = __any(!there);
            if (tid == 0) info[buf * INFO + 2 * BK] = gone;
        }
    };

    if constexpr (!EXACT) {                            // columns that no copy fills count as zero
        for (int i = tid; i < 2 * BK * CH; i += 64 * AT_WAVES) {
            const int key = i / CH % BK, piece = i % CH;
            if ((piece ^ (key & KSW)) * 16 >= a.d * ES) *(v4u*)(ks + i * 16) = v4u{0, 0, 0, 0};
        }
    }
    v16f o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    float m = -INFINITY, l = 0.f, lr = 0.f;            // l: sum of the weights, lr: as the second product takes them

    if (blocks > 0) {
        find_pages(0);
        find_key(0);
        copy_block(0, 0);
        put_key(0);
        if (blocks > 1) find_pages(1);
    }
    // where lane (i = lane & 15 of each 16) of a transposing read takes its 8 bytes: key 4 hf + (i >> 2), columns
    // 16 (lane >> 4 & 1) + 4 (i & 3) of a column tile
    const int tk = 4 * hf + ((lane & 15) >> 2);
    int vofs[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) {
        if constexpr (BF) {
            const int piece = (4 * t + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (tk & VSW) * 2;
            vofs[t] = tk * ROWB + piece * 16 + (lane & 1) * 8;
        } else {
            vofs[t] = 4 * hf * ROWB + (32 * t + l32) * 4;
        }
    }

    // Weights enter the second product rounded to bf16, whose errors (2^-9 of a weight in the mean) average out over
    // many keys.  Where a row has seen fewer than FEW, both terms of the weights go in (16 bits): the first tokens of
    // a prompt or a document, at no cost to the others.
    constexpr int FEW = 64;
    int had = 0;                                       // keys that the lane's half of the row has seen
    for (int t = 0; t < blocks; ++t) {
        const int buf = t & 1, j0 = first_of(t);
        __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0): this wavefront's copies of the block are there
        bwla_lds_barrier();                            // ... everyone's are, and the other buffer is free
        if (t + 1 < blocks) {
            find_key(t + 1);
            copy_block(t + 1, buf ^ 1);
            if (t + 2 < blocks) find_pages(t + 2);
        }
        const int* const inf = info + buf * INFO;
        const bool skip = j0 > w_last && j0 >= s.prefix;    // (scalars)
        if (!skip) {
            // ---- S^T
            v16f p[KT];
#pragma unroll
            for (int k = 0; k < KT; ++k) {
#pragma unroll
                for (int r = 0; r < 16; ++r) p[k][r] = 0.f;
                const char* src = ks + buf * S::TILE + (k * 32 + l32) * ROWB;
#pragma unroll
                for (int c = 0; c < CH / 2; ++c) {
                    const v4u kf = *(const v4u*)(src + ((2 * c + hf) ^ (l32 & KSW)) * 16);
                    if constexpr (BF) {
                        p[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, kf),
                                                                       __builtin_bit_cast(v8bf, qf[c]), p[k], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            p[k] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(qf[c][e]),
                                                                        p[k], 0, 0, 0);
                    }
                }
            }
            // ---- scores
            float c1 = a.c1;
            if constexpr (GENERAL) {
                c1 = 1.f;
                if (a.capped != 0.f) {
                    const float C = a.capped, c3 = a.c2 * (2.f * ATT_LOG2E);
#pragma unroll
                    for (int k = 0; k < KT; ++k)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            if constexpr (BF) {        // (an error of 1e-7 C: weights are rounded to 8 bits)
                                const float e = __builtin_amdgcn_exp2f(p[k][r] * c3);
                                p[k][r] = fmaf(-2.f * C, __builtin_amdgcn_rcpf(1.f + e), C);
                            } else {
                                p[k][r] = C * att_tanh(p[k][r] * a.c2);
                            }
                        }
                } else {
#pragma unroll
                    for (int k = 0; k < KT; ++k)
#pragma unroll
                        for (int r = 0; r < 16; ++r) p[k][r] *= a.c1;
                }
                if (a.slopes) {
                    if (s.pos) {
#pragma unroll
                        for (int k = 0; k < KT; ++k)
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                p[k][r] -= slope * fabsf((float)(me.p - inf[k * 32 + (r & 3) + 8 * (r >> 2) + 4 * hf]));
                    } else {
                        const float away = (float)(me.p - j0 - 4 * hf);
#pragma unroll
                        for (int k = 0; k < KT; ++k)
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                p[k][r] = fmaf(-slope, fabsf(away - (float)(k * 32 + (r & 3) + 8 * (r >> 2))), p[k][r]);
                    }
                }
            }
            // ---- mask: blocks that every row sees whole have none
            const bool whole = att_uniform(!inf[2 * BK] && !s.doc && w_first >= 0 &&
                                           (j0 + BK <= s.prefix || (j0 + BK - 1 <= w_first &&
                                                                    (a.window == INT32_MAX || (!s.pos && j0 > w_last - a.window)))));
            uint32_t used[KT];                         // bit r: some row of the wavefront sees the lane's key r
            bool fine = false;                         // weights as two bf16 terms: see below
            if (whole) {
                had += BK;
            } else {
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    uint32_t mine = 0;                 // bit r: the row sees the lane's key r
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const v4i kp = *(const v4i*)(inf + k * 32 + 8 * g + 4 * hf), kd = *(const v4i*)(inf + BK + k * 32 + 8 * g + 4 * hf);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool seen = att_sees(me, s.prefix, a.window, j0 + k * 32 + 8 * g + 4 * hf + e, kp[e], kd[e]);
                            p[k][4 * g + e] = seen ? p[k][4 * g + e] : -INFINITY;
                            mine |= seen ? 1u << (4 * g + e) : 0u;
                        }
                    }
                    had += __popc(mine);
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) mine |= __shfl_xor(mine, o, 64);
                    used[k] = mine;
                }
                fine = BF && att_uniform(__any(live & (had < FEW)));
            }
            // ---- running maximum and sum
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, p[k][r]);
            top = half_max(top) * c1;
            // the maximum moves on only when it is off by 2^8, which the fp32 sums and products hold as well
            if (__any(top > m + 8.f)) {
                const float now = fmaxf(m, top);
                const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
                l *= f;
                if constexpr (BF) lr *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[d][r] *= f;
                m = now;
            }
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p[k][r] = __builtin_amdgcn_exp2f(fmaf(p[k][r], c1, -base));
                    l += p[k][r];
                }
            // ---- O^T += V^T P^T; values of keys that no row sees stay out (they may be anything)
            const char* const vb = vs + buf * S::TILE;
            auto products = [&](auto masked) {
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    if constexpr (BF) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            v4u pf, pl;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float w0 = p[k][8 * u + 2 * e], w1 = p[k][8 * u + 2 * e + 1];
                                pf[e] = att_pack_bf16(w0, w1);
                                lr = att_add_bf16(pf[e], lr);
                                if constexpr (decltype(masked)::value) {
                                    if (fine) {
                                        pl[e] = att_pack_bf16(w0 - bwla_bf16_to_f32((uint16_t)pf[e]), w1 - bwla_bf16_to_f32((uint16_t)(pf[e] >> 16)));
                                        lr = att_add_bf16(pl[e], lr);
                                    }
                                }
                            }
#pragma unroll
                            for (int d = 0; d < DT; ++d) {
                                typedef uint32_t v2u __attribute__((ext_vector_type(2)));
                                const char* src = vb + vofs[d] + (k * 32 + 16 * u) * ROWB;
                                const v2u x0 = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                    (__attribute__((address_space(3))) v4s*)src));
                                const v2u x1 = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                    (__attribute__((address_space(3))) v4s*)(src + 8 * ROWB)));
                                v4u x = {x0[0], x0[1], x1[0], x1[1]};
                                if constexpr (decltype(masked)::value) {
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const uint32_t w = used[k] >> (8 * u + 2 * e);
                                        x[e] &= ((w & 1) ? 0xffffu : 0u) | ((w & 2) ? 0xffff0000u : 0u);
                                    }
                                }
                                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, x),
                                                                               __builtin_bit_cast(v8bf, pf), o[d], 0, 0, 0);
                                if constexpr (decltype(masked)::value) {
                                    if (fine) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, x),
                                                                                             __builtin_bit_cast(v8bf, pl), o[d], 0, 0, 0);
                                }
                            }
                        }
                    } else {
#pragma unroll
                        for (int r = 0; r < 16; ++r)
#pragma unroll
                            for (int d = 0; d < DT; ++d) {
                                float x = *(const float*)(vb + vofs[d] + (k * 32 + (r & 3) + 8 * (r >> 2)) * ROWB);
                                if constexpr (decltype(masked)::value) x = (used[k] >> r) & 1 ? x : 0.f;
                                o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p[k][r], o[d], 0, 0, 0);
                            }
                    }
                }
            };
            if (whole) products(std::false_type{});
            else products(std::true_type{});
        }
        if (t + 1 < blocks) put_key(buf ^ 1);
    }

    l = half_sum(l);
    lr = BF ? half_sum(lr) : l;
    if (!live) return;
    const float inv = lr > 0.f ? 1.f / lr : 0.f;
    const int64_t at = ((int64_t)(s.row0 + tok) * a.hq + head);
    char* const dst = a.out + at * a.d * ES;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int c = 32 * d + 2 * r + 4 * hf;
            if (EXACT || c < a.d) {
                if constexpr (BF) *(uint2*)(dst + c * 2) = make_uint2(att_pack_bf16(o[d][r] * inv, o[d][r + 1] * inv),
                                                                      att_pack_bf16(o[d][r + 2] * inv, o[d][r + 3] * inv));
                else *(float4*)(dst + c * 4) = make_float4(o[d][r] * inv, o[d][r + 1] * inv, o[d][r + 2] * inv, o[d][r + 3] * inv);
            }
        }
    if (hf == 0 && a.lse) a.lse[at] = l > 0.f ? (m + __log2f(l)) * ATT_LN2 : -INFINITY;
}

template <bool BF, int DP>
hipError_t at_launch(const AttArgs& a, hipStream_t st) {
    const int tiles = (int)(((int64_t)a.max_new * a.group + AT_ROWS - 1) / AT_ROWS);
    const int units = a.seqs * a.hkv;
    const int64_t grid = (int64_t)tiles * (units % 8 == 0 || units >= 32 ? (units + 7) / 8 * 8 : units);
    constexpr int lds = AtShape<BF, DP>::LDS;
    const bool general = a.capped != 0.f || a.slopes, exact = a.d == DP;
    auto go = [&](auto kernel) {
        const hipError_t e = bwla_ensure_lds((const void*)kernel, lds);
        if (e != hipSuccess) return e;
        kernel<<<dim3((unsigned)grid), 64 * AT_WAVES, lds, st>>>(a, tiles, units);
        return hipGetLastError();
    };
    if (exact) return general ? go(att_tile_kernel<BF, DP, true, true>) : go(att_tile_kernel<BF, DP, true, false>);
    return general ? go(att_tile_kernel<BF, DP, false, true>) : go(att_tile_kernel<BF, DP, false, false>);
}

}  // namespace
