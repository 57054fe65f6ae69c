// Attention of many rows over a cache of 8-bit codes (prompts, chunks): a workgroup of four wavefronts holds 128 rows of the products and
// walks over the cache in blocks of 64 keys, as for the other types.
//
//   y = c1 (q . code) ks(page),  w = 2^(y - m),  o = S sum_j [w vs(page) / S] code_j,  S the largest vs seen so far
//
// Codes are fp16 numbers exactly: a block's are fetched to registers while the block before is in work, become fp16 there, once for the
// workgroup, and go to LDS, from where the products on 32x32 fp16 MFMA read them as they read bf16 ones elsewhere.  The pages' scales
// stay outside the products: eight keys side by side lie in one page, so that a block has eight scales of each kind, scalars, which
// multiply scores (as they become weights, where there is no cap or bias) and weights (32 a lane).  Queries are brought to [2^14, 2^15)
// by one power of two for the wavefront's 32 rows, or one each where they lie apart, in one term for bf16 and two for fp32: what is less
// than 2^-29 of a row's largest element is lost.  The maximum m moves where it is off by 2^4, so that weights times vs / S stay below
// 2^4 and enter the second product times 2^11, in one term of 11 bits or two.
//
// Bound by vector instructions: a wavefront's block takes about 440 of them, 32 exponentials among them, beside 32 (128 columns) MFMA of 32
// cycles, with two wavefronts a SIMD (a prompt: MFMA 30 % of SIMD cycles, vector instructions 57 %, a quarter of a wavefront's time spent waiting to
// issue; chunks with a bias 26 and 56 %).  A prompt of 4096, 32 query heads of 128 columns, i8: 206 us, 667 TFLOP/s of the 1229 that a large fp16
// product reaches; chunks of 333 behind up to 7001, with a bias, 283 us; 1000 fp32 rows of documents 37 us, of which 17 are the start and a
// document's six blocks the rest.
// Scales in the exponent and an instance for each code: 214 -> 199 us; one power of two for all rows alike, whatever their size: 198, but a row
// beside larger ones lost its bits.  Not taken: eight wavefronts that share a block (prompt -3 %, chunks +9 %); conversions spread over the
// products (spills: 533 us); three or four wavefronts a SIMD (spills).
#pragma once
#include "attention_order.h"
#include "code8.h"

namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

template <int DP>
struct At8Shape {
    static constexpr int BK = 64;                      // keys of a block
    static constexpr int ROWB = DP * 2;                // bytes of a row in LDS
    static constexpr int CH = ROWB / 16;               // 16-byte pieces of a row
    static constexpr int TILE = BK * ROWB;             // bytes of a block of keys, and of values
    static constexpr int PIECES = BK * DP / 16 / (64 * AT_WAVES);      // of 16 codes, a thread
    static constexpr int LDS = 4 * TILE + AT_MAP / 8 + 2 * AT_WAVES * 4 + 8 * AT_WAVES;    // two blocks of each, a map of blocks, words of the wavefronts
};
template <int T, int DP>
constexpr int at8_groups() { return T == 2 || DP == 256 ? 1 : 2; }     // workgroups of a compute unit

// (fmaxf would make each number a quiet one first)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// T: terms of queries and weights, 1 for bf16, 2 for fp32; I8: integers (else e4m3); DP: columns, 64, 128 or 256; EXACT: d == DP; FORM: AttForm, scale, cap and bias
template <int T, bool I8, int DP, bool EXACT, int FORM>
__global__ __launch_bounds__(64 * AT_WAVES, (at8_groups<T, DP>())) void att8_tile_kernel(AttArgs a, Att8 e8, AtOrder order, AttSplit sp,
                                                                                      float* __restrict__ part, float4* __restrict__ stat) {
    using S = At8Shape<DP>;
    constexpr bool BF = T == 1;
    constexpr int ES = BF ? 2 : 4, BK = S::BK, ROWB = S::ROWB, CH = S::CH, DT = DP / 32, CS = CH / 2;
    constexpr bool GENERAL = FORM != ATT_PLAIN, CAPS = FORM == ATT_LONG || (FORM == ATT_SHORT && DP < 256);
    extern __shared__ __align__(16) char smem[];
    char* const ks = smem;                             // [2][BK][ROWB]
    char* const vs = smem + 2 * S::TILE;

    int split, unit, tile;
    at_place(blockIdx.x, order, split, unit, tile);
    const int b = unit / a.hkv, h = unit - b * a.hkv;
    const AttSeq s = att_seq(a, b);
    const int rows = s.fresh * a.group;
    // this workgroup's part of the cached tokens, if the sequence has several
    const bool whole_length = s.n <= sp.chunk;
    const int from = split * sp.chunk;
    if (tile * AT_ROWS >= rows || (split > 0 && from >= s.n)) return;

    const int lane = threadIdx.x & 63, wave = att_wave(), l32 = lane & 31, hf = lane >> 5;
    const int row = tile * AT_ROWS + wave * 32 + l32;
    const bool live = row < rows;
    const int tok = live ? row / a.group : 0, head = h * a.group + (live ? row - tok * a.group : 0);
    const AttRow me = att_row(s, tok, live);
    const float slope = GENERAL && a.slopes ? a.slopes[head] * ATT_LOG2E : 0.f;
    // rows that see nothing whatever the block: what they gather on the way, from queries of 0, is dropped at the end
    const bool blind = me.doc < 0;
    Terms<T> qf[CS];
    int q_exponent;                                    // ... of the power of two that was taken out of the rows
    bool apart;                                        // whether rows have their own: 2^row_exponent times that
    int row_exponent = 0;
    {
        const char* qp = a.q + (int64_t)(s.row0 + tok) * a.q_bytes + (int64_t)head * a.d * ES;
        v4u raw[CS][ES / 2];
        float most = 0.f;
        auto value = [&](int c, int e) {
            if constexpr (BF) return __uint_as_float(e & 1 ? raw[c][0][e / 2] & 0xffff0000u : raw[c][0][e / 2] << 16);
            else return __uint_as_float(raw[c][e / 4][e % 4]);
        };
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            const int at = (2 * c + hf) * 8;
#pragma unroll
            for (int i = 0; i < ES / 2; ++i)
                raw[c][i] = !blind && (EXACT || at < a.d) ? *(const v4u*)(qp + at * ES + 16 * i) : v4u{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = fabsf(value(c, e));
                most = fmaxf(most, v <= 3.402823466e38f ? v : 0.f);    // (what is not finite makes its row's scores so)
            }
        }
        // One power of two where the rows' largest elements lie within 2^10 of one another (or are 0): it goes into the keys' scales.  Else one a
        // row, so that none of them loses bits to another's size; what they have beyond 2^-60 of the largest one's multiplies the products.
        most = half_max(most);
        const auto exponent = [](float v) { return max((int)((__float_as_uint(v) >> 23) & 255) - 127, -100); };
        const int all = __builtin_amdgcn_readfirstlane(exponent(bwla_wave_max(most)));
        int up = most > 0.f ? exponent(most) : all;
        apart = some(up < all - 10);
        if (apart) row_exponent = up - (all - 60);
        else up = all;
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = ldexpf(value(c, e), 14 - up);
            qf[c] = terms_of<T>(v);
        }
        q_exponent = (apart ? all - 60 : all) - 14;
    }
    // indexes of the first and last row of this wavefront, and of the workgroup
    const int old = s.old;
    const int w_first = old + min(tile * AT_ROWS + wave * 32, rows - 1) / a.group;
    const int w_last = old + min(tile * AT_ROWS + wave * 32 + 31, rows - 1) / a.group;
    const int g_first = max(old + tile * AT_ROWS / a.group, 0);
    const int g_last = old + min(tile * AT_ROWS + AT_ROWS - 1, rows - 1) / a.group;
    // blocks of keys: those of the prefix, then from the first row's window to the last row's index
    const int pb = min((max(s.prefix, 0) + BK - 1) / BK, (s.n + BK - 1) / BK);
    int lo = s.pos || a.window == INT32_MAX ? 0 : max(g_first - a.window + 1, 0) / BK;
    if (lo < pb) lo = pb;
    const int end = min(max((g_last + BK) / BK, pb), (int)(((int64_t)from + sp.chunk + BK - 1) / BK));
    // documents: the blocks that may hold keys of the rows'
    if (s.doc) {
        uint32_t* const active = (uint32_t*)(smem + 4 * S::TILE);              // a bit for each block that may matter
        int* const range = (int*)(active + AT_MAP / 32);
        int dmin = blind ? INT32_MAX : me.doc, dmax = me.doc;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            dmin = min(dmin, __shfl_xor(dmin, i, 64));
            dmax = max(dmax, __shfl_xor(dmax, i, 64));
        }
        if (lane == 0) { range[wave] = dmin; range[AT_WAVES + wave] = dmax; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < AT_WAVES; ++w) {
            dmin = min(dmin, range[w]);
            dmax = max(dmax, range[AT_WAVES + w]);
        }
        // a wavefront looks at 32 blocks, whose word it writes, all loads on the way at once
        for (int w = from / BK / 32 + wave; w < (min(end, AT_MAP) + 31) / 32; w += AT_WAVES) {
            uint32_t word = 0;
            int d[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) d[i] = s.doc[min((w * 32 + i) * BK + lane % BK, s.n - 1)];
#pragma unroll
            for (int i = 0; i < 32; ++i) word |= __any((d[i] >= dmin) & (d[i] <= dmax)) ? 1u << i : 0u;
            if (lane == 0) active[w] = word;
        }
        __syncthreads();
    }
    // the block behind t, `end` where there is none
    auto behind = [&](int t) {
        for (;;) {
            ++t;
            if (t >= pb && t < lo) t = lo;
            if (t >= end) return end;
            if (!s.doc || t >= AT_MAP) return t;
            const uint32_t* const active = (const uint32_t*)(smem + 4 * S::TILE);
            const uint32_t left = (uint32_t)__builtin_amdgcn_readfirstlane((int)active[t / 32]) >> (t & 31);
            if (left & 1) return t;
            t = left ? t + __builtin_ctz(left) - 1 : (t | 31);
        }
    };

    const char* const kh = a.k + (int64_t)h * a.head_bytes;
    const char* const vh = a.v + (int64_t)h * a.head_bytes;
    const int slot_mask = (1 << a.page_shift) - 1;

    // ---- blocks.  Lane l looks up where key l of a block lies, and its page's scales; a lane that fetches a piece of a key's row has it
    // from there.  Pieces lie in LDS at piece ^ (key & KSW) of a row of keys, piece ^ (key & VSW) * 2 of values.
    constexpr int KSW = (CH < 16 ? CH : 16) - 1, VSW = CH < 16 ? 3 : 7;
    struct Found { int page, pos, doc; };
    // (without positions or documents an entry of the table is read for them and dropped: no branch lies in the way of what overlaps)
    const int32_t* const positions = s.pos ? s.pos : s.table;
    const int32_t* const documents = s.doc ? s.doc : s.table;
    const int has_pos = s.pos ? -1 : 0, has_doc = s.doc ? -1 : 0;
    auto look = [&](int t) {                           // (kept as loaded: nothing here waits)
        Found f;
        const int j = t * BK + lane, in = min(j, s.n - 1);
        f.page = s.table[in >> a.page_shift];
        f.pos = positions[in & has_pos];
        f.doc = documents[in & has_doc];
        f.pos = has_pos ? f.pos : j;
        f.doc = has_doc ? f.doc : 0;
        return f;
    };
    struct Key { int64_t at; int p, doc; float kscale, vscale; };              // doc: -1 where the key does not exist
    auto settle = [&](const Found& f, int t) {
        Key k;
        const int j = min(t * BK + lane, s.n - 1);
        const bool there = (unsigned)f.page < (unsigned)a.pages && t * BK + lane < s.n;
        const int page = there ? f.page : 0;           // (read, and not used)
        k.at = (int64_t)page * a.page_bytes + (int64_t)(j & slot_mask) * a.slot_bytes;
        k.p = max(f.pos, 0);
        k.doc = there ? max(f.doc, -1) : -1;
        k.kscale = e8.k_scale[page * e8.stride + h];
        k.vscale = e8.v_scale[page * e8.stride + h];
        return k;
    };
    constexpr int PER = DP / 16;                       // pieces of 16 codes of a row
    const int key0 = threadIdx.x / PER, piece = threadIdx.x % PER;
    constexpr int STEP = 64 * AT_WAVES / PER;          // keys between a thread's pieces
    v4u got_k[S::PIECES], got_v[S::PIECES];
    auto fetch_codes = [&](int64_t at) {
        const bool in = EXACT || piece * 16 < a.d;
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            const int key = key0 + i * STEP;
            const int64_t off = ((int64_t)__shfl((int)(at >> 32), key, 64) << 32) | (uint32_t)__shfl((int)at, key, 64);
            got_k[i] = in ? *(const v4u*)(kh + piece * 16 + off) : v4u{0, 0, 0, 0};
            got_v[i] = in ? *(const v4u*)(vh + piece * 16 + off) : v4u{0, 0, 0, 0};
        }
    };
    auto put_block = [&](int buf) {
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            const int key = key0 + i * STEP;
            char* const kr = ks + buf * S::TILE + key * ROWB;
            char* const vr = vs + buf * S::TILE + key * ROWB;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const Halves k0 = code_halves<I8>(got_k[i][2 * p]), k1 = code_halves<I8>(got_k[i][2 * p + 1]);
                *(v4u*)(kr + ((2 * piece + p) ^ (key & KSW)) * 16) = v4u{k0.lo, k0.hi, k1.lo, k1.hi};
                const Halves v0 = code_halves<I8>(got_v[i][2 * p]), v1 = code_halves<I8>(got_v[i][2 * p + 1]);
                *(v4u*)(vr + ((2 * piece + p) ^ (key & VSW) * 2) * 16) = v4u{v0.lo, v0.hi, v1.lo, v1.hi};
            }
        }
    };

    v16f o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    float m = -INFINITY, l = 0.f, base = 0.f;          // base: what weights take off their scores, m where there is one and it is not taken off before
    float top_scale = 0.f, down = 0.f;                 // S, and 2^11 / S

    // where lane (i = lane & 15 of each 16) of a transposing read takes its 8 bytes: key 4 hf + (i >> 2), columns
    // 16 (lane >> 4 & 1) + 4 (i & 3) of a column tile
    const int tk = 4 * hf + ((lane & 15) >> 2);
    int vofs[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) vofs[d] = tk * ROWB + ((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (tk & VSW) * 2) * 16 + (lane & 1) * 8;

    // ---- the steps of a tile of 32 keys
    struct Packed { Terms<T> w[2]; };                   // weights as operands: 16 keys each
    // A block's scales, of eight keys each: of keys, with what else a product is multiplied by; of values, as a factor F vs / S (two terms), or
    // that factor's logarithm and reciprocal.
    float kg[8], vg[8], lv[8];
    auto products = [&](const char* kb, int k, v16f& sc) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = 0.f;
        const char* src = kb + (k * 32 + l32) * ROWB;
        v16f low = sc;                                 // (second terms apart: half as many roundings of the large sum)
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            const v8h kf = *(const v8h*)(src + ((2 * c + hf) ^ (l32 & KSW)) * 16);
            sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[c].t[0], sc, 0, 0, 0);
            if constexpr (T == 2) low = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[c].t[1], low, 0, 0, 0);
        }
        if constexpr (T == 2) sc += low;
    };
    // Behind a matrix instruction of 8 passes 12 others have to be issued before its result is read.  The compiler sees to that, but not where a
    // branch that may be skipped lies between (it counts the longer way): weights were taken relative to a maximum of numbers that were
    // not there yet.
    auto arrive = [&](v16f& sc) { asm volatile("s_nop 11" : "+v"(sc)); };
    // ... and the same of the sums, where they are scaled right behind a product: what decided how long that was is a branch as well.
    auto arrived = [&] {
        if constexpr (DT == 2) asm volatile("s_nop 11" : "+v"(o[0]), "+v"(o[1]));
        else if constexpr (DT == 4) asm volatile("s_nop 11" : "+v"(o[0]), "+v"(o[1]), "+v"(o[2]), "+v"(o[3]));
        else asm volatile("s_nop 11" : "+v"(o[0]), "+v"(o[1]), "+v"(o[2]), "+v"(o[3]), "+v"(o[4]), "+v"(o[5]), "+v"(o[6]), "+v"(o[7]));
    };
    // Weights of a tile's scores as they enter the second product, w F vs / S (F = 2^11), and the sums of w alone.  (Without cap and bias scores
    // stay products until here: y - m is rounded once.)  One term: the factor is part of the exponent, and goes out of the sum for four keys
    // at once, which takes an instruction less a score and costs a weight 2^-13 at most: the logarithm is rounded where m is taken off it.  Two
    // terms: the weight, then the product.
    bool huge = false;                                 // scores of HUGE_SCORE and more, from which m is taken off before
    auto weigh = [&](const v16f& sc, Packed& out, int k) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float w[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int g = 4 * k + 2 * u + q;
                const float less = T == 1 ? lv[g] - base : -base;
#pragma unroll
                for (int e = 4 * q; e < 4 * q + 4; ++e) {
                    const float y = sc[8 * u + e];
                    w[e] = __builtin_amdgcn_exp2f(GENERAL ? y + less : fmaf(y, kg[g], less));
                }
                if constexpr (T == 1) {
                    l = fmaf((w[4 * q] + w[4 * q + 1]) + (w[4 * q + 2] + w[4 * q + 3]), vg[g], l);
                } else {
#pragma unroll
                    for (int e = 4 * q; e < 4 * q + 4; ++e) {
                        l += w[e];
                        w[e] *= vg[g];
                    }
                }
            }
            out.w[u] = terms_of<T>(w);
        }
    };
    // O^T += V^T P^T: operands, and their products
    struct Operands { v8h x[2 * DT]; };
    auto fetch = [&](const char* vb, int k) {
        Operands f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const char* at = vb + vofs[d] + (k * 32 + 16 * u) * ROWB;
                const v2u x0 = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)at));
                const v2u x1 = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at + 8 * ROWB)));
                f.x[u * DT + d] = __builtin_bit_cast(v8h, v4u{x0[0], x0[1], x1[0], x1[1]});
            }
        return f;
    };
    auto values = [&](const Operands& f, const Packed& p) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int n = 0; n < T; ++n) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.x[u * DT + d], p.w[u].t[n], o[d], 0, 0, 0);
    };
    // the compiler is told to have these now
    auto hold = [&](Packed& p) {
        if constexpr (T == 1) asm volatile("" : "+v"(p.w[0].t[0]), "+v"(p.w[1].t[0]), "+v"(l));
    };
    // Large scores.  From 2^20 on m, a rounded one, would be off by whole numbers of products that are not, and with one term the
    // logarithm of the values' factor loses bits to m much sooner.  There products are rounded, and m is taken off them before anything
    // else is added, so that the largest has a weight of 1 whatever its size, and keys weigh as their values' scales say.
    constexpr float HUGE_SCORE = T == 1 ? 0x1p12f : 0x1p20f;
    auto round_now = [&](v16f& sc, int k) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] *= kg[4 * k + r / 4];
#pragma unroll
        for (int g = 0; g < 4; ++g) kg[4 * k + g] = 1.f;
    };
    // The maximum moves only when it is off by 2^4; what was summed with the old one follows.
    // (first: what has to be added with the old one before)
    auto raise = [&](v16f& sc, int k, auto first) {
        float four[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            four[g] = max3(sc[4 * g], sc[4 * g + 1], max3(sc[4 * g + 2], sc[4 * g + 3], -INFINITY));
            if constexpr (!GENERAL) four[g] *= kg[4 * k + g];
        }
        float top = max3(four[0], four[1], max3(four[2], four[3], -INFINITY));
        top = half_max(top);
        if (__builtin_expect(some(top > m + 4.f), 0)) {
            first();
            const float now = fmaxf(m, top);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= f;
            base = m == -INFINITY ? 0.f : m;
            if constexpr (!GENERAL || T == 1) {        // (two terms and a cap or a bias: scores are rounded as it is)
                const bool was = huge;
                huge = some(fabsf(m) >= HUGE_SCORE && m > -INFINITY);
                base = huge || m == -INFINITY ? 0.f : m;
                if (!GENERAL && __builtin_expect(huge && !was, 0)) round_now(sc, k);
            }
        }
    };

    // blocks t, t1, t2, t3 in turn: in work, fetched, found, looked up
    int t = behind(from / BK - 1), t1 = t < end ? behind(t) : end, t2 = t1 < end ? behind(t1) : end;
    Key now{0, 0, -1, 0.f, 0.f}, next{0, 0, -1, 0.f, 0.f};                     // keys of t and t1
    Found far{0, 0, 0};                                // ... of t2, as loaded
    if (t < end) {
        const Found f0 = look(t), f1 = look(min(t1, end - 1));
        far = look(min(t2, end - 1));
        now = settle(f0, t);
        fetch_codes(now.at);
        next = settle(f1, min(t1, end - 1));
        put_block(0);
    }
    constexpr int AHEAD = CS < 4 ? CS : 4;             // operands of the first product read ahead of it
    constexpr uint64_t ALL = ~0ull;
    for (int buf = 0; t < end; buf ^= 1) {
        const int j0 = t * BK, t3 = t2 < end ? behind(t2) : end;
        const char* const kb = ks + buf * S::TILE;
        const char* const vb = vs + buf * S::TILE;
        bwla_lds_barrier();                            // everyone's codes of the block are there, and the other buffer is free
        // What comes next: codes of t1, addresses of t2, entries of t3 (or, at the end, of the last block once more: no branches).  Its
        // instructions go between the first products, its conversions between the last ones.
        Key after;
        auto prepare = [&] {
            fetch_codes(next.at);
            after = settle(far, min(t2, end - 1));
            far = look(min(t3, end - 1));
        };
        prepare();
        // Even: every key exists and is of one document, and in reach of the windows, so that a row of that document sees those up
        // to its index, or all of the prefix.  Else each wavefront works out what each of its rows sees (a bit for each key).  Values
        // of keys that no row of the workgroup sees may be anything: integers get a weight of 0, but e4m3 codes may be NaN and are
        // cleared.
        const int doc = __builtin_amdgcn_readfirstlane(now.doc);
        const bool even = doc >= 0 && !some(now.doc != doc) &&
                          (a.window == INT32_MAX || (!s.pos && j0 > g_last - a.window) || j0 + BK <= s.prefix);
        const bool mine = me.doc == doc;
        uint64_t ok = ALL, any = ALL;
        if (__builtin_expect(!even, 0)) {
            ok = att_seen(a, s, me, j0, now.p, now.doc);
            any = att_rows_or(ok);
            if constexpr (!I8) {
                uint64_t* const seen = (uint64_t*)(smem + 4 * S::TILE + AT_MAP / 8 + 2 * AT_WAVES * 4);
                if (lane == 0) seen[wave] = any;
                bwla_lds_barrier();
                const uint64_t all = seen[0] | seen[1] | seen[2] | seen[3];
                static_assert(AT_WAVES == 4, "one word each");
                for (int i = lane; i < BK / AT_WAVES * CH; i += 64) {
                    const int key = wave * (BK / AT_WAVES) + i / CH;
                    if (!((all >> key) & 1)) *(v4u*)(vs + buf * S::TILE + key * ROWB + i % CH * 16) = v4u{0, 0, 0, 0};
                }
                bwla_lds_barrier();
            }
        }
        if (even ? some(mine) && (j0 <= w_last || j0 < s.prefix) : any != 0) {
            // every row sees every key
            const bool whole = even && !some(!(mine | blind)) && (j0 + BK - 1 <= w_first || j0 + BK <= s.prefix);
            // a bias alone, and keys no later than rows: no cap, no distance either way
            [[maybe_unused]] const bool linear = GENERAL && (!CAPS || a.capped == 0.f) && a.slopes && !s.pos && (j0 >= s.prefix || j0 + BK - 1 <= w_first);
            const bool plainly = whole && (GENERAL || !apart);
            // scales of pages of which no row sees a key may be anything, and count as 0
            {
                // (an even block's keys up to the last row's are seen, and those of the prefix; what lies behind costs these rows no bits)
                const bool in_use = even ? j0 + (lane & 56) <= max(w_last, s.prefix - 1) : ((any >> (lane & 56)) & 0xff) != 0;
                const float vscale = in_use ? now.vscale : 0.f;
                if (__builtin_expect(some(vscale > top_scale), 0)) {
                    const float up = fmaxf(fmaxf(bwla_wave_max(vscale), top_scale), 0x1p-126f), f = top_scale / up;       // (a reciprocal has to be there)
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[d][r] *= f;
                    top_scale = up;
                    down = 1.f / up;
                }
                // (never 0: an unseen key's product is -inf, and a page of zeros still has weights; 2^-60 is nothing beside 2^11)
                const float kq = fmaxf(ldexpf(now.kscale, q_exponent) * (CAPS && a.capped != 0.f ? 1.f : a.c1), 0x1p-126f), vq = vscale * down * 2048.f, vn = fmaxf(vq, 0x1p-60f);
                const float logarithm = __builtin_amdgcn_logf(vn);
                // (of the logarithm as it is, rounded: what goes out of the sum is what went in)
                const float factor = T == 1 ? __builtin_amdgcn_exp2f(-logarithm) : vq;
                const auto of = [](float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); };
                if (a.page_shift >= 6 && even) {               // one page: its scales are all of them
                    const float k0 = of(kq, 0), v0 = of(factor, 0), l0 = of(logarithm, 0);
#pragma unroll
                    for (int i = 0; i < 8; ++i) { kg[i] = k0; vg[i] = v0; lv[i] = l0; }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        kg[i] = of(kq, 8 * i);
                        vg[i] = of(factor, 8 * i);
                        if constexpr (T == 1) lv[i] = of(logarithm, 8 * i);
                    }
                }
            }
            // a tile's scores made ready: scales, cap, bias, mask, and a maximum that will do for them
            auto ready = [&](v16f& sc, int k, auto first) {
                arrive(sc);
                const auto scaled = [&] {
#pragma unroll
                    for (int r = 0; r < 16; ++r) sc[r] = ldexpf(sc[r], row_exponent);
                };
                if constexpr (GENERAL) {
                    if (__builtin_expect(apart, 0)) scaled();
                    if (linear) {
                        // A slope times the row's distance to the first of four keys, and 0 to 3 slopes back: an instruction a score less
                        // than scale, distance and bias one after the other (chunks 284 -> 273 us, that prompt with a bias 269 -> 247).
                        const float to = -slope * (float)(me.p - j0 - k * 32 - 4 * hf), three = 3.f * slope;
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const float b = g ? fmaf(8.f * g, slope, to) : to;
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                sc[4 * g + e] = fmaf(sc[4 * g + e], kg[4 * k + g], e == 0 ? b : e == 1 ? b + slope : e == 2 ? fmaf(2.f, slope, b) : b + three);
                        }
                    } else {
#pragma unroll
                        for (int r = 0; r < 16; ++r) sc[r] *= kg[4 * k + r / 4];
                        if (CAPS && a.capped != 0.f) {
                            // The short form, off by 1.2e-7 of the cap, where every row sees every key, so that little of it is left in their
                            // sum (a row of two keys has an lse of 2, of which that is 1e-6); a prompt of 4096 with it there and nowhere: 269 and 284 us.
                            // (256 columns: nowhere, and caps in an instance of their own, as another body spills: 2048 rows with a bias 197 -> 239 us, with
                            // a cap 186, where the short form for all of them takes 160.)
                            if constexpr (FORM == ATT_LONG && DP < 256) {
                                capped_scores<16>(a, sc);
                            } else if (FORM == ATT_SHORT && whole) {
                                const float c3 = a.c2 * (2.f * ATT_LOG2E);
#pragma unroll
                                for (int r = 0; r < 16; ++r)
                                    sc[r] = fmaf(-2.f * a.capped, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(sc[r] * c3)), a.capped);
                            } else {
#pragma unroll
                                for (int r = 0; r < 16; ++r) sc[r] = a.capped * att_tanh(sc[r] * a.c2);
                            }
                        }
                        if (a.slopes && s.pos) {
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                sc[r] = fmaf(-slope, fabsf((float)(me.p - __shfl(now.p, k * 32 + (r & 3) + 8 * (r >> 2) + 4 * hf, 64))), sc[r]);
                        } else if (a.slopes) {
                            const float away = (float)(me.p - j0 - k * 32 - 4 * hf);
#pragma unroll
                            for (int r = 0; r < 16; ++r) sc[r] = fmaf(-slope, fabsf(away - (float)((r & 3) + 8 * (r >> 2))), sc[r]);
                        }
                    }
                }
                if (!__builtin_expect(plainly && !huge, 1)) {
                    if (!GENERAL && apart) scaled();
                    if (!GENERAL && huge) round_now(sc, k);
                    if (plainly) {                     // (here for the rounding alone)
                    } else if (even) {
                        const int most = (mine ? max(me.i, s.prefix - 1) : -1) - j0 - k * 32 - 4 * hf;
#pragma unroll
                        for (int r = 0; r < 16; ++r) sc[r] = (r & 3) + 8 * (r >> 2) <= most ? sc[r] : -INFINITY;
                    } else {
                        const uint32_t bits = (uint32_t)(ok >> (32 * k)) >> (4 * hf);
#pragma unroll
                        for (int r = 0; r < 16; ++r) sc[r] = (bits >> ((r & 3) + 8 * (r >> 2))) & 1 ? sc[r] : -INFINITY;
                    }
                }
                raise(sc, k, first);
                if (__builtin_expect(huge, 0)) {
                    const float all = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int r = 0; r < 16; ++r) sc[r] -= all;
                }
            };
            // (Order and priorities as in the kernel of the other types: the weights of one tile are taken while the other's products run.)
            constexpr int MFMAS = CS * T, VALU = 88;
            v16f s0, s1;
            Packed p0, p1;
            __builtin_amdgcn_s_setprio(1);
            products(kb, 0, s0);
            __builtin_amdgcn_s_setprio(0);
            ready(s0, 0, [] {});
            __builtin_amdgcn_s_setprio(1);
            products(kb, 1, s1);
            weigh(s0, p0, 0);
            hold(p0);                                  // (here, and not where they are used)
            if constexpr (T == 1) {
                __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 1);
#pragma unroll
                for (int i = 0; i < MFMAS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                    if (i < MFMAS - AHEAD) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
                    __builtin_amdgcn_sched_group_barrier(0x002, VALU / MFMAS, 1);
                }
            }
            __builtin_amdgcn_s_setprio(0);
            ready(s1, 1, [&] {
                values(fetch(vb, 0), p0);
                arrived();
                const v8h zero = {};
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int n = 0; n < T; ++n) p0.w[u].t[n] = zero;
            });
            __builtin_amdgcn_s_setprio(1);
            const Operands f0 = fetch(vb, 0);
            __builtin_amdgcn_sched_barrier(0);
            values(f0, p0);
            weigh(s1, p1, 1);
            if constexpr (T == 1) {
#pragma unroll
                for (int i = 0; i < 2 * DT; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 2);
                    __builtin_amdgcn_sched_group_barrier(0x002, VALU / (2 * DT), 2);
                }
            }
            const Operands f1 = fetch(vb, 1);
            __builtin_amdgcn_sched_barrier(0);
            values(f1, p1);
            __builtin_amdgcn_s_setprio(0);
        }
        put_block(buf ^ 1);
        now = next;
        next = after;
        t = t1;
        t1 = t2;
        t2 = t3;
    }

    l = half_sum(l);
    if (blind) l = 0.f;
    if (!live) return;
    const float back = top_scale * 0x1p-11f;
    if (!whole_length) {                               // in tiles of 16 rows, as the join reads them
        const int64_t to = ((int64_t)(unit * sp.row_tiles + row / 16) * sp.splits + split) * 16 + row % 16;
        if (hf == 0) stat[to] = make_float4(blind ? -INFINITY : att_part_max(m, l), l, l, 0.f);
        if (m != -INFINITY) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *(float4*)(part + to * DP + 32 * d + 2 * r + 4 * hf) = make_float4(o[d][r] * back, o[d][r + 1] * back, o[d][r + 2] * back, o[d][r + 3] * back);
        }
        return;
    }
    const float over = att_over(l, l);                 // (apart from `back`: their product may have few bits)
    const int64_t at = (int64_t)(s.row0 + tok) * a.hq + head;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int c = 32 * d + 2 * r + 4 * hf;
            if (EXACT || c < a.d) att_put<BF>(a, at, c, make_float4(o[d][r] * back, o[d][r + 1] * back, o[d][r + 2] * back, o[d][r + 3] * back), over);
        }
    if (hf == 0) att_put_lse(a, at, m, l);
}

template <int T, bool I8, int DP>
hipError_t at8_launch(const AttArgs& a, const Att8& e8, const AttSplit& sp, void* ws, hipStream_t st) {
    const int tiles = (sp.rows + AT_ROWS - 1) / AT_ROWS;
    const int units = a.seqs * a.hkv;
    if ((int64_t)tiles * units * sp.splits >= 1 << 24) return hipErrorInvalidConfiguration;       // (a grid has fewer than 2^32 threads)
    const AtOrder order = at_order_of(tiles, units, sp.splits, at8_groups<T, DP>());
    constexpr int lds = At8Shape<DP>::LDS;
    // (256 columns: caps have the instance that is exact to units of the score)
    const int form = DP == 256 && a.capped != 0.f ? ATT_LONG : att_form(a, T == 1);
    const bool exact = a.d == DP;
    float* const part = (float*)ws;
    float4* const stat = (float4*)((char*)ws + sp.part_bytes);
    auto go = [&](auto kernel) {
        const hipError_t e = bwla_ensure_lds((const void*)kernel, lds);
        if (e != hipSuccess) return e;
        kernel<<<dim3((unsigned)((int64_t)tiles * units * sp.splits)), 64 * AT_WAVES, lds, st>>>(a, e8, order, sp, part, stat);
        return hipGetLastError();
    };
    if (form == ATT_PLAIN) return exact ? go(att8_tile_kernel<T, I8, DP, true, ATT_PLAIN>) : go(att8_tile_kernel<T, I8, DP, false, ATT_PLAIN>);
    constexpr int SHORT = T == 1 ? ATT_SHORT : ATT_LONG;
    if (form == SHORT) return exact ? go(att8_tile_kernel<T, I8, DP, true, SHORT>) : go(att8_tile_kernel<T, I8, DP, false, SHORT>);
    return exact ? go(att8_tile_kernel<T, I8, DP, true, ATT_LONG>) : go(att8_tile_kernel<T, I8, DP, false, ATT_LONG>);
}
template <int T, bool I8>
hipError_t at8_launch_columns(const AttArgs& a, const Att8& e8, const AttSplit& s, void* ws, hipStream_t st) {
    if (a.d <= 64) return at8_launch<T, I8, 64>(a, e8, s, ws, st);
    if (a.d <= 128) return at8_launch<T, I8, 128>(a, e8, s, ws, st);
    return at8_launch<T, I8, 256>(a, e8, s, ws, st);
}

}  // namespace
