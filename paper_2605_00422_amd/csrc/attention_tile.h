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
// that keeps the keys' reads off each other's banks.
// A prompt of 8192 with 32 heads of 128 columns: 684 us, 804 TFLOP/s (a large bf16 product: 1127), in an unbroken row of calls (the first
// ones after a pause: 745); a cap 833 us, one above 128 1049, a bias 853, 64 columns 410.
// Of a SIMD's cycles 37 % are MFMA and 50 % vector instructions (of a row's scores: the test of the maximum, exponential, sum and
// rounding), 11 % both at once: two wavefronts a SIMD, 219 registers each, and what one wavefront's order interleaves.  With a cap 29 %
// and 65 %: its exponential and reciprocal take twice the cycles of other instructions.  A block of 64 keys takes two
// workgroups 3.2 us, one alone 2.2; 2048 tokens: 65 us, bound by workgroups of 32 blocks.  Four wavefronts and not eight, which share
// their copies: 790 against 787 us, with a cap 944 against 1007.
#pragma once
#include "attention.h"

namespace {

constexpr int AT_WAVES = 4;
constexpr int AT_ROWS = 32 * AT_WAVES;
constexpr int AT_MAP = 4096;                           // blocks of keys that the map of active ones covers; those behind count as active
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Workgroups are dealt round-robin to the 8 XCDs, and units (sequence, key-value head) to workgroups, so that the rows of one unit mostly
// lie on one XCD, whose L2 then has their keys and values.  (A few units at a time instead of all: 795 -> 810 us for a prompt of 8192
// with 32 heads.)  The parts of a divided cache come one after the other, the first, which all sequences have, in front (all units
// and parts at once: 296 -> 391 us for four chunks behind caches of 900 to 7001 tokens).  With each tile the units are turned by one
// an XCD, whose shader engines are dealt workgroups in turn as well: else each of the four has a sequence for itself, and where the
// shortest is done the next workgroup still waits for its own (297 -> 358 us there).  Later tiles of rows see more keys: the longest
// first, which evens out where there are many workgroups, or, where all run at once, the first half of them from the longest down
// and the second from the shortest up, so that a compute unit gets a long one and a short one.
struct AtOrder {
    int tiles, units, fold;
};
inline AtOrder at_order_of(int tiles, int units, int splits, int per_cu) {
    return AtOrder{tiles, units, (int64_t)tiles * units * splits <= (int64_t)per_cu * bwla_device_cus()};
}
__device__ __forceinline__ void at_place(int id, const AtOrder& o, int& split, int& unit, int& tile) {
    const int size = o.units * o.tiles;
    split = id / size;
    const int at = id - split * size, k = at / o.units, half = o.tiles / 2;
    unit = (int)((unsigned)(at - k * o.units + 8 * k) % (unsigned)o.units);
    tile = o.fold && k >= o.tiles - half ? k - (o.tiles - half) : o.tiles - 1 - k;
}

template <bool BF, int DP>
struct AtShape {
    static constexpr int ES = BF ? 2 : 4;
    static constexpr int BK = BF ? 64 : 32;            // keys of a block
    static constexpr int ROWB = DP * ES;               // bytes of a row in LDS
    static constexpr int CH = ROWB / 16;               // 16-byte pieces of a row
    static constexpr int TILE = BK * ROWB;             // bytes of a block of keys, and of values
    static constexpr int COPIES = BK * CH / (64 * AT_WAVES);
    static constexpr int LDS = 4 * TILE + AT_MAP / 8 + 2 * AT_WAVES * 4 + 8 * AT_WAVES;    // two blocks of each, a map of blocks, words of the wavefronts
};

// BF: bf16 (else fp32); DP: columns, 64, 128 or 256; EXACT: d == DP; FORM: AttForm, scale, cap and bias
template <bool BF, int DP, bool EXACT, int FORM>
__global__ __launch_bounds__(64 * AT_WAVES, DP == 256 ? 1 : 2) void att_tile_kernel(AttArgs a, AtOrder order, AttSplit sp, float* __restrict__ part,
                                                                                float4* __restrict__ stat) {
    using S = AtShape<BF, DP>;
    constexpr int ES = S::ES, BK = S::BK, ROWB = S::ROWB, CH = S::CH, KT = BK / 32, DT = DP / 32, CS = CH / 2;
    constexpr bool GENERAL = FORM != ATT_PLAIN;
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
    v4u qf[CS];
    {
        const char* qp = a.q + (int64_t)(s.row0 + tok) * a.q_bytes + (int64_t)head * a.d * ES;
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            const int at = (2 * c + hf) * 16;
            qf[c] = !blind && (EXACT || at < a.d * ES) ? *(const v4u*)(qp + at) : v4u{0, 0, 0, 0};
        }
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

    // ---- copies.  Lane l looks up where key l of a block lies; a lane that copies a piece of a key's row has it from there.
    // Pieces lie in LDS at piece ^ (key & KSW) of a row of keys, piece ^ (key & VSW) * 2 of values.
    constexpr int KSW = (CH < 16 ? CH : 16) - 1, VSW = BF ? (CH < 16 ? 3 : 7) : 0;
    struct Found { int page, pos, doc; };
    auto look = [&](int t) {                           // (kept as loaded: nothing here waits)
        Found f;
        const int j = t * BK + lane % BK, in = min(j, s.n - 1);
        f.page = s.table[in >> a.page_shift];
        f.pos = s.pos ? s.pos[in] : j;
        f.doc = s.doc ? s.doc[in] : 0;
        return f;
    };
    struct Key { int64_t at; int p, doc; };            // doc: -1 where the key does not exist
    auto settle = [&](const Found& f, int t) {
        Key k;
        const int j = min(t * BK + lane % BK, s.n - 1);
        const bool there = (unsigned)f.page < (unsigned)a.pages && t * BK + lane % BK < s.n;
        k.at = (int64_t)(there ? f.page : 0) * a.page_bytes + (int64_t)(j & slot_mask) * a.slot_bytes;   // (read, and not used)
        k.p = max(f.pos, 0);
        k.doc = there ? max(f.doc, -1) : -1;
        return k;
    };
    // (an instruction of a wavefront copies the rows of 64 / CH keys, or part of one; those of instruction i + 1 are STEP keys on,
    // which for most shapes leaves the order of their pieces)
    constexpr int PER = 64 / CH, STEP = AT_WAVES * 64 / CH;
    static_assert(CH <= 64, "a row is one instruction's at most");
    const int key0 = wave * PER + lane / CH, piece = lane % CH;
    const uint32_t lds0 = att_lds_address(ks + wave * 1024);
    auto copy = [&](int64_t at, int buf) {
        const uint32_t to = lds0 + buf * S::TILE;
        att_each(std::make_integer_sequence<int, S::COPIES>{}, [&](auto n) {
            constexpr int i = decltype(n)::value;
            const int key = key0 + i * STEP;
            const int64_t off = ((int64_t)__shfl((int)(at >> 32), key, 64) << 32) | (uint32_t)__shfl((int)at, key, 64);
            const int pk = piece ^ ((STEP % (KSW + 1) == 0 ? key0 : key) & KSW), pv = piece ^ ((STEP % (VSW + 1) == 0 ? key0 : key) & VSW) * 2;
            if (EXACT || pk * 16 < a.d * ES) att_copy16<i * AT_WAVES * 1024>(kh + pk * 16 + off, to);
            if (EXACT || pv * 16 < a.d * ES) att_copy16<i * AT_WAVES * 1024 + 2 * S::TILE>(vh + pv * 16 + off, to);
        });
    };
    if constexpr (!EXACT) {                            // columns that no copy fills count as zero
        for (int i = threadIdx.x; i < 2 * BK * CH; i += 64 * AT_WAVES) {
            const int key = i / CH % BK, piece = i % CH;
            if ((piece ^ (key & KSW)) * 16 >= a.d * ES) *(v4u*)(ks + i * 16) = v4u{0, 0, 0, 0};
        }
    }

    v16f o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    float m = -INFINITY, l = 0.f, lr = 0.f;            // l: sum of the weights, lr: as the second product takes them
    // Weights enter the second product rounded to bf16, whose errors (2^-9 of a weight in the mean) average out over
    // many keys.  In blocks that are masked for some row, where one has seen fewer than FEW (in a lane's half), what the rounding lost
    // goes in as well: the first tokens of a prompt or a document, at no cost to the others.  (A block that all rows see brings each
    // of them 64 keys at once.)
    constexpr int FEW = 64;
    int had = 0;

    // where lane (i = lane & 15 of each 16) of a transposing read takes its 8 bytes: key 4 hf + (i >> 2), columns
    // 16 (lane >> 4 & 1) + 4 (i & 3) of a column tile
    const int tk = 4 * hf + ((lane & 15) >> 2);
    int vofs[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        if constexpr (BF) vofs[d] = tk * ROWB + ((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (tk & VSW) * 2) * 16 + (lane & 1) * 8;
        else vofs[d] = 4 * hf * ROWB + (32 * d + l32) * 4;
    }

    // ---- the steps of a tile of 32 keys
    typedef v4u Packed[BF ? 2 : 4];                    // weights as operands: 16 keys each; fp32: as they are
    auto products = [&](const char* kb, int k, v16f& sc) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = 0.f;
        const char* src = kb + (k * 32 + l32) * ROWB;
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            const v4u kf = *(const v4u*)(src + ((2 * c + hf) ^ (l32 & KSW)) * 16);
            if constexpr (BF) {
                sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, kf), __builtin_bit_cast(v8bf, qf[c]), sc, 0, 0, 0);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(qf[c][e]), sc, 0, 0, 0);
            }
        }
    };
    // weights of a tile's scores, and their sums; low: what the weights lose when rounded
    auto weigh = [&](const v16f& sc, Packed& out, auto low) {
        const float c1 = GENERAL ? 1.f : a.c1, base = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(fmaf(sc[8 * u + e], c1, -base));
                if constexpr (!decltype(low)::value) l += w[e];
            }
            if constexpr (BF) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t p = att_pack_bf16(w[2 * e], w[2 * e + 1]);
                    if constexpr (decltype(low)::value)
                        p = att_pack_bf16(w[2 * e] - __uint_as_float(p << 16), w[2 * e + 1] - __uint_as_float(p & 0xffff0000u));
                    out[u][e] = p;
                    lr = att_add_bf16(p, lr);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) out[2 * u + e / 4][e % 4] = __float_as_uint(w[e]);
            }
        }
    };
    // O^T += V^T P^T: operands, and their products
    struct Operands { v4u x[BF ? 2 * DT : 1]; };
    auto fetch = [&](const char* vb, int k) {
        Operands f;
        if constexpr (BF) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
                    const char* at = vb + vofs[d] + (k * 32 + 16 * u) * ROWB;
                    const v2u x0 = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)at));
                    const v2u x1 = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(at + 8 * ROWB)));
                    f.x[u * DT + d] = v4u{x0[0], x0[1], x1[0], x1[1]};
                }
        }
        return f;
    };
    auto values = [&](const Operands& f, const char* vb, const Packed& p, int k) {
        if constexpr (BF) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, f.x[u * DT + d]), __builtin_bit_cast(v8bf, p[u]), o[d], 0, 0, 0);
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const float x = *(const float*)(vb + vofs[d] + (k * 32 + (r & 3) + 8 * (r >> 2)) * ROWB);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, __uint_as_float(p[r / 4][r % 4]), o[d], 0, 0, 0);
                }
        }
    };
    // The maximum moves only when it is off by 2^8, which the fp32 sums and products hold as well; what was summed with the
    // old one follows.
    // (first: what has to be added with the old one before)
    auto raise = [&](const v16f& sc, auto first) {
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, sc[r]);
        top = half_max(top) * (GENERAL ? 1.f : a.c1);
        if (__builtin_expect(att_uniform(__any(top > m + 8.f)), 0)) {
            first();
            const float now = fmaxf(m, top);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= f;
            lr *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= f;
        }
    };

    // blocks t, t1, t2, t3 in turn: in work, copied, found, looked up
    int t = behind(from / BK - 1), t1 = t < end ? behind(t) : end, t2 = t1 < end ? behind(t1) : end;
    Key now{0, 0, -1}, next{0, 0, -1};                 // keys of t and t1
    Found far{0, 0, 0};                                // ... of t2, as loaded
    if (t < end) {
        const Found f0 = look(t), f1 = look(min(t1, end - 1));
        far = look(min(t2, end - 1));
        now = settle(f0, t);
        copy(now.at, 0);
        next = settle(f1, min(t1, end - 1));
    }
    constexpr int AHEAD = CS < 4 ? CS : 4;             // operands of the first product read ahead of it
    constexpr uint64_t ALL = BK == 64 ? ~0ull : (1ull << BK) - 1;
    for (int buf = 0; t < end; buf ^= 1) {
        const int j0 = t * BK, t3 = t2 < end ? behind(t2) : end;
        const char* const kb = ks + buf * S::TILE;
        const char* const vb = vs + buf * S::TILE;
        __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0): this wavefront's copies of the block are there
        bwla_lds_barrier();                            // ... everyone's are, and the other buffer is free
        Key after = next;
        if (t2 < end) after = settle(far, t2);
        if (t3 < end) far = look(t3);
        if (t1 < end) copy(next.at, buf ^ 1);
        // Even: every key exists and is of one document, and in reach of the windows, so that a row of that document sees those up
        // to its index, or all of the prefix.  Else each wavefront works out what each of its rows sees (a bit for each key), and
        // values of keys that no row of the workgroup sees are cleared: they may be anything, and a weight of 0 does not make 0
        // of that.
        const int doc = __builtin_amdgcn_readfirstlane(now.doc);
        const bool even = doc >= 0 && att_uniform(__all(now.doc == doc) &&
                                                  (a.window == INT32_MAX || (!s.pos && j0 > g_last - a.window) || j0 + BK <= s.prefix));
        const bool mine = me.doc == doc;
        uint64_t ok = ALL, any = ALL;
        if (__builtin_expect(!even, 0)) {
            ok = att_seen(a, s, me, j0, now.p, now.doc) & ALL;
            any = att_rows_or(ok);
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
        if (att_uniform(even ? __any(mine) && (j0 <= w_last || j0 < s.prefix) : any != 0)) {
            // every row sees every key
            const bool whole = even && att_uniform(__all(mine | blind)) && (j0 + BK - 1 <= w_first || j0 + BK <= s.prefix);
            // a tile's scores made ready: cap, bias, mask, and a maximum that will do for them
            auto ready = [&](v16f& sc, int k, auto first) {
                if constexpr (GENERAL) att_transform<FORM>(a, sc, me.p, slope, j0, k, now.p, s.pos != nullptr);
                bool fine = false;
                if (__builtin_expect(whole, 1)) {
                    had += 16;
                } else {
                    if (even) {
                        const int most = (mine ? max(me.i, s.prefix - 1) : -1) - j0 - k * 32 - 4 * hf;
#pragma unroll
                        for (int r = 0; r < 16; ++r) sc[r] = (r & 3) + 8 * (r >> 2) <= most ? sc[r] : -INFINITY;
                        had += min(max((most & ~3) / 2 + 4, 0), 16);           // (four too many at most)
                    } else {
                        const uint32_t mine = (uint32_t)(ok >> (32 * k)) >> (4 * hf);
#pragma unroll
                        for (int r = 0; r < 16; ++r) sc[r] = (mine >> ((r & 3) + 8 * (r >> 2))) & 1 ? sc[r] : -INFINITY;
                        had += __popc(mine & 0x0f0f0f0fu);
                    }
                    fine = BF && att_uniform(__any(!blind & (had < FEW)));
                }
                raise(sc, first);
                if constexpr (BF) {
                    if (__builtin_expect(fine, 0)) {
                        Packed p;
                        weigh(sc, p, std::true_type{});
                        values(fetch(vb, k), vb, p, k);
                    }
                }
            };
            if constexpr (KT == 2) {
                // (Priority for what is mostly products over the other wavefronts' sums and copies: 832 -> 808 us.)
                // The weights of one tile are taken while the other's products run; operands are read ahead.  The compiler has to
                // be told: left to itself it reads each operand right in front of its product and waits (130 cycles each).
                v16f s0, s1;
                Packed p0, p1;
                __builtin_amdgcn_s_setprio(1);
                products(kb, 0, s0);
                __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
                for (int i = 0; i < CS - AHEAD; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
                __builtin_amdgcn_s_setprio(0);
                ready(s0, 0, [] {});
                __builtin_amdgcn_s_setprio(1);
                products(kb, 1, s1);
                weigh(s0, p0, std::false_type{});
                asm volatile("" : "+v"(p0[0]), "+v"(p0[1]), "+v"(l));          // (here, and not where they are used)
                __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 1);
#pragma unroll
                for (int i = 0; i < CS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                    if (i < CS - AHEAD) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
                    __builtin_amdgcn_sched_group_barrier(0x002, 72 / CS, 1);
                }
                __builtin_amdgcn_s_setprio(0);
                ready(s1, 1, [&] {
                    values(fetch(vb, 0), vb, p0, 0);
                    p0[0] = p0[1] = v4u{0, 0, 0, 0};
                });
                __builtin_amdgcn_s_setprio(1);
                const Operands f0 = fetch(vb, 0);
                __builtin_amdgcn_sched_barrier(0);
                values(f0, vb, p0, 0);
                weigh(s1, p1, std::false_type{});
#pragma unroll
                for (int i = 0; i < 2 * DT; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 2);
                    __builtin_amdgcn_sched_group_barrier(0x002, 72 / (2 * DT), 2);
                }
                const Operands f1 = fetch(vb, 1);
                __builtin_amdgcn_sched_barrier(0);
                values(f1, vb, p1, 1);
                __builtin_amdgcn_s_setprio(0);
            } else {
                v16f sc;
                Packed p;
                products(kb, 0, sc);
                ready(sc, 0, [] {});
                weigh(sc, p, std::false_type{});
                values(fetch(vb, 0), vb, p, 0);
            }
        }
        now = next;
        next = after;
        t = t1;
        t1 = t2;
        t2 = t3;
    }

    l = half_sum(l);
    lr = BF ? half_sum(lr) : l;
    if (blind) l = lr = 0.f;
    if (!live) return;
    if (!whole_length) {                               // in tiles of 16 rows, as the join reads them
        const int64_t to = ((int64_t)(unit * sp.row_tiles + row / 16) * sp.splits + split) * 16 + row % 16;
        if (hf == 0) stat[to] = make_float4(blind ? -INFINITY : att_part_max(m, l), l, lr, 0.f);
        if (m != -INFINITY) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *(float4*)(part + to * DP + 32 * d + 2 * r + 4 * hf) = make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
        }
        return;
    }
    const float over = att_over(l, lr);
    const int64_t at = (int64_t)(s.row0 + tok) * a.hq + head;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int c = 32 * d + 2 * r + 4 * hf;
            if (EXACT || c < a.d) att_put<BF>(a, at, c, make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]), over);
        }
    if (hf == 0) att_put_lse(a, at, m, l);
}

template <bool BF, int DP>
hipError_t at_launch(const AttArgs& a, const AttSplit& sp, void* ws, hipStream_t st) {
    const int tiles = (sp.rows + AT_ROWS - 1) / AT_ROWS;
    const int units = a.seqs * a.hkv;
    if ((int64_t)tiles * units * sp.splits >= 1 << 24) return hipErrorInvalidConfiguration;       // (a grid has fewer than 2^32 threads)
    const AtOrder order = at_order_of(tiles, units, sp.splits, DP == 256 ? 1 : 2);
    constexpr int lds = AtShape<BF, DP>::LDS;
    const int form = att_form(a, BF);
    const bool exact = a.d == DP;
    float* const part = (float*)ws;
    float4* const stat = (float4*)((char*)ws + sp.part_bytes);
    auto go = [&](auto kernel) {
        const hipError_t e = bwla_ensure_lds((const void*)kernel, lds);
        if (e != hipSuccess) return e;
        kernel<<<dim3((unsigned)((int64_t)tiles * units * sp.splits)), 64 * AT_WAVES, lds, st>>>(a, order, sp, part, stat);
        return hipGetLastError();
    };
    if (form == ATT_PLAIN) return exact ? go(att_tile_kernel<BF, DP, true, ATT_PLAIN>) : go(att_tile_kernel<BF, DP, false, ATT_PLAIN>);
    constexpr int SHORT = BF ? ATT_SHORT : ATT_LONG;
    if (form == SHORT) return exact ? go(att_tile_kernel<BF, DP, true, SHORT>) : go(att_tile_kernel<BF, DP, false, SHORT>);
    return exact ? go(att_tile_kernel<BF, DP, true, ATT_LONG>) : go(att_tile_kernel<BF, DP, false, ATT_LONG>);
}

}  // namespace
