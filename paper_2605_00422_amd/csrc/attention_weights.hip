// Sums of softmax weights per cached token, from queries and the logarithms of their sums.
//
// A wavefront keeps the keys of 64 cached tokens (32 where a row is wide) in registers as the stationary operand and
// walks over the rows (new tokens times the query heads of a group): S^T = K Q^T on 32x32 MFMA, exp2(y - lse) in fp32, added up per
// lane.  The rows come by asynchronous copies to LDS, a step of 64 (fp32: 32) ahead, once for the four wavefronts (each loading
// its own: 159 -> 99 us below, with the registers that this frees).  Each cached token belongs to one wavefront, so there is nothing to join but the 32 lanes
// that share its rows, once, at the end, and no atomics.  Where there are few cached tokens for the rows, the rows
// are dealt out over workgroups whose sums a second launch adds in order.
// 64 new tokens of four sequences of 6000 to 16384, 64 heads of 8 groups of 128 columns: 84 us, 600 TFLOP/s; of a SIMD's cycles 60 %
// are vector instructions (fma, exponential, sum for each weight) and 30 % MFMA, 11 % both at once.  A cap: 173 us, above 128 213 (31
// registers more than there are).  61 fp32 rows a head: 11 us, a chain of loads and fp32 products, and 4 for the second launch.
#include "attention.h"

namespace {

constexpr int WT_WAVES = 4;
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

template <bool BF, int DP>
struct WtShape {
    static constexpr int ES = BF ? 2 : 4;
    static constexpr int KT = BF && DP <= 128 ? 2 : 1;                  // tiles of 32 keys of a wavefront
    static constexpr int KEYS = 32 * KT * WT_WAVES;                     // cached tokens of a workgroup
    static constexpr int RT = BF ? 2 : 1, ROWS = 32 * RT;               // tiles of rows, and rows, of a step
    static constexpr int ROWB = DP * ES, CH = ROWB / 16;                // bytes and 16-byte pieces of a row in LDS
    static constexpr int TILE = ROWS * ROWB;
    static constexpr int COPIES = ROWS * CH / (64 * WT_WAVES);
    static constexpr int LDS = 2 * TILE;
};

// FORM: AttForm, scale, cap and bias
template <bool BF, int DP, bool EXACT, int FORM>
__global__ __launch_bounds__(64 * WT_WAVES, BF ? (DP <= 128 ? 3 : 2) : DP == 256 ? 1 : 2) void att_weights_kernel(AttArgs a, int parts, int64_t pitch, float* __restrict__ sums) {
    using S = WtShape<BF, DP>;
    constexpr int ES = S::ES, KT = S::KT, RT = S::RT, ROWS = S::ROWS, CH = S::CH, CS = CH / 2, KSW = (CH < 16 ? CH : 16) - 1;
    constexpr bool GENERAL = FORM != ATT_PLAIN;
    extern __shared__ __align__(16) char qs[];          // [2][ROWS][ROWB], pieces of a row at piece ^ (row & KSW)
    const int lane = threadIdx.x & 63, wave = att_wave(), l32 = lane & 31, hf = lane >> 5;
    const int h = blockIdx.y, b = blockIdx.z / parts, part = blockIdx.z - b * parts;
    const AttSeq s = att_seq(a, b);
    const int g0 = blockIdx.x * S::KEYS, j0 = g0 + wave * 32 * KT;
    if (g0 >= s.n) return;
    const int rows = s.fresh * a.group, old = s.old;
    const int slot_mask = (1 << a.page_shift) - 1;

    v4u kf[KT][CS];
#pragma unroll
    for (int k = 0; k < KT; ++k) {
        const int j = min(j0 + k * 32 + l32, s.n - 1);
        const int p = s.table[j >> a.page_shift];
        const bool there = (unsigned)p < (unsigned)a.pages;
        const char* src = a.k + (int64_t)(there ? p : 0) * a.page_bytes + (int64_t)h * a.head_bytes + (int64_t)(j & slot_mask) * a.slot_bytes;
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            const int at = (2 * c + hf) * 16;
            kf[k][c] = EXACT || at < a.d * ES ? *(const v4u*)(src + at) : v4u{0, 0, 0, 0};
        }
    }
    // lane i knows key i; whether they are keys that every row from some index on sees (without documents, or with a window to keep
    // to: none)
    AttKey key;
    {
        const int j = j0 + (KT == 2 ? lane : l32);
        key = att_key(a, s, j, j < s.n && (unsigned)s.table[min(j, s.n - 1) >> a.page_shift] < (unsigned)a.pages);
    }
    const bool plain = att_uniform(__all(key.doc >= 0) & !s.doc & (a.window == INT32_MAX));
    float sum[16 * KT];
#pragma unroll
    for (int e = 0; e < 16 * KT; ++e) sum[e] = 0.f;

    // tokens that can see a key from j on, up to (not with) the one that sees none of `keys` of them; the workgroup's steps
    auto from_token = [&](int j) { return j < s.prefix ? 0 : max(j - old, 0); };
    auto to_token = [&](int j, int keys) {
        return !s.pos && a.window != INT32_MAX && j >= s.prefix ? (int)min((int64_t)s.fresh, (int64_t)j + keys - 1 + a.window - old) : s.fresh;
    };
    const int t0 = from_token(g0), t1 = to_token(g0, S::KEYS);
    const int first = t0 * a.group / ROWS, steps = t1 > t0 ? (t1 * a.group + ROWS - 1) / ROWS : 0;
    const int w_row0 = from_token(j0) * a.group, w_row1 = j0 < s.n ? to_token(j0, 32 * KT) * a.group : 0;
    const uint32_t magic = (uint32_t)((0x100000000ull + a.group - 1) / a.group);       // 2^32 / group (group 1: 0, and not used)
    auto token_of = [&](int row) {
        if (a.group == 1) return row;
        const int t = (int)__umulhi((uint32_t)row, magic);                             // at most one too many
        return t * a.group > row ? t - 1 : t;
    };
    const int head0 = h * a.group;
    auto head_of = [&](int row, int t) { return head0 + row - t * a.group; };

    const int piece = lane % CH, key0 = (wave * 64 + lane) / CH;
    const uint32_t lds0 = att_lds_address(qs + wave * 1024);
    auto copy = [&](int step, int buf) {               // (rows behind the last one: the last one's, which count for nothing)
        att_each(std::make_integer_sequence<int, S::COPIES>{}, [&](auto n) {
            constexpr int i = decltype(n)::value;
            const int r = key0 + i * (WT_WAVES * 64 / CH), row = min(step * ROWS + r, rows - 1), t = token_of(row);
            const char* src = a.q + (int64_t)(s.row0 + t) * a.q_bytes + (int64_t)head_of(row, t) * a.d * ES;
            const int at = (piece ^ (r & KSW)) * 16;
            if (EXACT || at < a.d * ES) att_copy16<i * WT_WAVES * 1024>(src + at, lds0 + buf * S::TILE);
        });
    };
    if constexpr (!EXACT) {                            // columns that no copy fills count as zero
        for (int i = threadIdx.x; i < 2 * ROWS * CH; i += 64 * WT_WAVES)
            if ((i % CH ^ (i / CH & KSW)) * 16 >= a.d * ES) *(v4u*)(qs + i * 16) = v4u{0, 0, 0, 0};
    }
    struct Rows {
        float lse[RT];                                 // in base 2, +inf where the row sees nothing: its weights are 0
    };
    auto look = [&](int step) {
        Rows x;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = step * ROWS + r * 32 + l32, in = min(row, rows - 1), t = token_of(in);
            const float lse = a.lse[(int64_t)(s.row0 + t) * a.hq + head_of(in, t)];
            x.lse[r] = row < rows ? lse : -INFINITY;
        }
        return x;
    };
    int step = first + (part - first % parts + parts) % parts;
    Rows next;
    if (step < steps) {
        copy(step, 0);
        next = look(step);
    }
    for (int buf = 0; step < steps; step += parts, buf ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0): this wavefront's copies of the step are there
        bwla_lds_barrier();                            // ... everyone's are, and the other buffer is free
        const Rows x = next;
        if (step + parts < steps) {
            copy(step + parts, buf ^ 1);
            next = look(step + parts);
        }
#pragma unroll 1
        for (int r = 0; r < RT; ++r) {
            const int row0 = step * ROWS + r * 32;
            if (att_uniform(row0 + 31 < w_row0 || row0 >= w_row1)) continue;
            float lse = (RT == 2 && r ? x.lse[RT - 1] : x.lse[0]) * ATT_LOG2E;
            lse = lse == -INFINITY ? INFINITY : lse;
            const char* src = qs + buf * S::TILE + (r * 32 + l32) * S::ROWB;
            const int first_i = old + token_of(row0);
            const bool whole = plain & ((first_i >= j0 + 32 * KT - 1) | ((first_i >= 0) & (j0 + 32 * KT <= s.prefix)));
            v16f p[KT];
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e) p[k][e] = 0.f;
#pragma unroll
            for (int c = 0; c < CS; ++c) {
                if constexpr (!BF) {                   // (or all would be read ahead, into registers that there are not)
                    if (c % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                }
                const v4u q = *(const v4u*)(src + ((2 * c + hf) ^ (l32 & KSW)) * 16);
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    if constexpr (BF) {
                        p[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, kf[k][c]), __builtin_bit_cast(v8bf, q), p[k], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            p[k] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[k][c][e]), __uint_as_float(q[e]), p[k], 0, 0, 0);
                    }
                }
            }
            AttRow me{0, 0, 0};
            if (GENERAL || !whole) {
                const int row = row0 + l32, in = min(row, rows - 1), tok = token_of(in);
                me = att_row(s, tok, row < rows);
                if constexpr (GENERAL) {
                    const float slope = a.slopes ? a.slopes[head_of(in, tok)] * ATT_LOG2E : 0.f;
#pragma unroll
                    for (int k = 0; k < KT; ++k) att_transform<FORM>(a, p[k], me.p, slope, j0, k, key.p, s.pos != nullptr);
                }
            }
            if (__builtin_expect(!att_uniform(whole), 0)) {
                const uint64_t ok = att_seen(a, s, me, j0, key.p, key.doc);
#pragma unroll
                for (int k = 0; k < KT; ++k) {
                    const uint32_t mine = (uint32_t)(ok >> (32 * k)) >> (4 * hf);
#pragma unroll
                    for (int e = 0; e < 16; ++e) p[k][e] = (mine >> ((e & 3) + 8 * (e >> 2))) & 1 ? p[k][e] : -INFINITY;
                }
                // a row whose sum is NaN makes NaN of what it sees, and of nothing else
                if (__builtin_expect(att_uniform(__any(lse != lse)), 0)) {
#pragma unroll
                    for (int k = 0; k < KT; ++k)
#pragma unroll
                        for (int e = 0; e < 16; ++e) p[k][e] = lse != lse && p[k][e] != -INFINITY ? lse : p[k][e];
                    lse = lse != lse ? INFINITY : lse;
                }
            }
            const float c1 = GENERAL ? 1.f : a.c1;
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[k * 16 + e] += __builtin_amdgcn_exp2f(fmaf(p[k][e], c1, -lse));
        }
    }
    if (j0 >= s.n) return;
    // the 32 lanes' sums: each step halves what a lane holds, so that lane l32 ends with accumulator l32
    if constexpr (KT == 2) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float give = l32 & 16 ? sum[e] : sum[e + 16], mine = l32 & 16 ? sum[e + 16] : sum[e];
            sum[e] = mine + __shfl_xor(give, 16, 64);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] += __shfl_xor(sum[e], 16, 64);
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1)
#pragma unroll
        for (int e = 0; e < off; ++e) {
            const float give = l32 & off ? sum[e] : sum[e + off], mine = l32 & off ? sum[e + off] : sum[e];
            sum[e] = mine + __shfl_xor(give, off, 64);
        }
    const int r = l32 & 15, j = j0 + (KT == 2 ? (l32 >> 4) * 32 : 0) + (r & 3) + 8 * (r >> 2) + 4 * hf;
    if (j >= s.n || (KT == 1 && l32 >= 16)) return;
    if (parts > 1) {
        sums[(((int64_t)b * parts + part) * a.hkv + h) * pitch + j] = sum[0];
    } else {
        const int p = s.table[j >> a.page_shift];
        if ((unsigned)p < (unsigned)a.pages) a.weights[(((int64_t)p * a.hkv + h) << a.page_shift) + (j & slot_mask)] += sum[0];
    }
}

__global__ __launch_bounds__(256) void att_weights_add_kernel(AttArgs a, int parts, int64_t pitch, const float* __restrict__ sums) {
    const int j = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
    const AttSeq s = att_seq(a, b);
    if (j >= s.n) return;
    const int p = s.table[j >> a.page_shift];
    if ((unsigned)p >= (unsigned)a.pages) return;
    float sum = 0.f;
    for (int i = 0; i < parts; ++i) sum += sums[(((int64_t)b * parts + i) * a.hkv + h) * pitch + j];
    a.weights[(((int64_t)p * a.hkv + h) << a.page_shift) + (j & ((1 << a.page_shift) - 1))] += sum;
}

template <bool BF, int DP>
hipError_t launch(const AttArgs& a, int parts, void* ws, hipStream_t st) {
    constexpr int keys = WtShape<BF, DP>::KEYS, lds = WtShape<BF, DP>::LDS;
    const int64_t pitch = (a.max_len + 31) & ~31;
    const dim3 grid((a.max_len + keys - 1) / keys, a.hkv, a.seqs * parts);
    auto go = [&](auto kernel) {
        const hipError_t e = bwla_ensure_lds((const void*)kernel, lds);
        if (e != hipSuccess) return e;
        kernel<<<grid, 64 * WT_WAVES, lds, st>>>(a, parts, pitch, (float*)ws);
        return hipGetLastError();
    };
    constexpr int SHORT = BF ? ATT_SHORT : ATT_LONG;
    const int form = att_form(a, BF);
    hipError_t e;
    if (form == ATT_PLAIN) e = a.d == DP ? go(att_weights_kernel<BF, DP, true, ATT_PLAIN>) : go(att_weights_kernel<BF, DP, false, ATT_PLAIN>);
    else if (form == SHORT) e = a.d == DP ? go(att_weights_kernel<BF, DP, true, SHORT>) : go(att_weights_kernel<BF, DP, false, SHORT>);
    else e = a.d == DP ? go(att_weights_kernel<BF, DP, true, ATT_LONG>) : go(att_weights_kernel<BF, DP, false, ATT_LONG>);
    if (e != hipSuccess) return e;
    if (parts > 1) att_weights_add_kernel<<<dim3((a.max_len + 255) / 256, a.hkv, a.seqs), 256, 0, st>>>(a, parts, pitch, (const float*)ws);
    return hipGetLastError();
}

}  // namespace

AttWeightsPlan bwla_att_weights_plan(const AttArgs& a, int dtype) {
    const bool bf = dtype == BWLA_X_BF16;
    const int64_t keys = (bf && a.d <= 128 ? 2 : 1) * 32 * WT_WAVES;
    const int64_t groups = (a.max_len + keys - 1) / keys * a.hkv * a.seqs;
    const int64_t steps = ((int64_t)a.max_new * a.group + (bf ? 63 : 31)) / (bf ? 64 : 32);
    // parts until there are two workgroups a compute unit, of two steps at least, one in fp32
    int64_t parts = (512 + groups - 1) / groups;
    const int64_t most = bf ? steps / 2 : steps;
    if (parts > most) parts = most;
    if (parts > 65535 / a.seqs) parts = 65535 / a.seqs;
    AttWeightsPlan p;
    p.parts = parts < 1 ? 1 : (int)parts;
    p.bytes = p.parts > 1 ? (size_t)a.seqs * p.parts * a.hkv * ((a.max_len + 31) & ~31) * 4 : 0;
    return p;
}

hipError_t bwla_launch_attention_weights(const AttArgs& a, int dtype, void* ws, hipStream_t st) {
    const int parts = bwla_att_weights_plan(a, dtype).parts;
    if (dtype == BWLA_X_BF16) {
        if (a.d <= 64) return launch<true, 64>(a, parts, ws, st);
        if (a.d <= 128) return launch<true, 128>(a, parts, ws, st);
        return launch<true, 256>(a, parts, ws, st);
    }
    if (a.d <= 64) return launch<false, 64>(a, parts, ws, st);
    if (a.d <= 128) return launch<false, 128>(a, parts, ws, st);
    return launch<false, 256>(a, parts, ws, st);
}
