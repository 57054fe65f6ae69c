// Sums of softmax weights per cached token, from queries and the logarithms of their sums.
//
// A wavefront keeps the keys of 64 cached tokens (32 where a row is wide) in registers as the stationary operand and
// walks over the rows (new tokens times the query heads of a group), 32 a step: S^T = K Q^T on 32x32 MFMA, exp2(y - lse)
// in fp32, added up per lane.  Each cached token belongs to one wavefront, so there is nothing to join but the 32 lanes
// that share its rows, once, at the end, and no atomics.  Where there are few cached tokens for the rows, the rows
// are dealt out over workgroups whose sums a second launch adds in order.
#include "attention.h"

namespace {

constexpr int WT_WAVES = 4;
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

template <bool BF, int DP>
struct WtShape {
    static constexpr int KT = (BF ? DP : 2 * DP) > 256 ? 1 : 2;        // tiles of 32 keys of a wavefront
    static constexpr int KEYS = 32 * KT * WT_WAVES;                     // cached tokens of a workgroup
};

template <bool BF, int DP, bool EXACT>
__global__ __launch_bounds__(64 * WT_WAVES, DP * (BF ? 1 : 2) > 128 ? 1 : 2) void att_weights_kernel(AttArgs a, int parts, int64_t pitch, float* __restrict__ sums) {
    constexpr int ES = BF ? 2 : 4, CH = DP * ES / 16, KT = WtShape<BF, DP>::KT;
    const int lane = threadIdx.x & 63, wave = att_wave(), l32 = lane & 31, hf = lane >> 5;
    const int h = blockIdx.y, b = blockIdx.z / parts, part = blockIdx.z - b * parts;
    const AttSeq s = att_seq(a, b);
    const int j0 = (blockIdx.x * WT_WAVES + wave) * 32 * KT;
    if (j0 >= s.n) return;                             // (no barrier in this kernel)
    const int rows = s.fresh * a.group, old = s.n - s.fresh;
    const int slot_mask = (1 << a.page_shift) - 1;

    v4u kf[KT][CH / 2];
    AttKey key[KT];                                    // lane l32 knows key l32 of each tile
    bool all = true;
#pragma unroll
    for (int k = 0; k < KT; ++k) {
        const int j = min(j0 + k * 32 + l32, s.n - 1);
        const int p = s.table[j >> a.page_shift];
        const bool there = (unsigned)p < (unsigned)a.pages;
        const char* src = a.k + (int64_t)(there ? p : 0) * a.page_bytes + (int64_t)h * a.head_bytes + (int64_t)(j & slot_mask) * a.slot_bytes;
#pragma unroll
        for (int c = 0; c < CH / 2; ++c) {
            const int at = (2 * c + hf) * 16;
            kf[k][c] = EXACT || at < a.d * ES ? *(const v4u*)(src + at) : v4u{0, 0, 0, 0};
        }
        key[k] = att_key(a, s, j0 + k * 32 + l32, there);
        all &= key[k].doc >= 0;
    }
    // keys that every row from some index on sees (without documents, or with a window to keep to: none)
    const bool plain = att_uniform(__all(all) & !s.doc & (a.window == INT32_MAX));
    float sum[16 * KT];
#pragma unroll
    for (int e = 0; e < 16 * KT; ++e) sum[e] = 0.f;

    // tokens that can see a key of this wavefront
    int t0 = j0 < s.prefix ? 0 : max(j0 - old, 0), t1 = s.fresh;
    if (!s.pos && a.window != INT32_MAX && j0 >= s.prefix) t1 = (int)min((int64_t)t1, (int64_t)j0 + 32 * KT - 1 + a.window - old);
    const int first = t0 * a.group / 32, tiles = t1 > t0 ? (t1 * a.group + 31) / 32 : 0;
    // (from the part's first tile at or behind `first`)
    struct Tile {
        v4u q[CH / 2];
        float lse, slope;                              // lse in base 2, +inf where the row sees nothing: its weights are 0
        int tok;
        bool live;
    };
    auto fetch = [&](int tile) {
        Tile x;
        const int row = tile * 32 + l32;
        x.live = row < rows;
        x.tok = x.live ? row / a.group : 0;
        const int head = h * a.group + (x.live ? row - x.tok * a.group : 0);
        const int64_t at = (int64_t)(s.row0 + x.tok);
        const float lse = a.lse[at * a.hq + head] * ATT_LOG2E;
        x.lse = x.live & (lse != -INFINITY) ? lse : INFINITY;
        x.slope = a.slopes ? a.slopes[head] * ATT_LOG2E : 0.f;
        const char* qp = a.q + at * a.q_bytes + (int64_t)head * a.d * ES;
#pragma unroll
        for (int c = 0; c < CH / 2; ++c) {
            const int col = (2 * c + hf) * 16;
            x.q[c] = EXACT || col < a.d * ES ? *(const v4u*)(qp + col) : v4u{0, 0, 0, 0};
        }
        return x;
    };
    int tile = first + (part - first % parts + parts) % parts;
    Tile next;
    if (tile < tiles) next = fetch(tile);
    for (; tile < tiles; tile += parts) {
        const Tile x = next;
        if (tile + parts < tiles) next = fetch(tile + parts);
        const auto& qf = x.q;
        const float lse = x.lse, slope = x.slope;
        const int first_i = old + tile * 32 / a.group;
        const bool whole = plain & ((first_i >= j0 + 32 * KT - 1) | (j0 + 32 * KT <= s.prefix));
        AttRow me{0, 0, 0};
        if (!whole || a.slopes) me = att_row(s, x.tok, x.live);
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            v16f p;
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] = 0.f;
#pragma unroll
            for (int c = 0; c < CH / 2; ++c) {
                if constexpr (BF) {
                    p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, kf[k][c]), __builtin_bit_cast(v8bf, qf[c]), p, 0, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        p = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[k][c][e]), __uint_as_float(qf[c][e]), p, 0, 0, 0);
                }
            }
            if (a.capped != 0.f) {
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] = a.capped * att_tanh(p[r] * a.c2);
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] *= a.c1;
            }
            if (!whole || a.slopes) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int from = (r & 3) + 8 * (r >> 2) + 4 * hf;
                    const int kp = __shfl(key[k].p, from, 64), kd = __shfl(key[k].doc, from, 64);
                    p[r] = att_sees(me, s.prefix, a.window, j0 + k * 32 + from, kp, kd) ? p[r] - slope * fabsf((float)(me.p - kp)) : -INFINITY;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[k * 16 + r] += __builtin_amdgcn_exp2f(p[r] - lse);
        }
    }
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
    constexpr int keys = WtShape<BF, DP>::KEYS;
    const int64_t pitch = (a.max_len + 31) & ~31;
    const dim3 grid((a.max_len + keys - 1) / keys, a.hkv, a.seqs * parts);
    if (a.d == DP) att_weights_kernel<BF, DP, true><<<grid, 64 * WT_WAVES, 0, st>>>(a, parts, pitch, (float*)ws);
    else att_weights_kernel<BF, DP, false><<<grid, 64 * WT_WAVES, 0, st>>>(a, parts, pitch, (float*)ws);
    if (parts > 1) att_weights_add_kernel<<<dim3((a.max_len + 255) / 256, a.hkv, a.seqs), 256, 0, st>>>(a, parts, pitch, (const float*)ws);
    return hipGetLastError();
}

}  // namespace

AttWeightsPlan bwla_att_weights_plan(const AttArgs& a, int dtype) {
    const int wide = dtype == BWLA_X_BF16 ? a.d : 2 * a.d;
    const int64_t keys = (wide > 256 ? 1 : 2) * 32 * WT_WAVES;
    const int64_t groups = (a.max_len + keys - 1) / keys * a.hkv * a.seqs;
    const int64_t tiles = ((int64_t)a.max_new * a.group + 31) / 32;
    // parts until there are two workgroups a compute unit, of four steps at least (0.4 us each at 128 columns), one in
    // fp32 (3.5 us)
    int64_t parts = (512 + groups - 1) / groups;
    const int64_t most = dtype == BWLA_X_BF16 ? tiles / 4 : tiles;
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
