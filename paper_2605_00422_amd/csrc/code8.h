// The 8-bit codes of a cache: integers -127 .. 127, and e4m3 numbers (no infinities, 448 the largest, 0x7f and 0xff NaN).
#pragma once
#include "attention.h"

typedef uint32_t c8_v4u __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

template <bool I8>
__device__ __forceinline__ constexpr float code_top() { return I8 ? 127.f : 448.f; }

// four numbers within the codes' range to the nearest codes, ties to even
template <bool I8>
__device__ __forceinline__ uint32_t code_of4(float a, float b, float c, float d) {
    if constexpr (I8) {
        return ((uint32_t)(int)rintf(a) & 0xffu) | ((uint32_t)(int)rintf(b) & 0xffu) << 8 | ((uint32_t)(int)rintf(c) & 0xffu) << 16 |
               (uint32_t)(int)rintf(d) << 24;
    } else {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    }
}
// ... and one
template <bool I8>
__device__ __forceinline__ uint8_t code_of(float a) { return (uint8_t)code_of4<I8>(a, 0.f, 0.f, 0.f); }

// code number I of a word
template <bool I8, int I>
__device__ __forceinline__ float code_value(uint32_t w) {
    if constexpr (I8) return (float)(int8_t)(w >> (8 * I));
    else return __builtin_amdgcn_cvt_f32_fp8((int)w, I);
}

// Four codes as fp16 numbers, exactly, in order.  An e4m3 number is one by the conversion; an integer c by the number of bits
// 0x6400 + (c + 128), which is 1024 + c + 128, less 1152.
struct Halves {
    uint32_t lo, hi;
};
template <bool I8>
__device__ __forceinline__ Halves code_halves(uint32_t w) {
    Halves r;
    if constexpr (I8) {
        const uint32_t u = w ^ 0x80808080u;
        const v2h less = {(_Float16)-1152.f, (_Float16)-1152.f};
        r.lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + less);
        r.hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + less);
    } else {
        r.lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
        r.hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true));
    }
    return r;
}

// Eight numbers as operands: the nearest of fp16, and (two terms) what that leaves.  (The number that is taken off has to be the one that is
// kept: the compiler would make the first term of a product without rounding that to fp32 first, but the second of the rounded one,
// and near ties the two would not belong together.  So each is held in registers before its terms are made.)
template <int T>
struct Terms {
    v8h t[T];
};
template <int T>
__device__ __forceinline__ Terms<T> terms_of(const float* from) {
    Terms<T> r;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = from[e];
        if constexpr (T == 2) asm("" : "+v"(x[e]));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) r.t[0][e] = (_Float16)x[e];
    if constexpr (T == 2) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.t[1][e] = (_Float16)(x[e] - (float)r.t[0][e]);
    }
    return r;
}

// whether any lane has it: a scalar, so that what depends on it is a jump
__device__ __forceinline__ bool some(bool x) { return __builtin_amdgcn_ballot_w64(x) != 0; }
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, |%1|, |%2|, |%3|" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// N products (of a tile or a step) into capped scores.  Where none of a wavefront's is beyond 0.6 of the cap, which is the rule, the polynomial that
// att_tanh takes there alone (the same number: what unseen keys hold decides nothing; 2048 rows with a cap above 128: 120 -> 108 us).
template <int N, typename X>
__device__ __forceinline__ void capped_scores(const AttArgs& a, X& x) {
    float far = 0.f;
#pragma unroll
    for (int i = 0; i < N; i += 2) far = max3_abs(far, x[i], x[i + 1]);
    if (__builtin_expect(!some(far * a.c2 >= ATT_NEAR), 1)) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = a.capped * att_tanh_near(x[i] * a.c2);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = a.capped * att_tanh(x[i] * a.c2);
    }
}
