// Attention over rows in 8 bits: what the decoding step and the prefill share.  The scales belong to rows, so the products take codes and the scales
// go to the scores and the probabilities:
//
//   score(key) = (q . k_codes) * s_k * scale,   out = sum_key p(key) s_v(key) v_codes / sum_key p(key)
//
//   * q . (k_codes + 1152): a code + 128 becomes an fp16 by putting 0x64 before its byte (1024 + byte: one permutation for two values);
//     the query is an fp16 after the power of two that brings its largest entry into [2^14, 2^15), which loses nothing down to 2^-28
//     of that entry and 2^-39 of it below; the sums start at -1152 sum q.
//   * p s_v in bf16 (8 bits, as P has over caches in bf16, and no limit to the size of V; the denominator sums p before that) times the codes
//     + 128 in bf16, which loses nothing, less 128 times the sum of p s_v, through one more product, with a matrix of -128.  With the rounding of the
//     output that is 2.3e-3 of a value on average over 16 ragged streams, where the output's rounding alone is 2.0e-3.  (The prefill
//     takes both as fp16: see its `weigh`.  A run's own probabilities are bf16 there too, as over caches in bf16.)
#pragma once
#include "vs_cache8.h"

namespace vs {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// (fmaxf of values that come out of a selection is three instructions for one)
__device__ __forceinline__ float max_of_8(const float (&z)[8]) {
    float a, b;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(z[0]), "v"(z[1]), "v"(z[2]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(b) : "v"(z[3]), "v"(z[4]), "v"(z[5]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(z[6]), "v"(z[7]), "v"(a));
    asm("v_max_f32 %0, %1, %2" : "=v"(a) : "v"(a), "v"(b));
    return a;
}

// four codes of V as bf16: whole numbers 0..255, whose fp32 has nothing in its lower half
__device__ __forceinline__ void widen(unsigned w, unsigned& lo, unsigned& hi) {
    const unsigned a = __float_as_uint((float)(w & 255u)), b = __float_as_uint((float)((w >> 8) & 255u));
    const unsigned c = __float_as_uint((float)((w >> 16) & 255u)), d = __float_as_uint((float)(w >> 24));
    lo = __builtin_amdgcn_perm(b, a, 0x07060302u);
    hi = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// four codes of K as fp16, 1152 too large
__device__ __forceinline__ void widen_key(unsigned w, unsigned& lo, unsigned& hi) {
    lo = __builtin_amdgcn_perm(0x64646464u, w, 0x05010400u);
    hi = __builtin_amdgcn_perm(0x64646464u, w, 0x07030602u);
}
__device__ __forceinline__ f16x8 keys_of(unsigned x, unsigned y) {
    u32x4 a;
    unsigned lo, hi;
    widen_key(x, lo, hi);
    a[0] = lo, a[1] = hi;
    widen_key(y, lo, hi);
    a[2] = lo, a[3] = hi;
    return __builtin_bit_cast(f16x8, a);
}
// 8 V codes + 128 as bf16
__device__ __forceinline__ bf16x8 values_of(unsigned x, unsigned y) {
    u32x4 a;
    unsigned lo, hi;
    widen(x, lo, hi);
    a[0] = lo, a[1] = hi;
    widen(y, lo, hi);
    a[2] = lo, a[3] = hi;
    return __builtin_bit_cast(bf16x8, a);
}

// The queries of a set of 16 columns: lane (column, h) holds dims 32 i + 8 h ...
struct Queries {
    f16x8 q[4];
    float start;  // what the sums over codes + 1152 start at
    float f;      // the factor of the scores
};
__device__ __forceinline__ Queries queries_of(const raw16 (&w)[4], float scale_log2e) {
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) most = max_pairs(most, w[i][j] & 0x7fff7fffu);
    most = max(most & 0xffffu, most >> 16);
    most = over_rows(most, [](unsigned a, unsigned b) { return max(a, b); });
    // (Up to 2^126, and no further than scale_log2e 2^-up is an fp32 with all its bits: at the scale of Eq. 1 2^123, which makes the
    // smallest bf16 2^-10, an fp16 like any other.  A smaller scale may hold up back further: 128 values of the query are then off by 2^(-25 - up) each
    // at most, which over the largest keys, 2^128, is 2^-15 of a score.)
    const int most_up = min((int)((__float_as_uint(scale_log2e) >> 23) & 255u) - 1, 126);
    const int up = min(14 + 127 - (int)(most >> 7), most_up);
    const float factor = __uint_as_float((unsigned)(127 + up) << 23);
    const unsigned minus1152 = 0xe480e480u;
    const f16x8 off = __builtin_bit_cast(f16x8, u32x4{minus1152, minus1152, minus1152, minus1152});
    f32x4 start = {0.f, 0.f, 0.f, 0.f};
    Queries out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned pair = w[i][j >> 1];
            out.q[i][j] = (_Float16)(__uint_as_float(j & 1 ? pair & 0xffff0000u : pair << 16) * factor);
        }
        start = __builtin_amdgcn_mfma_f32_16x16x32_f16(off, out.q[i], start, 0, 0, 0);
    }
    out.start = start[0];
    // (a query that is not finite gives scores that are not numbers)
    out.f = most > 0x7f7fu ? __uint_as_float(0x7fc00000u) : ldexpf(scale_log2e, -up);
    return out;
}

// x *= f in the registers where x is: written as products, the compiler gives the sums other registers behind the branch around
// them, and copies them on every turn.
__device__ __forceinline__ void scale_in_place(f32x4& x, float f) {
    float a = x[0], b = x[1], c = x[2], d = x[3];
    asm volatile("v_mul_f32 %0, %0, %4\n\tv_mul_f32 %1, %1, %4\n\tv_mul_f32 %2, %2, %4\n\tv_mul_f32 %3, %3, %4" : "+v"(a), "+v"(b), "+v"(c), "+v"(d) : "v"(f));
    x = f32x4{a, b, c, d};
}

}  // namespace vs
