// The 4-bit format of K and V rows on the device: what a code stands for, matrix operands out of codes, floats as sums of bf16 terms.
//
// Codes are whole numbers 0..15, exact in bf16, so that products of codes are products of small exact numbers:
//   q . k          = sum over groups g of  step_g (q . code)_g + lo_g sum(q)_g
//   sum_j p_j v_jc = sum_j (p_j step_jg) code_jc + sum_j p_j lo_jg
// and fp32 factors enter as sums of two or three bf16 terms.
#pragma once

#include "air_tile.h"

namespace air {

typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// (lo, step) of a group, as held
__device__ __forceinline__ float lo_of(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float step_of(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

// Eight codes as a matrix operand, halves of bytes in the order 0 2 4 6 1 3 5 7 (half 2 i: the low one of byte i).  A byte below 16 read as e4m3 is its value times 2^-9 (an
// eighth's steps of 2^-6, below and above the least normal number alike), so that the conversion with a scale of 2^9 is exact.
__device__ __forceinline__ uint4 operand_of(uint32_t codes) {
    const uint32_t lo = codes & 0x0f0f0f0fu, hi = (codes >> 4) & 0x0f0f0f0fu;
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true));
    return r;
}

// Eight codes of K as the bf16 numbers 16 + code, elements in order: a code three bits up in the mantissa of 16.  Eight full-rate instructions where
// the exact conversion takes three and four of half the rate; what the product has too much, 16 sum(q), is taken off by the product with
// the sums.
constexpr float kCodeBias = 16.0f;
__device__ __forceinline__ uint4 biased_of(uint32_t codes) {
    uint4 r;
    r.x = (codes << 3 & 0x00780078u) | 0x41804180u;
    r.y = (codes >> 1 & 0x00780078u) | 0x41804180u;
    r.z = (codes >> 5 & 0x00780078u) | 0x41804180u;
    r.w = (codes >> 9 & 0x00780078u) | 0x41804180u;
    return r;
}
// bit of code i in a dword of eight: V in order; K in the order of biased_of
template <bool K>
__device__ __forceinline__ int code_shift(int i) {
    return K ? 4 * (i >> 1) + 16 * (i & 1) : 4 * i;
}

// Two floats as TERMS packed pairs of bf16 whose sum they are: all terms but the last cut off behind eight bits, so that three are exact and
// two lose 2^-17 of the value
template <int TERMS>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&t)[TERMS]) {
#pragma unroll
    for (int i = 0; i + 1 < TERMS; ++i) {
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        t[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        a -= __uint_as_float(x & 0xffff0000u);
        b -= __uint_as_float(y & 0xffff0000u);
    }
    const bf16x2 last = {(__bf16)a, (__bf16)b};
    t[TERMS - 1] = __builtin_bit_cast(uint32_t, last);
}

// ---- rows: a lane has eight elements
__device__ __forceinline__ void load8(const bf16_t *p, float (&x)[8]) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = a[i];
        x[4 + i] = b[i];
    }
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&x)[8]) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
    *reinterpret_cast<uint4 *>(p) = __builtin_bit_cast(uint4, v);
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
    *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// least and greatest that a NaN passes
__device__ __forceinline__ float least_of(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float most_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// over the 4 (LANES = 4) or 8 consecutive lanes of a group
template <int LANES>
__device__ __forceinline__ void range_of(float &low, float &high) {
    low = AIR_DPP_STEP(least_of, low, 0xB1);
    high = AIR_DPP_STEP(most_of, high, 0xB1);
    low = AIR_DPP_STEP(least_of, low, 0x4E);
    high = AIR_DPP_STEP(most_of, high, 0x4E);
    if (LANES == 8) {
        low = AIR_DPP_STEP(least_of, low, 0x141);
        high = AIR_DPP_STEP(most_of, high, 0x141);
    }
}

// a / b rounded correctly, out of 1 / b rounded correctly: the product, mended once by what it leaves (Markstein)
__device__ __forceinline__ float quotient(float a, float b, float inv) {
    const float q = a * inv;
    return fmaf(fmaf(-q, b, a), inv, q);
}
// 1 / b rounded correctly, for b of eight significant bits in 2^-120 .. 2^124: the hardware's reciprocal, off by at most one step, mended once (all
// 128 mantissas are tested)
__device__ __forceinline__ float reciprocal(float b) {
    const float y = __builtin_amdgcn_rcpf(b);
    return fmaf(fmaf(-b, y, 1.0f), y, y);
}

// (lo, step) of a group from its least and greatest element
__device__ __forceinline__ uint32_t pair_of(float low, float high) {
    if (!(most_of(-low, high) < 0x1p126f)) return 0x7fc0u;  // NaN, step 0
    const uint32_t u = __float_as_uint(low);
    const uint32_t lo = (u + (u >> 31 ? 0xffffu : 0u)) & 0xffff0000u;  // down: away from zero below it
    const float width = quotient(high - __uint_as_float(lo), 15.0f, 1.0f / 15.0f);
    const uint32_t step = (__float_as_uint(width) + 0xffffu) & 0xffff0000u;
    return (__uint_as_float(step) < 0x1p-120f ? 0u : step) | lo >> 16;
}

// which dword of a row holds elements 8 p .. 8 p + 7
template <int D, bool K>
__device__ __forceinline__ int dword_of(int p) {
    return K ? D / 32 * (p & 3) + (p >> 2) : p;
}

// eight elements as codes; pair: (lo, step) of their group
template <int GR, bool K>
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], uint32_t &pair) {
    float low = x[0], high = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        low = least_of(low, x[i]);
        high = most_of(high, x[i]);
    }
    range_of<GR / 8>(low, high);
    pair = pair_of(low, high);
    const float lo = lo_of(pair), step = step_of(pair), inv = step > 0.0f ? reciprocal(step) : 0.0f;
    // a quotient of 0 .. 15 (15 (1 + 2^-22) at most, as the step is no less than a fifteenth of the width but for its rounding) plus 1.5 2^23
    // has its nearest whole number, ties to even, in its last bits; eight of them shifted and added leave a constant too much
    constexpr uint32_t kBase = 0x4b400000u;
    uint32_t code = 0, excess = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = quotient(x[i] - lo, step, inv) + 0x1.8p23f;
        code += __float_as_uint(s) << code_shift<K>(i);
        excess += kBase << code_shift<K>(i);
    }
    return step > 0.0f ? code - excess : 0u;
}
template <int D, int GR, typename T, bool K>
__device__ __forceinline__ void append_row(const T *src, uint32_t *codes, uint32_t *scales, int p) {
    float x[8];
    load8(src + 8 * p, x);
    uint32_t pair;
    codes[dword_of<D, K>(p)] = codes_of<GR, K>(x, pair);
    if ((p & (GR / 8 - 1)) == 0) scales[p / (GR / 8)] = pair;
}

template <int D, int GR, typename T, bool K>
__device__ __forceinline__ void read_row(T *dst, const uint32_t *codes, const uint32_t *scales, int p) {
    const uint32_t code = codes[dword_of<D, K>(p)], pair = scales[p / (GR / 8)];
    const float lo = lo_of(pair), step = step_of(pair);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(step, (float)(code >> code_shift<K>(i) & 15u), lo);
    store8(dst + 8 * p, x);
}

}  // namespace air
