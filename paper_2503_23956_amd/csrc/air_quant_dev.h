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

// Eight codes as a matrix operand: the low halves of bytes 0..3, then the high ones.  A byte below 16 read as e4m3 is its value times 2^-9 (an
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

}  // namespace air
