// Products of 32 x 32 tiles, key tiles in LDS and the exponentials of the kernels that attend with many rows.
#pragma once

#include "air_tile.h"

namespace air {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

// A tile of 32 keys in LDS, in units of 16 bytes.  LDS serves 256 bytes at a time (64 banks of 4 bytes): both layouts put what one
// instruction of a wave reads side by side, so that the reads of a tile differ by constants only, and the pieces of a row that 16 lanes
// store together into different banks.
template <typename T, int D>
struct Row {
    static constexpr int kVec = Elem<T>::kVec, kPieces = D / kVec;  // 16-byte pieces of a row
    static constexpr int kSlices = kPieces / 2;                     // slices of the contraction: two pieces, one per half of a wave
    // K: [piece][row]: lane (n, h) reads piece h of a slice of row n
    static constexpr int kPiece = 32 + (kPieces == 8 ? 2 : 1);
    // V: [32 columns][row][column].  bf16 is read transposed, 32 bytes of rows r and r + 4 together (lanes 0..15 and 32..47): the halves of
    // rows 4..7 of every eight change places.  fp32 is read as 128 bytes of row r (lanes 0..31) and of row r + 4 (lanes 32..63):
    // neighbours
    static constexpr int kBlock = sizeof(T) == 2 ? (kPieces == 8 ? 136 : 132) : 264;
    static constexpr int kKTile = kPieces * kPiece, kVTile = D / 32 * kBlock;
    static __device__ __forceinline__ int k_at(int r, int p) { return p * kPiece + r; }
    static __device__ __forceinline__ int v_at(int r, int p) {
        if (sizeof(T) == 2) return (p >> 2) * kBlock + 4 * r + ((p & 3) ^ ((r >> 1) & 2));
        return (p >> 3) * kBlock + 8 * ((r & 24) | (r & 3) << 1 | (r >> 2 & 1)) + (p & 7);
    }
};

__device__ __forceinline__ f32x16 mma32(const uint4 &a, const uint4 &b, f32x16 acc, bf16_t) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(const uint4 &a, const uint4 &b, f32x16 acc, float) {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
    return acc;
}

// the eight bf16 numbers of x added to sum
__device__ __forceinline__ float sum_of(const uint4 &x, float sum) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i]), one, sum, false);
    return sum;
}
__device__ __forceinline__ float largest(const f32x16 &s) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    return mx;
}
// orders the LDS accesses of the lanes of one wave
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Factor that brings sums of the reference m to the reference top >= m; no logit but -inf: 0.  Sums of weight 0 are taken along, not left out:
// a value that is not finite, at a key whose weight is 0, makes its column no number wherever its key lies.
__device__ __forceinline__ float weight(float m, float top) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top); }

// s * c rounded, less the reference (two operations, not one)
__device__ __forceinline__ float rounded_exponent(float s, float c, float ref) {
#pragma clang fp contract(off)
    const float x = s * c;
    return x - ref;
}

// The reference is a rounded product, the exponent an exact one minus it: the largest logit's exponent is off zero by half a step of the
// reference, the same for all keys of the row, so that it cancels.  Beyond kHuge (no trained model's logits) that step leaves fp32's
// range of exponents: there the product is rounded as the reference was.
constexpr float kHuge = 0x1p26f;
constexpr float kSlack = 8.0f;  // probabilities may be as large as 2^8: fp32 sums and bf16 operands hold them without loss

// Operand V^T of output tile d for the keys 16 half .. 16 half + 15 of a tile, in the order that the logits' registers have: the transposed
// read gives a lane four keys of a column; its address is that of row (lane % 16) / 4 of them, 8 bytes at columns
// 16 ((lane / 16) % 2) + 4 (lane % 4).
__device__ __forceinline__ int v_lane(int lane) {
    return 64 * (4 * (lane >> 5) + ((lane & 15) >> 2)) + 32 * (((lane >> 4) ^ (lane >> 5)) & 1) + 8 * (lane & 3);
}
template <int D>
__device__ __forceinline__ uint4 read_v(const u32x4 *sv, int lane_bytes, int half, int d) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const char *at = reinterpret_cast<const char *>(sv) + lane_bytes + 16 * Row<bf16_t, D>::kBlock * d + 1024 * half;
    struct { s16x4 a, b; } v;
    v.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
    v.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 512));  // eight rows on
    return __builtin_bit_cast(uint4, v);
}

// four consecutive output elements
__device__ __forceinline__ void store4(bf16_t *p, const f32x4 &x) {
    typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
    bf16x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (__bf16)x[i];
    *reinterpret_cast<uint2 *>(p) = __builtin_bit_cast(uint2, v);
}
__device__ __forceinline__ void store4(float *p, const f32x4 &x) { *reinterpret_cast<f32x4 *>(p) = x; }

}  // namespace air
