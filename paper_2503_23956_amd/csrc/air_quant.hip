// air_quant_append and air_quant_read: rows of K and V into 4 bits, and what they stand for.
//
// Bound by memory: a lane holds eight elements of a row (a group of 32 is four lanes, of 64 eight), reads them with one 16-byte access (bf16) and
// writes its eight codes as one dword; least and greatest element of a group are exchanged with DPP moves, the first lane of the group
// writes (lo, step).
#include "air_device.h"
#include "air_internal.h"
#include "air_quant_dev.h"

namespace air {

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

__device__ __forceinline__ float min_f(float a, float b) { return fminf(a, b); }
// over the 4 (LANES = 4) or 8 consecutive lanes of a group
template <int LANES>
__device__ __forceinline__ void range_of(float &low, float &high) {
    low = AIR_DPP_STEP(min_f, low, 0xB1);
    high = AIR_DPP_STEP(fmaxf, high, 0xB1);
    low = AIR_DPP_STEP(min_f, low, 0x4E);
    high = AIR_DPP_STEP(fmaxf, high, 0x4E);
    if (LANES == 8) {
        low = AIR_DPP_STEP(min_f, low, 0x141);
        high = AIR_DPP_STEP(fmaxf, high, 0x141);
    }
}

// (lo, step) of a group from its least and greatest element
__device__ __forceinline__ uint32_t pair_of(float low, float high) {
    // (a NaN does not pass a minimum or maximum: the caller has put an infinity in its place)
    if (!(fmaxf(-low, high) < 0x1p126f)) return 0x7fc0u;  // NaN, step 0
    const uint32_t u = __float_as_uint(low);
    const uint32_t lo = (u + (u >> 31 ? 0xffffu : 0u)) & 0xffff0000u;  // down: away from zero below it
    const float width = (high - __uint_as_float(lo)) / 15.0f;
    const uint32_t step = (__float_as_uint(width) + 0xffffu) & 0xffff0000u;
    return (__uint_as_float(step) < 0x1p-120f ? 0u : step) | lo >> 16;
}

// which dword of a row holds elements 8 p .. 8 p + 7
template <int D, bool K>
__device__ __forceinline__ int dword_of(int p) {
    return K ? D / 32 * (p & 3) + (p >> 2) : p;
}

template <int D, int GR, typename T, bool K>
__device__ __forceinline__ void append_row(const T *src, uint32_t *codes, uint32_t *scales, int p) {
    float x[8];
    load8(src + 8 * p, x);
    float low = x[0], high = x[0];
    bool number = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        low = fminf(low, x[i]);
        high = fmaxf(high, x[i]);
        number = number && x[i] == x[i];
    }
    if (!number) high = INFINITY;
    range_of<GR / 8>(low, high);
    const uint32_t pair = pair_of(low, high);
    const float lo = lo_of(pair), step = step_of(pair), inv = 1.0f / step;
    uint32_t code = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // the quotient, rounded correctly: the product with the rounded reciprocal, mended once by what it leaves (Markstein)
        const float d = x[i] - lo, q = d * inv;
        const float s = fmaf(fmaf(-q, step, d), inv, q);
        const uint32_t c = step > 0.0f ? (uint32_t)fminf(rintf(s), 15.0f) : 0u;
        code |= c << (K ? (i & 3) * 8 + (i & 4) : 4 * i);
    }
    codes[dword_of<D, K>(p)] = code;
    if ((p & (GR / 8 - 1)) == 0) scales[p / (GR / 8)] = pair;
}

template <int D, int GR, typename T, bool K>
__device__ __forceinline__ void read_row(T *dst, const uint32_t *codes, const uint32_t *scales, int p) {
    const uint32_t code = codes[dword_of<D, K>(p)], pair = scales[p / (GR / 8)];
    const float lo = lo_of(pair), step = step_of(pair);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(step, (float)(code >> (K ? (i & 3) * 8 + (i & 4) : 4 * i) & 15u), lo);
    store8(dst + 8 * p, x);
}

template <int D, int GR, typename T, bool APPEND>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantAppendArgs a) {
    constexpr int kLanes = D / 8, kRows = 256 / kLanes;
    const int p = threadIdx.x & (kLanes - 1), t = blockIdx.x * kRows + threadIdx.x / kLanes;
    const int b = blockIdx.z, h = blockIdx.y;
    const int count = a.counts ? a.counts[b] : a.n_tokens, at = a.lens ? a.lens[b] : 0;
    const int64_t slot = (int64_t)at + t;
    if (t >= count || t >= a.n_tokens || slot < 0 || slot >= a.capacity) return;
    const int64_t cell = ((int64_t)b * a.Hkv + h) * a.capacity + slot;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        T *row = static_cast<T *>(a.rows[i]);
        if (!APPEND && !row) continue;
        row += b * a.row_b[i] + h * a.row_h[i] + t * a.row_t[i];
        uint32_t *codes = reinterpret_cast<uint32_t *>(a.codes[i] + cell * (D / 2)), *scales = a.scales[i] + cell * (D / GR);
        if (APPEND) {
            if (i == 0) append_row<D, GR, T, true>(row, codes, scales, p);
            else append_row<D, GR, T, false>(row, codes, scales, p);
        } else {
            if (i == 0) read_row<D, GR, T, true>(row, codes, scales, p);
            else read_row<D, GR, T, false>(row, codes, scales, p);
        }
    }
    if (APPEND && p == 0) {
        if (a.positions) a.positions[cell] = a.first[b] + t;
        if (a.weights) a.weights[cell] = 0.0f;
    }
}

hipError_t launch_quant_rows(hipStream_t s, const air_quant_cache &c, const air_quant_rows &r, bool append) {
    QuantAppendArgs a;
    a.codes[0] = static_cast<uint8_t *>(c.k_codes);
    a.codes[1] = static_cast<uint8_t *>(c.v_codes);
    a.scales[0] = static_cast<uint32_t *>(c.k_scales);
    a.scales[1] = static_cast<uint32_t *>(c.v_scales);
    a.rows[0] = r.k;
    a.rows[1] = r.v;
    a.row_b[0] = r.k_b;
    a.row_h[0] = r.k_h;
    a.row_t[0] = r.k_t;
    a.row_b[1] = r.v_b;
    a.row_h[1] = r.v_h;
    a.row_t[1] = r.v_t;
    a.lens = r.lens;
    a.counts = r.counts;
    a.first = r.first_positions;
    a.positions = r.positions;
    a.weights = r.weights;
    a.capacity = c.capacity;
    a.n_tokens = r.n_tokens;
    a.Hkv = c.n_kv_heads;
    a.batch = c.batch;
    const int rows = 256 / (c.head_dim / 8);
    const dim3 grid((unsigned)((r.n_tokens + rows - 1) / rows), (unsigned)c.n_kv_heads, (unsigned)c.batch);
#define AIR_CASE(D, GR, T, F)                                               \
    if (c.head_dim == D && c.group == GR && c.dtype == F) {                 \
        if (append) quant_rows_kernel<D, GR, T, true><<<grid, 256, 0, s>>>(a); \
        else quant_rows_kernel<D, GR, T, false><<<grid, 256, 0, s>>>(a);    \
    }
    AIR_CASE(128, 32, bf16_t, AIR_BF16)
    AIR_CASE(128, 64, bf16_t, AIR_BF16)
    AIR_CASE(64, 32, bf16_t, AIR_BF16)
    AIR_CASE(64, 64, bf16_t, AIR_BF16)
    AIR_CASE(128, 32, float, AIR_F32)
    AIR_CASE(128, 64, float, AIR_F32)
    AIR_CASE(64, 32, float, AIR_F32)
    AIR_CASE(64, 64, float, AIR_F32)
#undef AIR_CASE
    return hipGetLastError();
}

}  // namespace air
