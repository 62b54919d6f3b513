// What the kernels of air_quant_attn share: a call's arguments, what a sequence holds and asks, partial results.
#pragma once

#include "air_internal.h"
#include "air_quant_dev.h"

namespace air {

typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

struct QuantAttnArgs {
    const uint8_t *kc, *vc;
    const uint32_t *ks, *vs;
    const void *q;
    void *out;
    float *part_o;    // [pair][split][row][D]
    float2 *part_ml;  // [pair][split][row]
    // many rows with weights:
    float2 *part_norm; // [pair][split][row]: reference and sum that the weights are formed with
    float4 *row_ref;   // [pair][row]: reference, 1 / sum, slots seen (whole number), nothing
    uint4 *row_sums;   // [pair][row][2]: sums of the queries' groups as bf16 terms, as the product with lo takes them
    float *part_w;     // [share of the rows][pair][slot]: weights, where there are several shares
    int32_t w_splits;
    float *weights;
    int64_t q_b, q_h, q_t, out_b, out_h, out_t;
    const int32_t *lens, *counts;
    float c;  // scale * log2(e)
    int32_t Hkv, G, n_tokens, capacity, n_rows, splits, causal, appended;
    Div by_g, by_hkv, by_splits, by_stride, by_pairs, by_shares;  // by_stride: 4 splits; by_shares: w_splits
    int32_t pairs;
    float4 *kept;      // [pair][run of 32][lane]: logits, for the weights of calls with few rows; null: formed again
    int32_t max_runs;  // runs of a pair there
    QuantAppendArgs rows;  // what the first launch appends (few rows), else rows[0] null
};

constexpr int kRun = 64;  // slots that a wave takes at a time
constexpr int kFewRows = 8, kFewRun = 32;  // rows of a call of few, and slots of its waves

template <int N>
struct Words {
    uint32_t w[N];
};
template <int N>
__device__ __forceinline__ Words<N> load_words(const void *p) {
    Words<N> r;
    if (N == 4) *reinterpret_cast<uint4 *>(&r) = *static_cast<const uint4 *>(p);
    else if (N == 2) *reinterpret_cast<uint2 *>(&r) = *static_cast<const uint2 *>(p);
    else r.w[0] = *static_cast<const uint32_t *>(p);
    return r;
}

// What a sequence holds and asks
struct QuantSpan {
    int b, h, count, held, rows;
    int held_before;  // where the call appends its first row
    __device__ __forceinline__ QuantSpan(const QuantAttnArgs &a, int pair) {
        b = a.by_hkv.of(pair);
        h = pair - b * a.Hkv;
        const int n = a.counts ? a.counts[b] : a.n_tokens;
        count = n < 0 ? 0 : n > a.n_tokens ? a.n_tokens : n;
        held_before = a.lens[b];
        const int64_t all = (int64_t)held_before + (a.appended ? count : 0);
        held = all < 0 ? 0 : all > a.capacity ? a.capacity : (int)all;
        rows = count * a.G;
    }
    // slots that row r sees (r < rows)
    __device__ __forceinline__ int seen(const QuantAttnArgs &a, int r) const {
        if (!a.causal) return held;
        const int s = held - count + 1 + a.by_g.of(r);
        return s < 0 ? 0 : s;
    }
};

__device__ __forceinline__ float finite_or_zero(float ref) { return ref == -INFINITY ? 0.0f : ref; }

// weight of sums taken against the reference m in sums against top
__device__ __forceinline__ float part_weight(float m, float l, float top) {
    if (m == -INFINITY) return l == 0.0f ? 0.0f : 1.0f;  // (no finite logit: nothing, or NaN that stays)
    return __builtin_amdgcn_exp2f(m - top);
}

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t *p, float v) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void put4(float *p, const f32x4 &v) { *reinterpret_cast<f32x4 *>(p) = v; }
__device__ __forceinline__ void put4(bf16_t *p, const f32x4 &v) {
    const bf16x2 a = {(__bf16)v[0], (__bf16)v[1]}, b = {(__bf16)v[2], (__bf16)v[3]};
    *reinterpret_cast<uint2 *>(p) = uint2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}

// Second launch of a (sequence, KV head): rows joined over the splits, and what every slot was attended to - the logits once more, now against
// every row's maximum and sum.  The partial results of a row are requested all at once: a lane per split for (maximum, sum), and
// for the outputs D / 4 lanes a split.  AHEAD: requests do not wait for the sequence's rows to be known (what lies behind them is not used).
template <int D, typename T, bool AHEAD = false>
__device__ __forceinline__ void join_rows(const QuantAttnArgs &a, const QuantSpan &sp, int pair, float4 *lds) {
    constexpr int kLanes = D / 4, kPlaces = 256 / kLanes;  // places: splits of a row side by side, and rows
    int groups = 1;
    while (groups < a.splits && groups < kPlaces) groups *= 2;
    const int place = threadIdx.x / kLanes, x = threadIdx.x % kLanes, group = place & (groups - 1), lane = threadIdx.x & 63;
    const int rows = kPlaces / groups, all = AHEAD ? a.n_rows : sp.rows;
    const float2 *ml = a.part_ml + (size_t)pair * a.splits * a.n_rows;
    for (int first = blockIdx.x * rows; first < all; first += gridDim.x * rows) {
        const int row = first + place / groups, r = row < all ? row : all - 1;
        const float4 *o = reinterpret_cast<const float4 *>(a.part_o + ((size_t)pair * a.splits * a.n_rows + r) * D) + x;
        const size_t step = (size_t)a.n_rows * (D / 4);
        float4 sum = {0.f, 0.f, 0.f, 0.f};
        float top = -INFINITY, l = 0.0f;
        float4 part[8];
        float2 v[8];
        for (int s0 = group; s0 < a.splits; s0 += 8 * groups) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int s = s0 + k * groups;
                v[k] = float2{-INFINITY, 0.f};
                part[k] = float4{0.f, 0.f, 0.f, 0.f};
                if (s < a.splits) {
                    v[k] = ml[(size_t)s * a.n_rows + r];
                    part[k] = o[s * step];
                }
            }
            float most = top;
#pragma unroll
            for (int k = 0; k < 8; ++k) most = fmaxf(most, v[k].x);
            const float f0 = part_weight(top, l, most);
            sum.x *= f0, sum.y *= f0, sum.z *= f0, sum.w *= f0;
            l *= f0;
            top = most;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float f = part_weight(v[k].x, v[k].y, top);
                l = fmaf(f, v[k].y, l);
                sum.x = fmaf(f, part[k].x, sum.x);
                sum.y = fmaf(f, part[k].y, sum.y);
                sum.z = fmaf(f, part[k].z, sum.z);
                sum.w = fmaf(f, part[k].w, sum.w);
            }
        }
        if (groups > 1) {
            __syncthreads();
            lds[threadIdx.x] = sum;
            float2 *lds_ml = reinterpret_cast<float2 *>(lds + 256);
            if (x == 0) lds_ml[place] = float2{top, l};
            __syncthreads();
            if (group == 0) {
                float most = top;
                for (int k = 1; k < groups; ++k) most = fmaxf(most, lds_ml[place + k].x);
                const float f0 = part_weight(top, l, most);
                sum.x *= f0, sum.y *= f0, sum.z *= f0, sum.w *= f0;
                l *= f0;
                for (int k = 1; k < groups; ++k) {
                    const float2 w = lds_ml[place + k];
                    const float4 y = lds[threadIdx.x + k * kLanes];
                    const float f = part_weight(w.x, w.y, most);
                    l = fmaf(f, w.y, l);
                    sum.x = fmaf(f, y.x, sum.x);
                    sum.y = fmaf(f, y.y, sum.y);
                    sum.z = fmaf(f, y.z, sum.z);
                    sum.w = fmaf(f, y.w, sum.w);
                }
            }
        }
        if (group == 0 && row < sp.rows) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const int t = a.by_g.of(row);
            T *to = static_cast<T *>(a.out) + sp.b * a.out_b + ((int64_t)sp.h * a.G + row - t * a.G) * a.out_h + t * a.out_t + 4 * x;
            put4(to, f32x4{sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv});
        }
    }
}

// (maximum, 1 / sum) of a row over the splits; by 16 lanes, n of them
struct RowReference {
    float2 v[4];
    __device__ __forceinline__ void request(const QuantAttnArgs &a, int pair, int row, int rows, int n) {
        const float2 *ml = a.part_ml + (size_t)pair * a.splits * a.n_rows;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = float2{-INFINITY, 0.f};
            if (n + 16 * k < a.splits && row < rows) v[k] = ml[(size_t)(n + 16 * k) * a.n_rows + row];
        }
    }
    // real: false makes it that of a row without slots, whatever was read
    __device__ __forceinline__ void form(int n, bool real, float2 *to) const {
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, v[k].x);
        top = max16(top);
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += part_weight(v[k].x, v[k].y, top) * v[k].y;
        sum = sum16(sum);
        if (n == 0) *to = real ? float2{finite_or_zero(top), sum == 0.0f ? 0.0f : 1.0f / sum} : float2{0.f, 0.f};
    }
};

hipError_t launch_quant_many(hipStream_t s, const QuantAttnArgs &a, const QuantPlan &p, int head_dim, int group, int pairs);

}  // namespace air
