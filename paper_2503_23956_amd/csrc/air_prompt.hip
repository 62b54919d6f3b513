// air_prompt_attn: causal attention of prompts, pieces of prompts and single tokens over the full cache.
//
//   out_t = sum_j p_j v_j,   p = softmax over j <= t + kv_len - q_len of scale * q_t . k_j
//
// The rows of one (sequence, KV head) are its queries times the G query heads that share the KV head, token by token: row
// m = t G + g.  K and V are then read once for all heads of the group, a tile of rows spans few tokens (little of the causal
// triangle is wasted), and prompts, pieces and single tokens are one shape: rows x keys.
//
// Both products run on 32 x 32 tiles of the matrix unit, transposed: S^T = K Q^T leaves lane (n = lane % 32, h = lane / 32)
// with query n's logits at the keys 8 (i / 4) + 4 h + i % 4, i = 0..15.  Maximum and sum of a query need one exchange between two
// lanes, and registers 8 s .. 8 s + 7 are the operand P^T of O^T = V^T P^T as they are, when the operand V^T takes the keys in the same
// order: no probability leaves its lane.  The accumulators O^T have query n in the same lanes, so that a new reference maximum
// scales them with the lane's own factor.
//
// Softmax in the base-2 domain with a running reference per query; it is raised only when a logit lies more than kSlack above it.
//
// Measured (bf16, heads of 128): prompts of 7432 tokens, 28 / 4 heads, 384 to 407 us by card (1 PFLOP/s, matrix unit busy 47 % of the clocks at 2.05
// GHz); 16910 + 16001 tokens, 64 / 8 heads, 7.79 to 8.48 ms (1.1 PFLOP/s, matrix unit busy 55 % at 1.92 GHz; with inputs of zeros 1.34 PFLOP/s: bound by
// power); one token over 7432 keys 11 us (two launches).
#include <math.h>
#include <string.h>

#include "air_device.h"
#include "air_internal.h"
#include "air_tile.h"

namespace air {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

// Division by a number that the host knows: x / d = (x m) >> s for 0 <= x < 2^31, with 2^(s - 32) < d <= 2^(s - 31) and
// m = ceil(2^s / d) (m d - 2^s < d <= 2^(s - 31): the quotient is off by less than 1 / d)
struct Div {
    uint32_t m, s;
    __device__ __forceinline__ int of(int x) const { return (int)(((uint64_t)(uint32_t)x * m) >> s); }
};
static Div div_by(int d) {
    Div r;
    r.s = 31;
    while ((1ll << (r.s - 31)) < d) ++r.s;
    r.m = (uint32_t)(((1ull << r.s) + (uint64_t)d - 1) / (uint64_t)d);
    return r;
}

struct PromptSpan {
    int64_t q_off, k_off, v_off, out_off;
    int32_t q_len, kv_len;
    int32_t n_tiles;  // row tiles
    int32_t row0;     // first row (query x query head of the group) in the partial results
};
struct PromptArgs {
    const void *q, *k, *v;
    void *out;
    float *part_o;    // [split][KV head][row][D]
    float2 *part_ml;  // [split][KV head][row]
    int64_t q_h, q_t, k_h, k_t, v_h, v_t, out_h, out_t;
    float c;  // scale * log2(e)
    int32_t G, Hkv, n_seqs, n_tiles, n_rows, splits;
    Div by_g, by_hkv, by_splits, by_rows;
    // The sequences lie in `s` by falling number of row tiles.  A launch takes the tiles by falling index inside their sequence, so that
    // tiles of about equal length run side by side and the shortest at the end: of rank rank0[i] on, i + 1 sequences have a tile of the
    // index in question (behind the last sequence: INT32_MAX)
    int32_t rank0[AIR_MAX_BATCH];
    int32_t row0[AIR_MAX_BATCH];  // PromptSpan::row0 (behind the last sequence: INT32_MAX)
    PromptSpan s[AIR_MAX_BATCH];
};
static_assert(AIR_MAX_BATCH == 64 && sizeof(PromptArgs) <= 4096, "a lane per sequence; the size of an argument block");

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

// the elements that are finite, 0 in place of the others
__device__ __forceinline__ u32x4 finite_part(u32x4 x, bf16_t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = (x[i] & 0x7f80u) == 0x7f80u ? 0u : x[i] & 0xffffu;
        const uint32_t hi = (x[i] & 0x7f800000u) == 0x7f800000u ? 0u : x[i] & 0xffff0000u;
        x[i] = lo | hi;
    }
    return x;
}
__device__ __forceinline__ u32x4 finite_part(u32x4 x, float) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (x[i] & 0x7f800000u) == 0x7f800000u ? 0u : x[i];
    return x;
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

// One row tile of 32 of a wave against a tile of 32 keys in LDS
template <typename T, int D>
struct Attend {
    using R = Row<T, D>;
    static constexpr int ND = D / 32;  // output tiles of 32 columns
    f32x16 acc[ND];
    float m, l;  // reference (scaled logits), this lane's part of the sum
    uint4 q[R::kSlices];

    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    }

    // last: last key of the tile that the lane's query sees, counted from the tile's first (read when masked, uniform over the wave).
    // two (bf16, uniform over the workgroup): probabilities of the second product as the sum of two bf16 numbers, of which 2^-16 is lost,
    // not 2^-8 as with one
    __device__ __forceinline__ void step(const u32x4 *sk, const u32x4 *sv, bool masked, bool two, int last, float c) {
        const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int sl = 0; sl < R::kSlices; ++sl) s = mma32(__builtin_bit_cast(uint4, sk[R::k_at(n, 2 * sl + h)]), q[sl], s, T());
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (8 * (i >> 2) + 4 * h + (i & 3) > last) s[i] = -INFINITY;
        }
        const float mx = largest(s) * c;
        if (__ballot(mx > m + kSlack) != 0ull) {
            const float m_new = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32, 64)));
            const float f = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);  // no logit but -inf yet: nothing to scale
            l *= f;
            m = m_new;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        if (__builtin_expect(__ballot(fabsf(ref) > kHuge) == 0ull, 1)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], c, -ref);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = rounded_exponent(s[i], c, ref);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i]);
        if constexpr (sizeof(T) == 2) {
            const int at = v_lane(lane);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                bf16x8 x, y;
                if (two) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float p = s[8 * half + i], top = __uint_as_float(__float_as_uint(p) & 0xffff0000u);
                        x[i] = (__bf16)top;
                        // (not negative, and 0 only with p: an infinite value stays the infinity that it is with one term)
                        y[i] = (__bf16)__builtin_amdgcn_fmed3f(p - top, 0x1p-126f, p);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = (__bf16)s[8 * half + i];
                }
                const uint4 p = __builtin_bit_cast(uint4, x);
                uint4 v[ND];
#pragma unroll
                for (int d = 0; d < ND; ++d) v[d] = read_v<D>(sv, at, half, d);
                l = sum_of(p, l);
#pragma unroll
                for (int d = 0; d < ND; ++d) acc[d] = mma32(v[d], p, acc[d], T());
                if (two) {
                    const uint4 rest = __builtin_bit_cast(uint4, y);
                    l = sum_of(rest, l);
#pragma unroll
                    for (int d = 0; d < ND; ++d) acc[d] = mma32(v[d], rest, acc[d], T());
                }
            }
        } else {
            const float *base = reinterpret_cast<const float *>(sv) + 32 * h + n;
#pragma unroll
            for (int i = 0; i < 16; ++i) l += s[i];
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const float v = base[4 * R::kBlock * d + 256 * (i >> 2) + 64 * (i & 3)];
                    acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[i], acc[d], 0, 0, 0);
                }
        }
    }
};

// What a thread loads of a tile of keys, kLoads rows apart by kRowStep, on its way to LDS
template <typename T, int D, int THREADS, int KEYS>
struct Stage {
    using R = Row<T, D>;
    static constexpr int kLoads = KEYS * R::kPieces / THREADS, kRowStep = THREADS / R::kPieces;
    static_assert(kLoads >= 1 && kLoads * THREADS == KEYS * R::kPieces, "whole rounds of loads");
    int piece, row;
    uint32_t k_lane, v_lane;  // bytes from a tile's first row (token strides are below 2^24 elements)
    u32x4 k[kLoads], v[kLoads];

    __device__ __forceinline__ void init(const PromptArgs &a, int thread) {
        piece = thread % R::kPieces;
        row = thread / R::kPieces;
        k_lane = (uint32_t)(row * (int)a.k_t + R::kVec * piece) * (uint32_t)sizeof(T);
        v_lane = (uint32_t)(row * (int)a.v_t + R::kVec * piece) * (uint32_t)sizeof(T);
    }
    // keys from kb on, of kv_len in all; kg, vg: the first key's and value's rows
    __device__ __forceinline__ void load(const PromptArgs &a, const T *kg, const T *vg, int kb, int kv_len) {
        const char *kp = (const char *)(kg + kb * a.k_t), *vp = (const char *)(vg + kb * a.v_t);
        const int end = kv_len - 1 - kb;
        if (end >= KEYS - 1) {
            const uint32_t k_step = kRowStep * (uint32_t)a.k_t * (uint32_t)sizeof(T), v_step = kRowStep * (uint32_t)a.v_t * (uint32_t)sizeof(T);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) k[i] = *reinterpret_cast<const u32x4 *>(kp + (uint64_t)i * k_step + k_lane);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) v[i] = *reinterpret_cast<const u32x4 *>(vp + (uint64_t)i * v_step + v_lane);
        } else {  // rows past the last key re-read it
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = min(row + kRowStep * i, end);
                k[i] = *reinterpret_cast<const u32x4 *>(kp + (uint32_t)(r * (int)a.k_t + R::kVec * piece) * (uint32_t)sizeof(T));
                v[i] = *reinterpret_cast<const u32x4 *>(vp + (uint32_t)(r * (int)a.v_t + R::kVec * piece) * (uint32_t)sizeof(T));
            }
        }
    }
    // Of a tile that some row does not see all of: that row's probability of 0 must not meet an infinity.  Values behind the last
    // key (`left` are left from the tile's first) become 0, and so does what is not finite: true if there was any (add_not_finite
    // gives it to the rows that see it)
    __device__ __forceinline__ bool clean(int left) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (row + kRowStep * i >= left) v[i] = (u32x4){0, 0, 0, 0};
            const u32x4 x = finite_part(v[i], T());
#pragma unroll
            for (int w = 0; w < 4; ++w) bad = bad || x[w] != v[i][w];
            v[i] = x;
        }
        return bad;
    }
    __device__ __forceinline__ void store(u32x4 *sk, u32x4 *sv) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = row + kRowStep * i;
            sk[(r >> 5) * R::kKTile + R::k_at(r & 31, piece)] = k[i];
            sv[(r >> 5) * R::kVTile + R::v_at(r & 31, piece)] = v[i];
        }
    }
};

// the values of keys [key0, key1) that are not finite, added to the accumulators of a row that sees the keys up to `last` (whole, as their weights
// are not known here: what a weight of 0 makes no number elsewhere becomes an infinity)
template <typename T, int ND>
__device__ __forceinline__ void add_not_finite(f32x16 (&acc)[ND], const T *vg, int64_t v_t, int key0, int key1, int last, int h) {
    for (int key = key0; key < key1 && key <= last; ++key)
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float v = ldf(vg + key * v_t + 32 * d + 8 * (i >> 2) + 4 * h + (i & 3));
                if (!(fabsf(v) < INFINITY)) acc[d][i] += v;
            }
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

// Brings the arguments that every workgroup needs into registers together: left to themselves, they are read where they are used, one wait for
// memory behind the other (one token over 7432 keys 12.3 us so, 11.8 like this).
__device__ __forceinline__ void fetch(const PromptArgs &a) {
    asm volatile("" ::"s"(a.q), "s"(a.k), "s"(a.v), "s"(a.out), "s"(a.q_h), "s"(a.q_t), "s"(a.k_h), "s"(a.k_t), "s"(a.v_h), "s"(a.v_t), "s"(a.G),
                 "s"(a.Hkv), "s"(a.n_seqs), "s"(a.splits), "s"(a.by_g.m), "s"(a.by_hkv.m), "s"(a.by_splits.m), "s"(a.s[0].q_off), "s"(a.s[0].k_off),
                 "s"(a.s[0].v_off), "s"(a.s[0].q_len), "s"(a.s[0].n_tiles));
}

// Sequence, row tile and split of the workgroups with number y of a KV head.  The KV head itself is the fastest index of a launch: with 1,
// 2, 4 or 8 of them every XCD, dealt workgroups round-robin, works on one head's K and V.
struct Place {
    int tile, split, q_len, kv_len, row0;
    int64_t q_off, k_off, v_off, out_off;
};
__device__ __forceinline__ int64_t of_lane(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32);
}
__device__ __forceinline__ Place place_of(const PromptArgs &a, int y) {
    Place p;
    const int rank = a.by_splits.of(y);
    p.split = y - rank * a.splits;
    if (a.n_seqs == 1) {
        p.tile = a.s[0].n_tiles - 1 - rank;
        p.q_len = a.s[0].q_len, p.kv_len = a.s[0].kv_len, p.row0 = a.s[0].row0;
        p.q_off = a.s[0].q_off, p.k_off = a.s[0].k_off, p.v_off = a.s[0].v_off, p.out_off = a.s[0].out_off;
    } else {
        // every lane loads a sequence, all at once, and a vote finds the one, in place of a chain of loads
        const int i = threadIdx.x & 63;
        const int rank0 = a.rank0[i], n_tiles = a.s[i].n_tiles, q_len = a.s[i].q_len, kv_len = a.s[i].kv_len, row0 = a.s[i].row0;
        const int64_t q_off = a.s[i].q_off, k_off = a.s[i].k_off, v_off = a.s[i].v_off, out_off = a.s[i].out_off;
        const int k = __popcll(__ballot(rank0 <= rank));
        const int off = rank - __builtin_amdgcn_readlane(rank0, k - 1), level = off / k, seq = __builtin_amdgcn_readfirstlane(off - level * k);
        p.tile = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_readlane(n_tiles, k - 1) - 1 - level);
        p.q_len = __builtin_amdgcn_readlane(q_len, seq), p.kv_len = __builtin_amdgcn_readlane(kv_len, seq);
        p.row0 = __builtin_amdgcn_readlane(row0, seq);
        p.q_off = of_lane(q_off, seq), p.k_off = of_lane(k_off, seq), p.v_off = of_lane(v_off, seq), p.out_off = of_lane(out_off, seq);
    }
    return p;
}

// ---------------------------------------------------------------------------------------
// Many rows, bf16: eight waves of 32 rows, two a SIMD; key blocks of 64 in LDS (three buffers), the loads of the block after next in
// flight.  A wave forms the logits of its next 32 keys (matrix unit) under the exponentials of the present ones (vector unit), in one run
// of instructions without a branch; the operands of the logits after those are read from LDS meanwhile.
// KW 1: 256 rows, every wave takes both halves of a block, one barrier a block.  KW 2: 128 rows, two waves share 32 rows and take a
// half of every block each; their sums are joined at the end through LDS: twice the workgroups where a call has few rows.
// (Two row tiles a wave, to halve the reads of LDS, need more than 256 registers: the accumulators then wander between the two
// register files, 12.4 ms against 8.9 for 2 x 16910 tokens of 64 heads.)
// ---------------------------------------------------------------------------------------
template <typename T, int D, int KW>
__global__ __launch_bounds__(512, 2) void prompt_pipe_kernel(PromptArgs a) {
    fetch(a);
    using R = Row<T, D>;
    static_assert(sizeof(T) == 2, "bf16");
    constexpr int NW = 8, RW = NW / KW, kRows = 32 * RW, kKeys = 64, ND = D / 32, NS = R::kSlices, kBufs = 3;
    __shared__ u32x4 tiles[2 * kBufs * (R::kKTile + R::kVTile)];
    __shared__ float2 s_ml[KW == 2 ? RW * 32 : 1];
    __shared__ int s_bad;
    auto sk = [&](int b) { return tiles + b % kBufs * (2 * R::kKTile); };  // the two tiles of block b
    auto sv = [&](int b) { return tiles + 2 * kBufs * R::kKTile + b % kBufs * (2 * R::kVTile); };
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rw = wave % RW, kw = wave / RW;
    const int y = a.by_hkv.of(blockIdx.x), kvh = blockIdx.x - y * a.Hkv;
    const Place pl = place_of(a, y);
    const int n_rows = pl.q_len * a.G, shift = pl.kv_len - pl.q_len;
    const int row0 = pl.tile * kRows, end_row = min(row0 + kRows, n_rows);
    // keys that every row of the tile sees, and that any does
    const int see_all = max(0, a.by_g.of(row0) + shift + 1), see_any = max(0, a.by_g.of(end_row - 1) + shift + 1);
    const int n_blocks = (see_any + kKeys - 1) / kKeys;
    const int per_split = (n_blocks + a.splits - 1) / a.splits;
    const int b0 = pl.split * per_split, b1 = min(n_blocks, b0 + per_split);

    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    float l = 0.f, ref = -INFINITY, top = -INFINITY, mul = a.c, sub = 0.f;  // top: the logit (scaled) from which on the reference is raised
    bool huge = false;
    const int row = row0 + 32 * rw + n, m_row = min(row, n_rows - 1), tok = a.by_g.of(m_row), head = kvh * a.G + m_row - tok * a.G;
    const int last = tok + shift;  // last key that the lane's query sees
    uint4 q[NS];
    {
        const T *qp = (const T *)a.q + pl.q_off + tok * a.q_t + head * a.q_h;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) q[sl] = *reinterpret_cast<const uint4 *>(qp + R::kVec * (2 * sl + h));
    }

    const T *kg = (const T *)a.k + pl.k_off + kvh * a.k_h, *vg = (const T *)a.v + pl.v_off + kvh * a.v_h;
    Stage<T, D, 64 * NW, kKeys> stage;
    stage.init(a, threadIdx.x);
    auto load = [&](int b) {
        if (b < b1) stage.load(a, kg, vg, b * kKeys, pl.kv_len);
    };
    auto keep = [&](int b) {
        if (b >= b1) return;
        if ((b + 1) * kKeys > see_all && stage.clean(pl.kv_len - b * kKeys)) s_bad = 1;
        stage.store(sk(b), sv(b));
    };
    // operands of the logits of the 32 keys whose tile starts at sk_
    auto read_k = [&](u32x4(&x)[NS], const u32x4 *sk_) {
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) x[sl] = sk_[R::k_at(n, 2 * sl + h)];
    };
    auto logits = [&](f32x16 &s, const u32x4(&x)[NS]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) s = mma32(__builtin_bit_cast(uint4, x[sl]), q[sl], s, T());
    };
    // masks, reference: what has to be known of the logits of the keys from kb on before their exponentials are formed
    auto settle = [&](f32x16 &s, float mx, int kb) {
        if (__builtin_expect(kb + 32 > see_all, 0)) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (kb + 8 * (i >> 2) + 4 * h + (i & 3) > last) s[i] = -INFINITY;
            mx = largest(s);
        }
        mx *= a.c;
        if (__builtin_expect(__ballot(mx > top) != 0ull, 0)) {
            const float now = fmaxf(ref, fmaxf(mx, __shfl_xor(mx, 32, 64)));
            const float f = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref - now);  // no logit but -inf yet: nothing to scale
            l *= f;
            ref = now;
            top = now + kSlack;
            sub = now == -INFINITY ? 0.f : now;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= f;
            huge = huge || __ballot(fabsf(sub) > kHuge) != 0ull;
        }
        if (__builtin_expect(huge, 0)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = rounded_exponent(s[i], a.c, ref == -INFINITY ? 0.f : ref);
            mul = 1.f;
            sub = 0.f;
        }
    };
    const int v_at = v_lane(lane);
    // The next 32 keys' logits into `next` (operands: kf), their largest into mx, while the values of this 32 keys are weighed; kf then
    // takes the operands of the keys behind those.  meet: the tile that k_after points to is whole only behind a barrier.
    auto turn = [&](f32x16 &s, f32x16 &next, float &mx, u32x4(&kf)[NS], const u32x4 *sv_, const u32x4 *k_after, bool meet) {
        uint4 vf[2][ND], p[2];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int d = 0; d < ND; ++d) vf[0][d] = read_v<D>(sv_, v_at, 0, d);
        logits(next, kf);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            bf16x8 x;
            // rounded to bf16, 2^-8 of a probability: a second term, as Attend has it, would be half as much work again for the matrix unit,
            // which is what these kernels wait for
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[8 * half + i], mul, -sub));
            p[half] = __builtin_bit_cast(uint4, x);
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) vf[1][d] = read_v<D>(sv_, v_at, 1, d);
        if (meet) lds_barrier();
        read_k(kf, k_after);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] = mma32(vf[half][d], p[half], acc[d], T());
        l = sum_of(p[1], sum_of(p[0], l));  // the sum of what the second product takes: the weights add up to one as they are used
        mx = largest(next);
        __builtin_amdgcn_s_setprio(0);
    };
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
    if (b0 < b1) {
        f32x16 sa, sb;
        float mx;
        u32x4 kf[NS];
        load(b0);
        keep(b0);
        load(b0 + 1);
        if constexpr (KW == 2) {
            keep(b0 + 1);
            load(b0 + 2);
        }
        lds_barrier();
        read_k(kf, sk(b0) + kw * R::kKTile);
        logits(sa, kf);
        settle(sa, largest(sa), b0 * kKeys + 32 * kw);
        // (behind the last block: logits of whatever lies there, not used)
        if constexpr (KW == 1) {
            read_k(kf, sk(b0) + R::kKTile);
            for (int b = b0; b < b1; ++b) {
                const u32x4 *v_now = sv(b), *k_next = sk(b + 1);
                keep(b + 1);  // (into the buffer of block b - 2, which every wave has left before the last barrier)
                load(b + 2);
                turn(sa, sb, mx, kf, v_now, k_next, true);
                settle(sb, mx, b * kKeys + 32);
                turn(sb, sa, mx, kf, v_now + R::kVTile, k_next + R::kKTile, false);
                if (b + 1 < b1) settle(sa, mx, (b + 1) * kKeys);
            }
        } else {
            read_k(kf, sk(b0 + 1) + kw * R::kKTile);
            auto block = [&](int b, f32x16 &s, f32x16 &next) {
                keep(b + 2);  // (into the buffer of block b - 1: its values were read before the last barrier)
                load(b + 3);
                turn(s, next, mx, kf, sv(b) + kw * R::kVTile, sk(b + 2) + kw * R::kKTile, true);
                if (b + 1 < b1) settle(next, mx, (b + 1) * kKeys + 32 * kw);
            };
            for (int b = b0; b < b1; b += 2) {
                block(b, sa, sb);
                if (b + 1 < b1) block(b + 1, sb, sa);
            }
        }
    }
    l += __shfl_xor(l, 32, 64);
    if constexpr (KW == 2) {  // the two waves of 32 rows: lane by lane
        static_assert(sizeof(tiles) >= RW * 32 * D * sizeof(float), "the tiles' memory holds the sums of half the waves");
        f32x4 *sums = reinterpret_cast<f32x4 *>(tiles) + rw * (4 * ND * 64) + lane;
        lds_barrier();
        if (kw == 1) {
            if (h == 0) s_ml[rw * 32 + n] = make_float2(ref, l);
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) sums[(4 * d + i) * 64] = (f32x4){acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]};
        }
        lds_barrier();
        if (kw == 1) return;
        const float2 other = s_ml[rw * 32 + n];
        const float now = fmaxf(ref, other.x);
        const float f0 = weight(ref, now), f1 = weight(other.x, now);
        ref = now;
        l = l * f0 + other.y * f1;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 x = sums[(4 * d + i) * 64];
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[d][4 * i + j] = acc[d][4 * i + j] * f0 + x[j] * f1;
            }
    }
    if (s_bad) add_not_finite(acc, vg, a.v_t, max(b0 * kKeys, see_all / kKeys * kKeys), min(b1 * kKeys, see_any), last, h);
    if (a.splits == 1) {
        // through LDS (clear of the sums above), so that a row leaves in whole lines
        const float inv = 1.0f / l;
        if (KW == 1) lds_barrier();
        u32x4 *rows = (rw < 4 ? sv(1) : sk(1)) + (rw & 3) * (32 * R::kPieces);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = l == 0.f ? 0.f : acc[d][4 * i + j] * inv;
                store4(reinterpret_cast<T *>(rows + n * R::kPieces + ((4 * d + i) ^ (n & (R::kPieces - 1)))) + 4 * h, o);
            }
        wave_sync();
        T *out = (T *)a.out + pl.out_off + R::kVec * (lane % R::kPieces);
#pragma unroll
        for (int i = 0; i < R::kPieces / 2; ++i) {
            const int r = lane / R::kPieces + (64 / R::kPieces) * i, m = row0 + 32 * rw + r;
            const u32x4 o = rows[r * R::kPieces + ((lane % R::kPieces) ^ (r & (R::kPieces - 1)))];
            const int to = a.by_g.of(m), hd = kvh * a.G + m - to * a.G;
            if (m < n_rows) *reinterpret_cast<u32x4 *>(out + to * a.out_t + hd * a.out_h) = o;
        }
    } else if (row < n_rows) {
        const int64_t slot = ((int64_t)pl.split * a.Hkv + kvh) * a.n_rows + pl.row0 + row;
        if (h == 0) a.part_ml[slot] = make_float2(ref, l);
        float *po = a.part_o + slot * D + 4 * h;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store4(po + 32 * d + 8 * i, (f32x4){acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]});
    }
}

// ---------------------------------------------------------------------------------------
// Many rows, fp32: four waves of 32 rows share the key tiles of 32 in LDS (two buffers, one barrier a tile, the next tile's loads in flight).
// The fp32 matrix unit sets the pace: 64 clocks a product of 32 x 32 x 2.  Two workgroups a CU, so that one's exponentials, stores and reads
// of LDS run under the other's products.  28 / 4 heads of 128: 5000 tokens 1.42 ms, 126 of the 146 TFLOP/s that a product of matrices reaches (in
// tiles of 32 rows, which read K and V from the L2 caches four times as often, 1.86 ms); 2048 tokens 290 us (356).
// ---------------------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void prompt_share_kernel(PromptArgs a) {
    fetch(a);
    using R = Row<T, D>;
    constexpr int kRows = 128, ND = D / 32;
    __shared__ u32x4 sk[2][R::kKTile], sv[2][R::kVTile];
    __shared__ int s_bad;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int y = a.by_hkv.of(blockIdx.x), kvh = blockIdx.x - y * a.Hkv;
    const Place pl = place_of(a, y);
    const int n_rows = pl.q_len * a.G, shift = pl.kv_len - pl.q_len;
    const int row0 = pl.tile * kRows, end_row = min(row0 + kRows, n_rows);
    const int see_all = max(0, a.by_g.of(row0) + shift + 1), see_any = max(0, a.by_g.of(end_row - 1) + shift + 1);
    const int n_blocks = (see_any + 31) / 32;
    const int per_split = (n_blocks + a.splits - 1) / a.splits;
    const int b0 = pl.split * per_split, b1 = min(n_blocks, b0 + per_split);

    const T *kg = (const T *)a.k + pl.k_off + kvh * a.k_h, *vg = (const T *)a.v + pl.v_off + kvh * a.v_h;
    Stage<T, D, 256, 32> stage;
    stage.init(a, threadIdx.x);
    if (b0 < b1) stage.load(a, kg, vg, b0 * 32, pl.kv_len);
    Attend<T, D> at;
    at.clear();
    const int row = row0 + 32 * wave + n, m_row = min(row, n_rows - 1), tok = a.by_g.of(m_row), head = kvh * a.G + m_row - tok * a.G;
    const int last = tok + shift;
    // last key that a row of the wave sees
    const int wave_last = row0 + 32 * wave < n_rows ? a.by_g.of(min(row0 + 32 * wave + 31, n_rows - 1)) + shift : -1;
    {
        const T *q = (const T *)a.q + pl.q_off + tok * a.q_t + head * a.q_h;
#pragma unroll
        for (int sl = 0; sl < R::kSlices; ++sl) at.q[sl] = *reinterpret_cast<const uint4 *>(q + R::kVec * (2 * sl + h));
    }
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
        const bool masked = (b + 1) * 32 > see_all;
        if (masked && stage.clean(pl.kv_len - b * 32)) s_bad = 1;
        stage.store(sk[b & 1], sv[b & 1]);  // (read for block b - 2, which every wave has left before the last barrier)
        lds_barrier();
        if (b + 1 < b1) stage.load(a, kg, vg, (b + 1) * 32, pl.kv_len);
        if (b * 32 <= wave_last) at.step(sk[b & 1], sv[b & 1], masked, false, last - b * 32, a.c);
    }
    const float l = at.l + __shfl_xor(at.l, 32, 64);
    if (s_bad) add_not_finite(at.acc, vg, a.v_t, max(b0, see_all / 32) * 32, min(b1 * 32, see_any), last, h);
    if (row >= n_rows) return;
    if (a.splits == 1) {
        const float inv = 1.0f / l;
        T *o = (T *)a.out + pl.out_off + tok * a.out_t + head * a.out_h + 4 * h;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = l == 0.f ? 0.f : at.acc[d][4 * i + j] * inv;
                store4(o + 32 * d + 8 * i, x);
            }
    } else {
        const int64_t slot = ((int64_t)pl.split * a.Hkv + kvh) * a.n_rows + pl.row0 + row;
        if (h == 0) a.part_ml[slot] = make_float2(at.m, l);
        float *po = a.part_o + slot * D + 4 * h;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store4(po + 32 * d + 8 * i, (f32x4){at.acc[d][4 * i], at.acc[d][4 * i + 1], at.acc[d][4 * i + 2], at.acc[d][4 * i + 3]});
    }
}

// ---------------------------------------------------------------------------------------
// Few rows: 32 of one (sequence, KV head).  Four waves share the rows and deal the key tiles of 32 among themselves; each moves its
// tiles through LDS of its own, the next tile's loads in flight, without a barrier: one wave takes in 32 keys in about 1.3 us, a launch of 16
// tokens over 7432 keys each 244 MB in 39 us (the join 5 more).
// TWO (bf16): where a sequence has one tile of rows (tokens, steps, pieces of a few queries), its probabilities are the sum of two bf16 numbers.
// Such a sequence reads K and V for one tile only and waits for them, not for the matrix unit: one token over 7432 keys 10.9 us with one term and
// 10.9 with two, 16 of them 43.1 to 43.9 and 43.4 to 43.7, the error of their rows against fp64 0.0020 and 0.0017.  A prompt's tiles keep the
// matrix unit busy: 2048 tokens with 14 / 2 heads of 64 take 25.7 us with one term, 28.9 with two; calls without a sequence of one tile run
// a kernel that does not ask (26.6 where it asks).
// ---------------------------------------------------------------------------------------
template <typename T, int D, bool TWO>
__global__ __launch_bounds__(256) void prompt_few_kernel(PromptArgs a) {
    fetch(a);
    using R = Row<T, D>;
    constexpr int NW = 4;
    __shared__ u32x4 tiles[NW][R::kKTile + R::kVTile];
    __shared__ float s_m[NW][32], s_l[NW][32];
    __shared__ int s_bad;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int y = a.by_hkv.of(blockIdx.x), kvh = blockIdx.x - y * a.Hkv;
    const Place pl = place_of(a, y);
    const int n_rows = pl.q_len * a.G, shift = pl.kv_len - pl.q_len;
    const int row0 = pl.tile * 32, end_row = min(row0 + 32, n_rows);
    const int see_all = max(0, a.by_g.of(row0) + shift + 1), see_any = max(0, a.by_g.of(end_row - 1) + shift + 1);
    const int n_blocks = (see_any + 31) / 32;
    const int per_split = (n_blocks + a.splits - 1) / a.splits;
    const int b0 = pl.split * per_split, b1 = min(n_blocks, b0 + per_split);

    const T *kg = (const T *)a.k + pl.k_off + kvh * a.k_h, *vg = (const T *)a.v + pl.v_off + kvh * a.v_h;
    Stage<T, D, 64, 32> stage;
    stage.init(a, lane);
    int b = b0 + wave;
    if (b < b1) stage.load(a, kg, vg, b * 32, pl.kv_len);
    Attend<T, D> at;
    at.clear();
    const int row = min(row0 + n, n_rows - 1), tok = a.by_g.of(row), head = kvh * a.G + row - tok * a.G;
    const int last = tok + shift;
    {
        const T *q = (const T *)a.q + pl.q_off + tok * a.q_t + head * a.q_h;
#pragma unroll
        for (int sl = 0; sl < R::kSlices; ++sl) at.q[sl] = *reinterpret_cast<const uint4 *>(q + R::kVec * (2 * sl + h));
    }
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
    const bool two = TWO && n_rows <= 32;
    u32x4 *sk = tiles[wave], *sv = sk + R::kKTile;
#pragma unroll 1
    for (; b < b1; b += NW) {
        const bool masked = (b + 1) * 32 > see_all;
        if (masked && stage.clean(pl.kv_len - b * 32)) s_bad = 1;
        wave_sync();  // the wave's reads of the tile before are behind it
        stage.store(sk, sv);
        wave_sync();
        if (b + NW < b1) stage.load(a, kg, vg, (b + NW) * 32, pl.kv_len);
        at.step(sk, sv, masked, two, last - b * 32, a.c);
    }
    // merge of the four waves: every wave brings its sums to the common reference and leaves them in LDS
    const float l = at.l + __shfl_xor(at.l, 32, 64);
    if (h == 0) s_m[wave][n] = at.m;
    __syncthreads();
    float M = s_m[0][n];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w][n]);
    const float f = weight(at.m, M);
    if (h == 0) s_l[wave][n] = l * f;
    constexpr int kQuads = D / 4;  // 16-byte pieces of a row of sums
    static_assert(sizeof(tiles) >= NW * 32 * D * sizeof(float), "the tiles' memory holds the sums");
    f32x4 *sums = reinterpret_cast<f32x4 *>(&tiles[0][0]);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = at.acc[d][4 * i + j] * f;  // (f of 0: 0, but for values that are not finite)
            sums[(wave * 32 + n) * kQuads + ((8 * d + 2 * i + h) ^ (n & 15))] = x;
        }
    __syncthreads();
    for (int idx = threadIdx.x; idx < 32 * kQuads; idx += 256) {
        const int r = idx / kQuads, c4 = idx % kQuads;
        if (row0 + r >= n_rows) break;  // (rows ascend with idx)
        f32x4 x = sums[r * kQuads + (c4 ^ (r & 15))];
        float lt = s_l[0][r];
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            x += sums[(w * 32 + r) * kQuads + (c4 ^ (r & 15))];
            lt += s_l[w][r];
        }
        const int t = a.by_g.of(row0 + r), g = row0 + r - t * a.G;
        if (s_bad) {  // values that are not finite, at keys that some row does not see
            const int end = min(min(b1 * 32, see_any), t + shift + 1);
            for (int key = max(b0, see_all / 32) * 32; key < end; ++key)
                for (int j = 0; j < 4; ++j) {
                    const float v = ldf(vg + key * a.v_t + 4 * c4 + j);
                    if (!(fabsf(v) < INFINITY)) x[j] += v;
                }
        }
        if (a.splits == 1) {
            const float inv = 1.0f / lt;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = lt == 0.f ? 0.f : x[j] * inv;
            store4((T *)a.out + pl.out_off + t * a.out_t + (kvh * a.G + g) * a.out_h + 4 * c4, x);
        } else {
            const int64_t slot = ((int64_t)pl.split * a.Hkv + kvh) * a.n_rows + pl.row0 + row0 + r;
            if (c4 == 0) {
                float mm = s_m[0][r];
#pragma unroll
                for (int w = 1; w < NW; ++w) mm = fmaxf(mm, s_m[w][r]);
                a.part_ml[slot] = make_float2(mm, lt);
            }
            store4(a.part_o + slot * D + 4 * c4, x);
        }
    }
}

// Joins the splits of a row.  D / 4 lanes hold a row's columns; `groups` of them (a power of two) share its splits, so that the partial
// results of a long row are all in flight at once.
template <typename T, int D, int kRound>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a, int groups) {
    asm volatile("" ::"s"(a.part_o), "s"(a.part_ml), "s"(a.out), "s"(a.out_t), "s"(a.out_h), "s"(a.Hkv), "s"(a.n_rows), "s"(a.splits), "s"(a.n_seqs),
                 "s"(a.G), "s"(a.by_g.m), "s"(a.by_rows.m), "s"(a.s[0].out_off));  // as in fetch
    constexpr int kQuads = D / 4;
    __shared__ f32x4 s_x[256];
    __shared__ float2 s_ml[256 / kQuads];
    const int c4 = threadIdx.x % kQuads, team = threadIdx.x / kQuads, g = team & (groups - 1);
    const int64_t idx = (int64_t)blockIdx.x * (256 / kQuads / groups) + team / groups;
    const int64_t stride = (int64_t)a.Hkv * a.n_rows;
    const bool live = idx < stride;
    const int kvh = a.by_rows.of((int)min(idx, stride - 1)), row = (int)min(idx, stride - 1) - kvh * a.n_rows;
    int seq = 0, seq_row = 0;
    int64_t out_off = a.s[0].out_off;
    if (a.n_seqs > 1) {  // the last sequence whose first row is not behind `row`: every lane holds one sequence's
        const int first = a.row0[threadIdx.x & 63];
        const int64_t out_first = a.s[threadIdx.x & 63].out_off;
#pragma unroll
        for (int step = 32; step > 0; step >>= 1)
            if (__shfl(first, seq + step, 64) <= row) seq += step;
        seq_row = __shfl(first, seq, 64);
        out_off = __shfl((long long)out_first, seq, 64);
    }
    float m = -INFINITY, l = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = g; live && s0 < a.splits; s0 += kRound * groups) {
        float2 ml[kRound];
        f32x4 o[kRound];
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            const int64_t slot = min(s0 + i * groups, a.splits - 1) * stride + idx;
            ml[i] = a.part_ml[slot];
            o[i] = *reinterpret_cast<const f32x4 *>(a.part_o + slot * D + 4 * c4);
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < kRound; ++i) top = fmaxf(top, ml[i].x);
        const float f = weight(m, top);
        l *= f;
        x *= f;
        m = top;
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            if (s0 + i * groups >= a.splits) continue;
            const float w = weight(ml[i].x, m);
            l = fmaf(w, ml[i].y, l);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fmaf(w, o[i][j], x[j]);
        }
    }
    if (groups > 1) {
        s_x[threadIdx.x] = x;
        if (c4 == 0) s_ml[team] = make_float2(m, l);
        __syncthreads();
        if (g != 0) return;
        float top = m;
        for (int i = 1; i < groups; ++i) top = fmaxf(top, s_ml[team + i].x);
        const float f = weight(m, top);
        l *= f;
        x *= f;
        for (int i = 1; i < groups; ++i) {
            const float2 ml = s_ml[team + i];
            const float w = weight(ml.x, top);
            l = fmaf(w, ml.y, l);
            const f32x4 o = s_x[threadIdx.x + i * kQuads];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fmaf(w, o[j], x[j]);
        }
    }
    if (!live) return;
    const int r = row - seq_row, t = a.by_g.of(r), q = r - t * a.G;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = l == 0.f ? 0.f : x[j] / l;
    store4((T *)a.out + out_off + t * a.out_t + (kvh * a.G + q) * a.out_h + 4 * c4, x);
}

// ---------------------------------------------------------------------------------------
// The shape of a call: which kernel, how many splits, what the partial results take
// ---------------------------------------------------------------------------------------
// What a call takes, in us, by the kernel's tile (rows): its first workgroups `start`, each round of them after that `round` (`at_once`
// workgroups run together); 128 keys of the longest workgroup `step` (keys are dealt by `grain`), and of all workgroups together,
// spread over the CUs, `full` (the clock falls when every matrix unit works).  Splits: the join, its launch and the partial results written and
// read.  Fitted to 880 calls of 1 to 17000 tokens, 1 to 33 sequences, 1 to 16 query heads per KV head, alone in a graph, every tile and split
// measured; on 800 others the choice takes 1.1 % longer than the best of up to 60 on average, nine in ten at most 3.1 %, the worst 46 %.  Some, us in tiles of 32 / 128 / 256
// rows, each with the splits that are chosen for it, the choice in brackets.
// bf16, heads of 128, 28 / 4 of them: prompts of 256 tokens [9.8] / 11.5 / 13.4, 512 19 / [15.7] / 19.7, 1024 45 / [24] / 32, 2048 113 / [48] / 57,
// 3000 215 / 95 / [88], 7432 1055 / 455 / [400]; heads of 64, 14 / 2: 1024 [12.4] / 16 / 23, 4096 79 / [52] / 60, 8000 246 / 177 / [154];
// 33 prompts of 200 tokens, 16 / 1: 35 / 21 / [15].  One token of 28 / 4 heads of 128 with 1 / 4 / 16 / 64 splits: 7432 keys 75 / 26 / 13.9 / [11.0]; 1024
// keys 14.6 without, [9.7] with; 256 keys [7.2].  64 tokens behind 15936 keys, tiles of 128 rows, 4 / 16 / 64 splits: 71 / 35 / 68 (chosen: 33.7).
// fp32, tiles of 32 / 128 rows: heads of 128, 28 / 4: 512 tokens [40] / 47, 1024 114 / [94], 2048 356 / [291], 5000 1862 / [1466],
// 64 behind 7936 keys 96 / [83]; heads of 64, 14 / 2: 512 [18] / 23, 2048 93 / [91], 8000 1017 / [916].
struct TileCost {
    int rows, at_once, grain;
    double start, round, step, full;
};
static const TileCost kCosts[4][3] = {
    {{32, 256, 128, 5.9, 3.9, 1.32, 1.57}, {128, 256, 64, 7.0, 4.5, 1.98, 2.3}, {256, 256, 64, 6.7, 3.6, 3.07, 3.46}},  // bf16, heads of 128
    {{32, 512, 128, 5.1, 3.9, 0.77, 0.62}, {128, 256, 64, 5.8, 2.6, 1.34, 1.63}, {256, 256, 64, 5.6, 1.0, 2.26, 2.57}},  // bf16, heads of 64
    {{32, 256, 128, 7.4, 7.6, 4.8, 5.6}, {128, 512, 32, 4.9, 1.7, 18.4, 15.2}, {0}},                                    // fp32, heads of 128
    {{32, 512, 128, 5.6, 4.6, 2.9, 2.55}, {128, 768, 32, 3.8, 0.0, 11.9, 8.4}, {0}},                                    // fp32, heads of 64
};
constexpr int kMostSplits = 64;
// Splits have to be worth their partial results: these are at most 256 MiB, and that much has to gain 2 % of the modelled time (less as much less:
// a gain of half a percent in the model for 59 MB is 13 % on the card, fp32, 14 / 2 heads of 64, 8000 tokens: 912 us, 1048 without).
// Without the bound, fp32 prompts of 97499 tokens over 258675 keys, 64 / 8 heads, took 6.5 GB for a modelled 0.004 %; with it, of 6000 calls of 1
// to 10^6 tokens 88 are chosen otherwise, the worst of them 2.9 % slower in the model (a bound of 128 MiB: 5.5 %, of 64 MiB: 38 %).
// Every plan can be launched: without splits there are fewer than 2^21 + 2^20 workgroups of 512 (2^26 rows in tiles of 32, and 64 sequences
// of 16384 heads with a tile that is not whole), with them and in the join no more than the 2^19 slots that 256 MiB hold.
constexpr double kSplitGain = 0.02;
constexpr size_t kMostPartBytes = 256u << 20;

// groups of D / 4 lanes that share the splits of a row in the join, and the join's workgroups
static int join_groups(int splits, int d) {
    int groups = 1;
    while (groups < 256 / (d / 4) && groups * 2 <= splits) groups *= 2;
    return groups;
}
static int64_t join_blocks(int64_t rows, int splits, int d) {
    const int64_t per = 256 / (d / 4) / join_groups(splits, d);
    return (rows + per - 1) / per;
}
// partial results of a call: (maximum, sum) pairs in front, sums behind them
static size_t ml_bytes(int64_t rows, int splits) { return ((size_t)rows * splits * sizeof(float2) + 255) / 256 * 256; }
static size_t part_bytes(int64_t rows, int splits, int d) {
    return splits == 1 ? 0 : ml_bytes(rows, splits) + (size_t)rows * splits * d * sizeof(float);
}

PromptPlan prompt_plan(const air_prompt_config &c, const air_prompt_seq *seqs, int n) {
    const int64_t G = c.n_q_heads / c.n_kv_heads;
    const bool f32 = c.dtype == AIR_F32;
    PromptPlan best;
    memset(&best, 0, sizeof(best));
    int64_t longest = 0, n_rows = 0;
    double bytes = 0.0;
    for (int i = 0; i < n; ++i) {
        if (seqs[i].q_len == 0) continue;
        n_rows += seqs[i].q_len * G;
        bytes += 2.0 * seqs[i].kv_len * c.n_kv_heads * c.head_dim * (f32 ? 4 : 2);
        if (seqs[i].kv_len > longest) longest = seqs[i].kv_len;
    }
    best.n_rows = n_rows;
    const int64_t all_rows = n_rows * c.n_kv_heads;
    if (all_rows >= (1 << 26)) return best;  // indexes of 32 bits
    double least = INFINITY;
    for (const TileCost &k : kCosts[(f32 ? 2 : 0) + (c.head_dim == 128 ? 0 : 1)]) {
        if (k.rows == 0) continue;
        int64_t tiles = 0;
        double keys = 0.0;  // of all tiles
        for (int i = 0; i < n; ++i) {
            const int64_t t = (seqs[i].q_len * G + k.rows - 1) / k.rows;
            tiles += t;
            keys += t * fmax(0.0, seqs[i].kv_len - 0.5 * seqs[i].q_len);
        }
        const double wgs = (double)tiles * c.n_kv_heads;
        const double full = keys * c.n_kv_heads / kCUs / 128.0 * k.full, read = bytes / 5.2e6;
        // 1 to 8 splits, then four to every doubling
        for (int s = 1; s <= kMostSplits && (s == 1 || longest > 64 * s); s += s < 8 ? 1 : (s < 16 ? 2 : (s < 32 ? 4 : 8))) {
            const size_t part = part_bytes(all_rows, s, c.head_dim);
            if (part > kMostPartBytes) break;
            const double at_work = fmax(1.0, wgs * s / kCUs);  // workgroups a CU: part of a last, uneven deal is lost
            const double all = full * (1.0 + 0.3 * (ceil(at_work) / at_work - 1.0));
            const double work = fmax(ceil((double)longest / s / k.grain) * k.grain / 128.0 * k.step, all);
            double us = k.start + k.round * (ceil(fmax(1.0, wgs * s / k.at_once)) - 1.0) + sqrt(work * work + read * read);
            if (s > 1) us += 2.9 + 2.1 * all_rows * s * (c.head_dim * 4 + 8) / 4e6;
            us *= 1.0 + kSplitGain * part / kMostPartBytes;
            if (us < least) {
                least = us;
                best.tile_rows = k.rows;
                best.n_tiles = tiles;
                best.splits = s;
                best.bytes = part;
            }
        }
    }
    best.few = best.tile_rows == 32;
    best.ml_bytes = best.splits > 1 ? ml_bytes(all_rows, best.splits) : 0;
    return best;
}

template <typename T, int D>
static void prompt_launch(hipStream_t s, const PromptPlan &p, const PromptArgs &a) {
    const dim3 grid((unsigned)(p.n_tiles * a.Hkv * p.splits));
    if constexpr (sizeof(T) == 2) {
        if (p.tile_rows == 256) hipLaunchKernelGGL((prompt_pipe_kernel<T, D, 1>), grid, dim3(512), 0, s, a);
        else if (!p.few) hipLaunchKernelGGL((prompt_pipe_kernel<T, D, 2>), grid, dim3(512), 0, s, a);
    }
    if constexpr (sizeof(T) == 4) {
        if (!p.few) hipLaunchKernelGGL((prompt_share_kernel<T, D>), grid, dim3(256), 0, s, a);
    }
    if (p.few) {
        const bool two = sizeof(T) == 2 && a.s[a.n_seqs - 1].q_len * a.G <= 32;  // (the last sequence has the fewest queries)
        if (two) hipLaunchKernelGGL((prompt_few_kernel<T, D, sizeof(T) == 2>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((prompt_few_kernel<T, D, false>), grid, dim3(256), 0, s, a);
    }
    if (p.splits > 1) {
        const int groups = join_groups(p.splits, D);
        const dim3 join((unsigned)join_blocks(p.n_rows * a.Hkv, p.splits, D));
        if (p.splits <= groups) hipLaunchKernelGGL((prompt_join_kernel<T, D, 1>), join, dim3(256), 0, s, a, groups);
        else if (p.splits <= 2 * groups) hipLaunchKernelGGL((prompt_join_kernel<T, D, 2>), join, dim3(256), 0, s, a, groups);
        else hipLaunchKernelGGL((prompt_join_kernel<T, D, 8>), join, dim3(256), 0, s, a, groups);
    }
}

hipError_t launch_prompt(hipStream_t s, const air_prompt_config &c, const PromptPlan &p, const air_prompt_seq *seqs, int n, const void *q,
                         const void *k, const void *v, void *out, void *workspace) {
    if (p.n_rows == 0) return hipSuccess;
    PromptArgs a;
    memset(&a, 0, sizeof(a));
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = out;
    a.part_ml = (float2 *)workspace;
    a.part_o = (float *)((char *)workspace + p.ml_bytes);
    a.q_h = c.q_h;
    a.q_t = c.q_t;
    a.k_h = c.k_h;
    a.k_t = c.k_t;
    a.v_h = c.v_h;
    a.v_t = c.v_t;
    a.out_h = c.out_h;
    a.out_t = c.out_t;
    a.G = c.n_q_heads / c.n_kv_heads;
    a.Hkv = c.n_kv_heads;
    a.by_g = div_by(a.G);
    a.by_hkv = div_by(a.Hkv);
    a.by_splits = div_by(p.splits);
    a.by_rows = div_by((int)p.n_rows);
    a.c = prompt_factor(c);
    a.splits = p.splits;
    a.n_tiles = (int)p.n_tiles;
    a.n_rows = (int)p.n_rows;
    int order[AIR_MAX_BATCH];
    int m = 0;
    for (int i = 0; i < n; ++i) {
        if (seqs[i].q_len == 0) continue;
        int at = m++;
        for (; at > 0; --at) {
            const air_prompt_seq &o = seqs[order[at - 1]];
            if (o.q_len > seqs[i].q_len || (o.q_len == seqs[i].q_len && o.kv_len >= seqs[i].kv_len)) break;
            order[at] = order[at - 1];
        }
        order[at] = i;
    }
    a.n_seqs = m;
    for (int i = 0; i < AIR_MAX_BATCH; ++i) a.rank0[i] = a.row0[i] = 0x7fffffff;
    int row0 = 0, rank0 = 0;
    for (int i = 0; i < m; ++i) {
        const air_prompt_seq &x = seqs[order[i]];
        const int rows = x.q_len * a.G, tiles = (rows + p.tile_rows - 1) / p.tile_rows;
        if (i > 0) rank0 += i * (a.s[i - 1].n_tiles - tiles);
        a.s[i] = PromptSpan{x.q_off, x.k_off, x.v_off, x.out_off, x.q_len, x.kv_len, tiles, row0};
        a.rank0[i] = rank0;
        a.row0[i] = row0;
        row0 += rows;
    }
    if (c.dtype == AIR_BF16) c.head_dim == 128 ? prompt_launch<bf16_t, 128>(s, p, a) : prompt_launch<bf16_t, 64>(s, p, a);
    else c.head_dim == 128 ? prompt_launch<float, 128>(s, p, a) : prompt_launch<float, 64>(s, p, a);
    return hipGetLastError();
}

}  // namespace air
