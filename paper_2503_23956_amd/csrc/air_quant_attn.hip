// air_quant_attn: attention over a cache held in 4 bits, and what every slot was attended to.
//
// The rows of one (sequence, KV head) are its queries times the G query heads that share the KV head, token by token: row t G + i.  A wave takes
// 64 slots at a time, for 16 rows.  S = Q K^T by 16 x 16 products of codes, one group at a time; each group's product is
// scaled by the slot's step, and one product more adds sum(q)_g lo_g (three bf16 terms of the sums).  A lane (n, c) then has the logits of slots
// 16 t + n, t = 0..3, and rows 4 c .. 4 c + 3.  Probabilities go through LDS in fp32, slot 16 t + n at place 4 n + t, and come back as the
// operand of the second product: lane (n, c) takes row n and 16 places from 16 c on, times the group's steps, as bf16 terms.  The codes
// of V go to LDS as they lie in memory and come back transposed (ds_read_b64_tr_b4: 16 slots of one element per lane), the places' order
// and that of the codes in an operand in the lanes' row addresses.  sum_j p_j lo_j is kept per lane, for its own slots.
//
// Waves share nothing until their ends: each deals itself every (4 splits)-th run of 64 slots, K requested one run ahead, and the four
// partial results of a workgroup are joined in LDS.
//
// Bound by the vector unit once a call fills the chip (codes into operands and factors into terms, for 16 rows at a time: 64 pairs of 12 rows over 16 k
// slots, heads of 128, bf16 52 us, 4.2 TB/s), below that by one pass over code that is new to the CU and by dependent accesses (two windows of 64 fp32 rows
// over 656 and 131 slots, heads of 64, with weights, 14.5 us in two launches).  32 rows a wave took 512 registers, one wave a SIMD: 8 x 4 pairs of 32
// rows over 4000 slots 34.2 against 24.7 us.
#include "air_quant_attn.h"

namespace air {

constexpr float kSlack = 8.0f;  // how far (base 2) a logit may lie above the reference of its row

template <int D, int GR, typename T>
struct QuantShape {
    static constexpr int NG = D / GR, KM = D / 32, KG = GR / 32, NT = D / 16;
    static constexpr bool kF32 = sizeof(T) == 4;
    static constexpr int QT = kF32 ? 3 : 1, PT = kF32 ? 3 : 2;  // bf16 terms of a query's elements; of p step
    static constexpr int kRowBytes = D / 2, kVStride = kRowBytes + 8;  // (rows of V in LDS: 8 bytes more, 32 rows on different banks)
    static constexpr int kPStride = 68;                                // floats
    static constexpr int kVBytes = kRun * kVStride, kPBytes = 16 * kPStride * 4, kSBytes = NG * kRun * 4;
    static constexpr int kWave = kVBytes + kPBytes + kSBytes;
    static constexpr int kLds = 4 * kWave > 4 * 16 * D * 4 + 4 * 16 * 8 ? 4 * kWave : 4 * 16 * D * 4 + 4 * 16 * 8;
};

__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// 16 rows of queries as operands: elements 32 m + 8 c .. + 7 of row n in lane (n, c), and the sums of their groups for the product with lo
template <int D, int GR, typename T>
struct QueryTile {
    using S = QuantShape<D, GR, T>;
    uint4 e[S::QT][S::KM], sums;

    uint4 raw[S::kF32 ? 2 * S::KM : 1];  // fp32: as they are read

    __device__ __forceinline__ void request(const QuantAttnArgs &a, int b, int h, int row, int rows) {
        const int c = (threadIdx.x >> 4) & 3;
        const bool real = row < rows;
        const int t = a.by_g.of(real ? row : 0), i = (real ? row : 0) - t * a.G;
        const T *q = static_cast<const T *>(a.q) + b * a.q_b + ((int64_t)h * a.G + i) * a.q_h + t * a.q_t + 8 * c;
#pragma unroll
        for (int m = 0; m < S::KM; ++m) {
            uint4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
            if (real) x = *reinterpret_cast<const uint4 *>(q + 32 * m);
            if (S::kF32 && real) y = *reinterpret_cast<const uint4 *>(q + 32 * m + 4);
            if (S::kF32) {
                raw[2 * m % (S::kF32 ? 2 * S::KM : 1)] = x;
                raw[(2 * m + 1) % (S::kF32 ? 2 * S::KM : 1)] = y;
            } else {
                e[0][m] = x;
            }
        }
    }
    // real: false makes it a row of zeros
    __device__ __forceinline__ void form(bool real) {
        const int c = (threadIdx.x >> 4) & 3;
        float part[S::NG] = {};
#pragma unroll
        for (int m = 0; m < S::KM; ++m) {
            float sum = 0.0f;
            if constexpr (S::kF32) {
                f32x4 u = __builtin_bit_cast(f32x4, raw[2 * m]), v = __builtin_bit_cast(f32x4, raw[2 * m + 1]);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    u[k] = real ? u[k] : 0.0f;
                    v[k] = real ? v[k] : 0.0f;
                }
                uint32_t w[4][S::QT];
                // (the order in which operand_of gives K's codes)
                split_pair<S::QT>(u[0], v[0], w[0]);
                split_pair<S::QT>(u[1], v[1], w[1]);
                split_pair<S::QT>(u[2], v[2], w[2]);
                split_pair<S::QT>(u[3], v[3], w[3]);
#pragma unroll
                for (int k = 0; k < S::QT; ++k) e[k][m] = uint4{w[0][k], w[1][k], w[2][k], w[3][k]};
                sum = ((u[0] + u[1]) + (u[2] + u[3])) + ((v[0] + v[1]) + (v[2] + v[3]));
            } else {
                uint32_t w[4] = {e[0][m].x, e[0][m].y, e[0][m].z, e[0][m].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    w[k] = real ? w[k] : 0u;
                    sum += __uint_as_float(w[k] << 16) + __uint_as_float(w[k] & 0xffff0000u);
                }
                e[0][m] = uint4{w[0], w[1], w[2], w[3]};
            }
            part[m / S::KG] += sum;
        }
        // lanes c = 2, 3 take the bias off: their operand has the steps in the place of lo
        uint32_t t3[S::NG][3];  // bf16 terms of the sums, in the low halves
#pragma unroll
        for (int g = 0; g < S::NG; ++g) {
            part[g] += __shfl_xor(part[g], 16, 64);
            part[g] += __shfl_xor(part[g], 32, 64);
            split_pair<3>(c < 2 ? part[g] : S::kF32 ? 0.0f : -kCodeBias * part[g], 0.0f, t3[g]);
        }
        // contraction indices 8 c .. 8 c + 7 of the product with lo, whose other operand repeats (lo_0, lo_1), (lo_2, lo_3): terms one and two
        // in even lanes c, three in odd ones (four groups); all three in even ones (two groups, one group beside a zero)
        const bool even = (c & 1) == 0;
        if (S::NG == 4) {
            const uint32_t a01 = t3[0][0] | t3[1 % S::NG][0] << 16, a23 = t3[2 % S::NG][0] | t3[3 % S::NG][0] << 16;
            const uint32_t b01 = t3[0][1] | t3[1 % S::NG][1] << 16, b23 = t3[2 % S::NG][1] | t3[3 % S::NG][1] << 16;
            const uint32_t c01 = t3[0][2] | t3[1 % S::NG][2] << 16, c23 = t3[2 % S::NG][2] | t3[3 % S::NG][2] << 16;
            sums = even ? uint4{a01, a23, b01, b23} : uint4{c01, c23, 0, 0};
        } else {
            uint32_t w[3];
#pragma unroll
            for (int k = 0; k < 3; ++k) w[k] = S::NG == 2 ? t3[0][k] | t3[S::NG - 1][k] << 16 : t3[0][k] & 0xffffu;
            sums = even ? uint4{w[0], w[1], w[2], 0} : uint4{0, 0, 0, 0};
        }
    }
};

// the other operand of the product with sum(q), as the queries' sums lie: slot n's lo; its steps in lanes c = 2, 3
template <int NG>
__device__ __forceinline__ uint4 lo_operand(const Words<NG> &pairs) {
    const uint32_t pick = threadIdx.x & 32 ? (NG == 1 ? 0x0c0c0302u : 0x07060302u) : (NG == 1 ? 0x0c0c0100u : 0x05040100u);
    const uint32_t a = __builtin_amdgcn_perm(pairs.w[1 % NG], pairs.w[0], pick);
    if (NG < 4) return uint4{a, a, a, a};
    const uint32_t b = __builtin_amdgcn_perm(pairs.w[3 % NG], pairs.w[2 % NG], pick);
    return uint4{a, b, a, b};
}
template <bool F32>
__device__ __forceinline__ uint4 key_operand(uint32_t codes) {
    return F32 ? operand_of(codes) : biased_of(codes);
}

// logits (before the factor) of rows 4 c .. 4 c + 3 at slot n of a tile
template <int D, int GR, typename T>
__device__ __forceinline__ f32x4 logits(const QueryTile<D, GR, T> &q, const uint4 (&k)[D / 32], const Words<D / GR> &pairs, const uint4 &lo) {
    using S = QuantShape<D, GR, T>;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 s = mma<bf16_t>(q.sums, lo, zero);
#pragma unroll
    for (int g = 0; g < S::NG; ++g) {
        f32x4 x = zero;
#pragma unroll
        for (int j = 0; j < S::KG; ++j)
#pragma unroll
            for (int k3 = 0; k3 < S::QT; ++k3) x = mma<bf16_t>(q.e[k3][g * S::KG + j], k[g * S::KG + j], x);
        const float step = step_of(pairs.w[g]);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = fmaf(step, x[i], s[i]);
    }
    return s;
}

// ---- references.  A row's reference is a number `ref` in the base-2 domain, the same in all of its exponents 2^(s c - ref): that it is a rounded
// maximum cancels when the row is divided by its sum.  Beyond kHuge the exponents' own products are rounded like it: equal logits
// stay equal.
constexpr float kHuge = 0x1p20f;
__device__ __forceinline__ float exponent(float s, float c, float ref, bool huge) {
    if (__builtin_expect(huge, 0)) {
        float x = s * c;
        asm volatile("" : "+v"(x));  // (rounded by itself)
        return x - ref;
    }
    return fmaf(s, c, -ref);
}
// the logit above which a reference `top`, of the logit `high`, is raised: kSlack further on, to 0.2 (base 2); at once beyond kHuge
__device__ __forceinline__ float limit_of(float high, float top, float c) {
    return fabsf(top) > kHuge ? high : (top + kSlack) * (1.0f / c);
}

// What a wave requests ahead: N tiles of 16 slots
template <int D, int GR, int N = 4>
struct KeyRun {
    Words<D / 32> code[N];
    Words<D / GR> pair[N];
    // held: slots held, or the capacity where the others are masked later; from there on they are read as the last one
    __device__ __forceinline__ void load(const uint8_t *codes, const uint32_t *pairs, int slot0, int held) {
        const int n = threadIdx.x & 15, c = (threadIdx.x >> 4) & 3;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int at = slot0 + 16 * t + n, slot = at < held ? at : held - 1;
            code[t] = load_words<D / 32>(codes + ((uint32_t)slot * (D / 2) + D / 8 * c));
            pair[t] = load_words<D / GR>(reinterpret_cast<const uint8_t *>(pairs) + (uint32_t)slot * (D / GR * 4));
        }
    }
};
template <int D, int GR>
struct ValueRun {
    static constexpr int kPieces = D / 32;  // 16-byte pieces of a row; of a lane
    uint4 code[kPieces];
    Words<D / GR> pair[4];
    __device__ __forceinline__ void load(const uint8_t *codes, const uint32_t *pairs, int slot0, int held) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int at = slot0 + i * (64 / kPieces) + lane / kPieces, slot = at < held ? at : held - 1;
            code[i] = *reinterpret_cast<const uint4 *>(codes + ((uint32_t)slot * (D / 2) + 16 * (lane % kPieces)));
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int at = slot0 + 16 * t + (lane & 15), slot = at < held ? at : held - 1;
            pair[t] = load_words<D / GR>(reinterpret_cast<const uint8_t *>(pairs) + (uint32_t)slot * (D / GR * 4));
        }
    }
};

template <int D, int GR, typename T>
__global__ __launch_bounds__(256, 2) void quant_attn_kernel(QuantAttnArgs a) {
    using S = QuantShape<D, GR, T>;
    constexpr int NG = S::NG;
    __shared__ __align__(16) uint8_t lds[S::kLds];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, c = lane >> 4;
    const int pair = blockIdx.y, block = a.by_splits.of(blockIdx.x), split = blockIdx.x - block * a.splits;
    // requested before the sequence's length is there: queries, the wave's first run of keys (whatever lies in it)
    const size_t base = (size_t)pair * a.capacity;
    const uint8_t *kc = a.kc + base * (D / 2), *vc = a.vc + base * (D / 2);
    const uint32_t *ks = a.ks + base * NG, *vs = a.vs + base * NG;
    const int row0 = block * 16;
    int u = split * 4 + wave;
    const QuantSpan sp(a, pair);
    KeyRun<D, GR> key;
    QueryTile<D, GR, T> q;
    q.request(a, sp.b, sp.h, row0 + n, a.n_rows);
    if (u * kRun < a.capacity) key.load(kc, ks, u * kRun, a.capacity);
    if (row0 >= sp.rows) return;
    const int row_end = row0 + 16 < sp.rows ? row0 + 16 : sp.rows;
    const int most = sp.seen(a, row_end - 1), least = sp.seen(a, row0);

    uint8_t *vb = lds + wave * S::kWave;
    float *pb = reinterpret_cast<float *>(vb + S::kVBytes), *sb = reinterpret_cast<float *>(vb + S::kVBytes + S::kPBytes);
    // rows of V that the lane gives to the transposed reads: place x of a group of 16 lanes is slot 16 (k & 3) + (k >> 2) with
    // k = 16 c + 8 (x >> 3) + the place of code x & 7 in an operand
    const int k_of = 16 * c + (n & 8) + ((n & 1) ? 4 + ((n & 7) >> 1) : (n & 7) >> 1);
    const uint8_t *v_read = vb + (16 * (k_of & 3) + (k_of >> 2)) * S::kVStride;

    q.form(row0 + n < sp.rows);

    f32x4 acc[S::NT];
    float m[4], l[4], al[4][NG];
    float limit[4];  // the logit above which the reference is raised
    bool huge = false;
#pragma unroll
    for (int i = 0; i < S::NT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = limit[i] = -INFINITY;
        l[i] = 0.0f;
#pragma unroll
        for (int g = 0; g < NG; ++g) al[i][g] = 0.0f;
    }

    const int runs = (most + kRun - 1) / kRun, stride = 4 * a.splits;
    for (; u < runs; u += stride) {
        ValueRun<D, GR> val;  // (on its way during the first product)
        val.load(vc, vs, u * kRun, sp.held);
        const bool masked = (u + 1) * kRun > least;
        const int next = u + stride < runs ? u + stride : u;
        // ---- logits
        f32x4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            uint4 k[S::KM];
#pragma unroll
            for (int i = 0; i < S::KM; ++i) k[i] = key_operand<S::kF32>(key.code[t].w[i]);
            const uint4 lo = lo_operand<NG>(key.pair[t]);
            s[t] = logits<D, GR, T>(q, k, key.pair[t], lo);
            if (NG == 4) __builtin_amdgcn_sched_barrier(0);  // (operands of all four tiles at once do not fit the registers)
        }
        key.load(kc, ks, next * kRun, a.capacity);
        // ---- V to LDS, its steps beside it (group g by lanes c = g)
        wave_sync();
#pragma unroll
        for (int i = 0; i < S::KM; ++i) {
            uint2 *to = reinterpret_cast<uint2 *>(vb + (i * (64 / S::KM) + lane / S::KM) * S::kVStride + 16 * (lane % S::KM));
            to[0] = uint2{val.code[i].x, val.code[i].y};
            to[1] = uint2{val.code[i].z, val.code[i].w};
        }
        Words<NG> (&vp)[4] = val.pair;
        if (masked) {  // slots that are not held: no step, no lo, whatever lies there
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int g = 0; g < NG; ++g) vp[t].w[g] = u * kRun + 16 * t + n < sp.held ? vp[t].w[g] : 0u;
        }
        if (c < NG) {
            f32x4 st;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                uint32_t w = vp[t].w[0];
#pragma unroll
                for (int g = 1; g < NG; ++g) w = c == g ? vp[t].w[g] : w;
                st[t] = step_of(w);
            }
            *reinterpret_cast<f32x4 *>(sb + c * kRun + 4 * n) = st;
        }
        // ---- softmax against a running reference, raised when a logit lies more than kSlack above it
        if (masked) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = row0 + 4 * c + i, seen = row < sp.rows ? sp.seen(a, row) : sp.held;
#pragma unroll
                for (int t = 0; t < 4; ++t) s[t][i] = u * kRun + 16 * t + n < seen ? s[t][i] : -INFINITY;
            }
        }
        bool raise = false;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) raise = raise || s[t][i] > limit[i];
        if (__any(raise)) {
            bool big = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float high = max16(fmaxf(fmaxf(s[0][i], s[1][i]), fmaxf(s[2][i], s[3][i]))), top = high * a.c;
                const bool up = top > m[i];
                const float f = up ? __builtin_amdgcn_exp2f(m[i] - top) : 1.0f;
                m[i] = up ? top : m[i];
                if (up) limit[i] = limit_of(high, top, a.c);
                big = big || fabsf(finite_or_zero(m[i])) > kHuge;
                l[i] *= f;
#pragma unroll
                for (int g = 0; g < NG; ++g) al[i][g] *= f;
#pragma unroll
                for (int j = 0; j < S::NT; ++j) acc[j][i] *= f;
            }
            huge = huge || __any(big);
        }
        wave_sync();  // (the probabilities of the tile in front have been read)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float ref = finite_or_zero(m[i]);
            f32x4 p;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                p[t] = __builtin_amdgcn_exp2f(exponent(s[t][i], a.c, ref, huge));
                l[i] += p[t];
            }
            if (masked) {
                // a lo of NaN counts only where the row sees it
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int g = 0; g < NG; ++g) al[i][g] = fmaf(p[t], s[t][i] == -INFINITY ? 0.0f : lo_of(vp[t].w[g]), al[i][g]);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int g = 0; g < NG; ++g) al[i][g] = fmaf(p[t], lo_of(vp[t].w[g]), al[i][g]);
            }
            *reinterpret_cast<f32x4 *>(pb + (4 * c + i) * S::kPStride + 4 * n) = p;
        }
        wave_sync();
        // ---- second product: two halves of 32 places
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float *pr = pb + n * S::kPStride + 16 * c + 8 * j;
            const f32x4 p0 = *reinterpret_cast<const f32x4 *>(pr), p1 = *reinterpret_cast<const f32x4 *>(pr + 4);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float *sr = sb + g * kRun + 16 * c + 8 * j;
                const f32x4 s0 = *reinterpret_cast<const f32x4 *>(sr), s1 = *reinterpret_cast<const f32x4 *>(sr + 4);
                uint32_t w[4][S::PT];
                split_pair<S::PT>(p0[0] * s0[0], p0[1] * s0[1], w[0]);
                split_pair<S::PT>(p0[2] * s0[2], p0[3] * s0[3], w[1]);
                split_pair<S::PT>(p1[0] * s1[0], p1[1] * s1[1], w[2]);
                split_pair<S::PT>(p1[2] * s1[2], p1[3] * s1[3], w[3]);
#pragma unroll
                for (int x = 0; x < GR / 16; ++x) {
                    const int tile = g * (GR / 16) + x;
                    typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
                    const i32x2 code = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(v_read + 8 * tile));
                    const uint4 v = operand_of((uint32_t)(j ? code.y : code.x));
#pragma unroll
                    for (int k = 0; k < S::PT; ++k) acc[tile] = mma<bf16_t>(uint4{w[0][k], w[1][k], w[2][k], w[3][k]}, v, acc[tile]);
                }
            }
        }
    }

    // ---- the lanes' sums, then the four waves'
    __syncthreads();
    float *ob = reinterpret_cast<float *>(lds);  // [wave][row][D]
    float2 *mlb = reinterpret_cast<float2 *>(lds + 4 * 16 * D * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        l[i] = sum16(l[i]);
#pragma unroll
        for (int g = 0; g < NG; ++g) al[i][g] = sum16(al[i][g]);
#pragma unroll
        for (int j = 0; j < S::NT; ++j) ob[(wave * 16 + 4 * c + i) * D + 16 * j + n] = acc[j][i] + al[i][j / (GR / 16)];
        if (n == 0) mlb[wave * 16 + 4 * c + i] = float2{m[i], l[i]};
    }
    __syncthreads();
    const int x = threadIdx.x >> 4, row = row0 + x;
    if (row < sp.rows) {
        float top = -INFINITY, f[4], sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, mlb[w * 16 + x].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = part_weight(mlb[w * 16 + x].x, mlb[w * 16 + x].y, top);
            sum += f[w] * mlb[w * 16 + x].y;
        }
        const size_t part = ((size_t)pair * a.splits + split) * a.n_rows + row;
        if (a.part_ml && n == 0) a.part_ml[part] = float2{top, sum};
        if (a.splits > 1 || a.out) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const int t = a.by_g.of(row);
            T *to = static_cast<T *>(a.out) + sp.b * a.out_b + ((int64_t)sp.h * a.G + row - t * a.G) * a.out_h + t * a.out_t;
#pragma unroll
            for (int j = 0; j < S::NT; ++j) {
                float o = 0.0f;
#pragma unroll
                for (int w = 0; w < 4; ++w) o = fmaf(f[w], ob[(w * 16 + x) * D + 16 * j + n], o);
                if (a.splits > 1) a.part_o[part * D + 16 * j + n] = o;
                else put(to + 16 * j + n, o * inv);
            }
        }
    }
}

// ST: tiles of 16 slots of a wave, four or, where that would be few waves, one
template <int D, int GR, typename T, int TILES, int ST>
__global__ __launch_bounds__(256, 2) void quant_finish_kernel(QuantAttnArgs a) {
    using S = QuantShape<D, GR, T>;
    constexpr int kSlots = 16 * ST;
    constexpr int NG = S::NG, kOperands = S::QT * S::KM + 1;
    __shared__ uint4 ql[TILES][kOperands][64];
    __shared__ float2 rl[TILES * 16];  // (maximum, 1 / sum) of the rows
    __shared__ float4 jl[256 + 8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, c = lane >> 4;
    const int pair = blockIdx.y;
    const QuantSpan sp(a, pair);
    const size_t base = (size_t)pair * a.capacity;
    const uint8_t *kc = a.kc + base * (D / 2);
    const uint32_t *ks = a.ks + base * NG;
    const int stride = gridDim.x * 4, u0 = blockIdx.x * 4 + wave;
    // what is needed first is requested before the sequence's length is there
    static_assert(TILES <= 4, "a wave forms one tile of queries");
    KeyRun<D, GR, ST> key;
    QueryTile<D, GR, T> own;
    RowReference refs[TILES];  // 16 lanes a row
    const auto request = [&](int row0, int rows) {
        if (wave < TILES) own.request(a, sp.b, sp.h, row0 + 16 * wave + n, rows);
#pragma unroll
        for (int r = 0; r < TILES; ++r) refs[r].request(a, pair, row0 + 16 * r + (threadIdx.x >> 4), rows, n);
    };
    if (a.weights) {
        if (u0 * kSlots < a.capacity) key.load(kc, ks, u0 * kSlots, a.capacity);
        if (ST == 1) request(0, a.n_rows);  // (in larger calls the registers are needed in between)
    }
    if (sp.rows == 0) return;
    const int runs = a.weights ? (sp.held + kSlots - 1) / kSlots : 0;
    if (a.splits > 1 && a.out) join_rows<D, T>(a, sp, pair, jl);
    if ((int)blockIdx.x * 4 >= runs) return;

    float *weights = a.weights + base;
    for (int row0 = 0; row0 < sp.rows; row0 += 16 * TILES) {
        const int left = (sp.rows - row0 + 15) / 16, tiles = left < TILES ? left : TILES;
        if (ST > 1 || row0 > 0) request(row0, sp.rows);
        __syncthreads();
        if (wave < TILES) {
            own.form(row0 + 16 * wave + n < sp.rows);
#pragma unroll
            for (int k = 0; k < S::QT; ++k)
#pragma unroll
                for (int i = 0; i < S::KM; ++i) ql[wave][k * S::KM + i][lane] = own.e[k][i];
            ql[wave][kOperands - 1][lane] = own.sums;
        }
#pragma unroll
        for (int r = 0; r < TILES; ++r) {
            const int x = 16 * r + (threadIdx.x >> 4);
            refs[r].form(n, row0 + x < sp.rows, rl + x);
        }
        __syncthreads();
        for (int u = u0; u < runs; u += stride) {
            uint4 k[ST][S::KM], lo[ST];
            Words<NG> pairs[ST];
#pragma unroll
            for (int t = 0; t < ST; ++t) {
#pragma unroll
                for (int i = 0; i < S::KM; ++i) k[t][i] = key_operand<S::kF32>(key.code[t].w[i]);
                lo[t] = lo_operand<NG>(key.pair[t]);
                pairs[t] = key.pair[t];
            }
            // the run after this one; behind the last one the first again, for the next rows
            key.load(kc, ks, (u + stride < runs ? u + stride : u0) * kSlots, a.capacity);
            float w[ST] = {};
            for (int r = 0; r < tiles; ++r) {
                QueryTile<D, GR, T> q;
#pragma unroll
                for (int k3 = 0; k3 < S::QT; ++k3)
#pragma unroll
                    for (int i = 0; i < S::KM; ++i) q.e[k3][i] = ql[r][k3 * S::KM + i][lane];
                q.sums = ql[r][kOperands - 1][lane];
                float2 ref[4];
                int seen[4];
                const int row = row0 + 16 * r + 4 * c;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ref[i] = rl[16 * r + 4 * c + i];
                    seen[i] = row + i < sp.rows ? sp.seen(a, row + i) : 0;
                }
                const bool huge = __any(fmaxf(fmaxf(fabsf(ref[0].x), fabsf(ref[1].x)), fmaxf(fabsf(ref[2].x), fabsf(ref[3].x))) > kHuge);
#pragma unroll
                for (int t = 0; t < ST; ++t) {
                    const f32x4 s = logits<D, GR, T>(q, k[t], pairs[t], lo[t]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = __builtin_amdgcn_exp2f(exponent(s[i], a.c, ref[i].x, huge)) * ref[i].y;
                        w[t] += u * kSlots + 16 * t + n < seen[i] ? p : 0.0f;
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < ST; ++t) {
                w[t] += __shfl_xor(w[t], 16, 64);
                w[t] += __shfl_xor(w[t], 32, 64);
                const int slot = u * kSlots + 16 * t + n;
                if (c == t && slot < sp.held) weights[slot] += w[t];
            }
        }
    }
}

// ---------------------------------------------------------------------------------------
// At most eight rows (a token of up to eight query heads per KV head, a few tokens of fewer), 32 slots at a time: half of a 16 x 16 product's
// rows would be idle.  The first product's are; its logits of slots 16 .. 31 of a run then move to the idle lanes, so that softmax, sums and steps are
// formed once per logit: lane (n, c) has rows 4 (c & 1) + i at slot 16 (c >> 1) + n.  The factors p step are formed there, of two slots and
// two rows after an exchange between lanes n and n ^ 1, and go through LDS as bf16 terms (two, or with fp32 three): the first one in rows 0 .. 7 of
// the second product's operand, the second one in rows 8 .. 15, joined at the end, the third one in a product of its own.  (One fp16 number would be
// 10 % fewer instructions, but its range needs a unit, and next to a value 2^20 times as large, whatever that weighs, the others' codes
// would be lost.)
//
// Small calls are bound by the chain of dependent accesses and by the instructions of one pass over code that is new to the CU: one token over 7432
// slots, 28 / 4 heads of 128, 12.2 us with the launch that joins 59 splits (13.8 with 64 slots at a time: twice the code of a pass, 200 registers in place of
// 162); queries, first keys and new rows are requested before the length is there.  Large ones are bound by memory: 16 tokens over 14 to 17 k slots,
// 64 / 8 heads of 128, with weights, 111 us, 88 of them here (404 MB with the logits kept, 4.6 TB/s).
//
// The wave whose run has slots that the call appends writes them, and takes them from LDS into what it has read of the run.
// ---------------------------------------------------------------------------------------
template <int D, int GR, typename T>
struct FewShape {
    using S = QuantShape<D, GR, T>;
    static constexpr int kWStride = 80, kWRows = S::kF32 ? 24 : 16;  // bytes: 32 places of 16 bits and 16 more, 16 rows on different banks
    static constexpr int kVBytes = kFewRun * S::kVStride, kWBytes = S::NG * kWRows * kWStride, kWave = kVBytes + kWBytes;
    static constexpr int kEnd = 4 * 16 * D * 4 + 4 * 16 * 8, kLds = 4 * kWave > kEnd ? 4 * kWave : kEnd;
};

// (x of lanes 0 .. 31, y of lanes 0 .. 31)
__device__ __forceinline__ float lower_halves(float x, float y) {
    return __uint_as_float(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false)[0]);
}
// x of the lane beside: n ^ 1
__device__ __forceinline__ float swap_pairs(float x) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xf, 0xf, true));
}
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// What the call appends, in codes, for the wave whose run has its slots: it does not wait for the cache's memory to have them
template <int D, int GR>
struct alignas(16) NewRow {
    uint32_t k[D / 8], v[D / 8], kp[D / GR], vp[D / GR];
};
// rows of slots slot0 .. slot0 + 31 into the cache and, token by token of the call, into `rows`.  first: the eight elements of K and V that the lane
// has requested of token lane / (D / 8)
template <int D, int GR, typename T>
__device__ __forceinline__ void append_run(const QuantAttnArgs &a, const QuantSpan &sp, int slot0, const float (&first)[2][8], NewRow<D, GR> *rows) {
    constexpr int kLanes = D / 8, kRows = 64 / kLanes;
    const int lane = threadIdx.x & 63, p = lane & (kLanes - 1);
    for (int t0 = 0; t0 < sp.count; t0 += kRows) {
        const int t = t0 + lane / kLanes;
        const int64_t slot = (int64_t)sp.held_before + t;
        if (t >= sp.count || slot < slot0 || slot >= slot0 + kFewRun || slot >= sp.held) continue;
        const int64_t cell = ((int64_t)sp.b * a.Hkv + sp.h) * a.capacity + slot;
        float x[2][8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (t0 > 0) {
                load8(static_cast<const T *>(a.rows.rows[i]) + sp.b * a.rows.row_b[i] + sp.h * a.rows.row_h[i] + t * a.rows.row_t[i] + 8 * p, x[i]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] = first[i][e];
            }
        }
        uint32_t pair[2];
        const uint32_t k = codes_of<GR, true>(x[0], pair[0]), v = codes_of<GR, false>(x[1], pair[1]);
        reinterpret_cast<uint32_t *>(a.rows.codes[0] + cell * (D / 2))[dword_of<D, true>(p)] = rows[t].k[dword_of<D, true>(p)] = k;
        reinterpret_cast<uint32_t *>(a.rows.codes[1] + cell * (D / 2))[p] = rows[t].v[p] = v;
        if ((p & (GR / 8 - 1)) == 0) {
            a.rows.scales[0][cell * (D / GR) + p / (GR / 8)] = rows[t].kp[p / (GR / 8)] = pair[0];
            a.rows.scales[1][cell * (D / GR) + p / (GR / 8)] = rows[t].vp[p / (GR / 8)] = pair[1];
        }
        if (p == 0) {
            if (a.rows.positions) a.rows.positions[cell] = a.rows.first[sp.b] + t;
            if (a.rows.weights) a.rows.weights[cell] = 0.0f;
        }
    }
}

template <int D, int GR, typename T>
__global__ __launch_bounds__(256, 2) void quant_few_kernel(QuantAttnArgs a) {
    using S = QuantShape<D, GR, T>;
    using F = FewShape<D, GR, T>;
    constexpr int NG = S::NG;
    __shared__ __align__(16) uint8_t lds[F::kLds];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, c = lane >> 4, upper = c >> 1, rc = c & 1;
    __shared__ NewRow<D, GR> news[4][kFewRows];
    const int pair = blockIdx.y, split = blockIdx.x, b = a.by_hkv.of(pair), h = pair - b * a.Hkv;

    // requested before the sequence's length is there: the wave's first run (whatever lies in it), queries, new rows
    const size_t base = (size_t)pair * a.capacity;
    const uint8_t *kc = a.kc + base * (D / 2), *vc = a.vc + base * (D / 2);
    const uint32_t *ks = a.ks + base * NG, *vs = a.vs + base * NG;
    const int stride = 4 * a.splits;
    int u = split * 4 + wave;
    KeyRun<D, GR, 2> key;
    QueryTile<D, GR, T> q;
    q.request(a, b, h, n, a.n_rows);
    if (u * kFewRun < a.capacity) key.load(kc, ks, u * kFewRun, a.capacity);
    const bool append = a.rows.rows[0] != nullptr;
    float first[2][8] = {};
    if (append && lane / (D / 8) < a.n_tokens) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            load8(static_cast<const T *>(a.rows.rows[i]) + b * a.rows.row_b[i] + h * a.rows.row_h[i] + lane / (D / 8) * a.rows.row_t[i] + 8 * (lane & (D / 8 - 1)), first[i]);
    }
    const QuantSpan sp(a, pair);
    if (sp.rows == 0) return;
    q.form(n < sp.rows);
    const int most = sp.seen(a, sp.rows - 1), least = sp.seen(a, 0);
    const int runs = (most + kFewRun - 1) / kFewRun;
    int new_run = -1;  // the wave's run with slots that the call appends: at most two runs have any
    if (append) {
        const int r0 = sp.held_before < 0 ? 0 : sp.held_before / kFewRun;
        for (int r = r0; r < runs && r < r0 + 2; ++r)
            if (r - a.by_stride.of(r) * stride == u) new_run = r;
        if (new_run >= 0) append_run<D, GR, T>(a, sp, new_run * kFewRun, first, news[wave]);
    }

    uint8_t *vb = lds + wave * F::kWave, *wb = vb + F::kVBytes;
    // rows of V that the lane gives to the transposed reads: slot 8 c + the place of code n & 7 in an operand, of two tiles of 16 elements
    const uint8_t *v_read = vb + (8 * c + ((n & 1) ? 4 + ((n & 7) >> 1) : (n & 7) >> 1)) * S::kVStride + (n & 8);

    f32x4 acc[S::NT];
    float m[4], limit[4], l[4], al[4][NG];
    bool huge = false;
#pragma unroll
    for (int i = 0; i < S::NT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = limit[i] = -INFINITY;
        l[i] = 0.0f;
#pragma unroll
        for (int g = 0; g < NG; ++g) al[i][g] = 0.0f;
    }

    for (; u < runs; u += stride) {
        // V on its way during the first product: the codes, and the pairs of the lane's slot
        constexpr int kPieces = D / 32, kLoads = kPieces / 2;
        uint4 code[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = u * kFewRun + i * (64 / kPieces) + lane / kPieces, slot = at < a.capacity ? at : a.capacity - 1;
            code[i] = *reinterpret_cast<const uint4 *>(vc + ((uint32_t)slot * (D / 2) + 16 * (lane % kPieces)));
        }
        const int own = u * kFewRun + 16 * upper + n;
        Words<NG> vp = load_words<NG>(reinterpret_cast<const uint8_t *>(vs) + (uint32_t)(own < a.capacity ? own : a.capacity - 1) * (NG * 4));
        if (u == new_run) {  // slots of the call's own rows: what was read there is not them yet
            for (int t = 0; t < sp.count; ++t) {
                const int slot = sp.held_before + t - u * kFewRun;
                if (slot < 0 || slot >= kFewRun) continue;
                const NewRow<D, GR> &row = news[wave][t];
                wave_sync();
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (slot == 16 * x + n) {
                        key.code[x] = load_words<D / 32>(row.k + D / 32 * c);
                        key.pair[x] = load_words<NG>(row.kp);
                    }
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    if (slot == i * (64 / kPieces) + lane / kPieces) code[i] = *reinterpret_cast<const uint4 *>(row.v + 4 * (lane % kPieces));
                if (slot == 16 * upper + n) vp = load_words<NG>(row.vp);
            }
        }
        const bool masked = (u + 1) * kFewRun > least;
        const int next = u + stride < runs ? u + stride : u;
        // ---- logits
        f32x4 s4[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint4 k[S::KM];
#pragma unroll
            for (int i = 0; i < S::KM; ++i) k[i] = key_operand<S::kF32>(key.code[t].w[i]);
            s4[t] = logits<D, GR, T>(q, k, key.pair[t], lo_operand<NG>(key.pair[t]));
        }
        key.load(kc, ks, next * kFewRun, a.capacity);
        f32x4 s;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = lower_halves(s4[0][i], s4[1][i]);
        if (masked) {
#pragma unroll
            for (int g = 0; g < NG; ++g) vp.w[g] = own < sp.held ? vp.w[g] : 0u;  // (whatever lies there)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 4 * rc + i, seen = row < sp.rows ? sp.seen(a, row) : sp.held;
                s[i] = own < seen ? s[i] : -INFINITY;
            }
        }
        if (a.kept) a.kept[((size_t)pair * a.max_runs + u) * 64 + lane] = float4{s[0], s[1], s[2], s[3]};
        // ---- V to LDS
        wave_sync();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            uint2 *to = reinterpret_cast<uint2 *>(vb + (i * (64 / kPieces) + lane / kPieces) * S::kVStride + 16 * (lane % kPieces));
            to[0] = uint2{code[i].x, code[i].y};
            to[1] = uint2{code[i].z, code[i].w};
        }
        // ---- softmax against a running reference, raised when a logit lies more than kSlack above it
        bool raise = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) raise = raise || s[i] > limit[i];
        if (__any(raise)) {
            bool big = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float high = max_halves(max16(s[i])), top = high * a.c;
                const bool up = top > m[i];
                const float f = up ? __builtin_amdgcn_exp2f(m[i] - top) : 1.0f;
                m[i] = up ? top : m[i];
                if (up) limit[i] = limit_of(high, top, a.c);
                big = big || fabsf(finite_or_zero(m[i])) > kHuge;
                l[i] *= f;
#pragma unroll
                for (int g = 0; g < NG; ++g) al[i][g] *= f;
#pragma unroll
                for (int j = 0; j < S::NT; ++j) acc[j][i] *= f;
            }
            huge = huge || __any(big);
        }
        bool odd = false;  // a lo of NaN in a run that some row does not see all of: it counts only where the row sees it
        if (masked) {
#pragma unroll
            for (int g = 0; g < NG; ++g) odd = odd || (vp.w[g] & 0x7f80u) == 0x7f80u;
            odd = __any(odd);
        }
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = __builtin_amdgcn_exp2f(exponent(s[i], a.c, finite_or_zero(m[i]), huge));
            l[i] += p[i];
        }
        if (__builtin_expect(odd, 0)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int g = 0; g < NG; ++g) al[i][g] = fmaf(p[i], s[i] == -INFINITY ? 0.0f : lo_of(vp.w[g]), al[i][g]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int g = 0; g < NG; ++g) al[i][g] = fmaf(p[i], lo_of(vp.w[g]), al[i][g]);
        }
        // lanes n and n + 1 share their slots: the even one takes rows 0 and 1 of both, the odd one 2 and 3
        const bool second = n & 1;
        float two[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float other = swap_pairs(second ? p[i] : p[i + 2]);
            two[i][0] = second ? other : p[i];
            two[i][1] = second ? p[i + 2] : other;
        }
        uint8_t *to = wb + (4 * rc + (second ? 2 : 0)) * F::kWStride + 32 * upper + 2 * (n & 14);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const float own_step = step_of(vp.w[g]), other = swap_pairs(own_step), step[2] = {second ? other : own_step, second ? own_step : other};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t w[S::PT];
                split_pair<S::PT>(two[i][0] * step[0], two[i][1] * step[1], w);
#pragma unroll
                for (int k = 0; k < S::PT; ++k) *reinterpret_cast<uint32_t *>(to + (g * F::kWRows + 8 * k + i) * F::kWStride) = w[k];
            }
        }
        wave_sync();
        // ---- second product
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const uint8_t *from = wb + (g * F::kWRows + n) * F::kWStride + 16 * c;
            const uint4 w = *reinterpret_cast<const uint4 *>(from);
            uint4 w3 = {0, 0, 0, 0};
            if (S::kF32 && n < 8) w3 = *reinterpret_cast<const uint4 *>(from + 16 * F::kWStride);
#pragma unroll
            for (int x = 0; x < GR / 32; ++x) {
                const int tile = g * (GR / 16) + 2 * x;
                typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
                const i32x2 vcode = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(v_read + 8 * tile));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint4 v = operand_of((uint32_t)(j ? vcode.y : vcode.x));
                    acc[tile + j] = mma<bf16_t>(w, v, acc[tile + j]);
                    if (S::kF32) acc[tile + j] = mma<bf16_t>(w3, v, acc[tile + j]);
                }
            }
        }
    }

    // ---- the lanes' sums, then the four waves'
    __syncthreads();
    float *ob = reinterpret_cast<float *>(lds);  // [wave][half of the lanes][8 rows][D]: the halves are added with the waves
    float2 *mlb = reinterpret_cast<float2 *>(lds + 4 * 16 * D * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = wave * 16 + 8 * upper + 4 * rc + i;
        l[i] = sum16(l[i]);
#pragma unroll
        for (int g = 0; g < NG; ++g) al[i][g] = sum16(al[i][g]);
#pragma unroll
        for (int j = 0; j < S::NT; ++j) ob[at * D + 16 * j + n] = acc[j][i] + al[i][j / (GR / 16)];
        if (n == 0) mlb[at] = float2{m[i], l[i]};
    }
    __syncthreads();
    const int row = threadIdx.x >> 5, x = threadIdx.x & 31;
    if (row < sp.rows) {
        float high = -INFINITY, f[8], sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) high = fmaxf(high, mlb[w * 8 + row].x);
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            f[w] = part_weight(mlb[w * 8 + row].x, mlb[w * 8 + row].y, high);
            sum = fmaf(f[w], mlb[w * 8 + row].y, sum);
        }
        const size_t part = ((size_t)pair * a.splits + split) * a.n_rows + row;
        if (a.part_ml && x == 0) a.part_ml[part] = float2{high, sum};
        if (a.splits > 1 || a.out) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const int t = a.by_g.of(row);
            T *to = static_cast<T *>(a.out) + sp.b * a.out_b + ((int64_t)sp.h * a.G + row - t * a.G) * a.out_h + t * a.out_t;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                float o = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) o = fmaf(f[w], ob[(w * 8 + row) * D + 32 * j + x], o);
                if (a.splits > 1) a.part_o[part * D + 32 * j + x] = o;
                else put(to + 32 * j + x, o * inv);
            }
        }
    }
}

// Second launch behind it: rows joined, and the slots' weights out of the logits that were kept
template <int D, typename T>
__global__ __launch_bounds__(256) void quant_few_finish_kernel(QuantAttnArgs a) {
    __shared__ float4 jl[256 + 8];
    __shared__ float2 rl[8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, c = lane >> 4;
    const int pair = blockIdx.y, stride = gridDim.x * 4;
    const QuantSpan sp(a, pair);
    // Two runs of 32 slots at a time; what is needed first is requested before the sequence's length is there
    const float4 *kept = a.kept + (size_t)pair * a.max_runs * 64 + lane;
    float *weights = a.weights + (size_t)pair * a.capacity;
    int u = blockIdx.x * 4 + wave;
    float4 s[2] = {};
    float was[2] = {};
    const auto request = [&](int run) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = kept[((size_t)run * 2 + t) * 64];
            const int slot = run * kRun + 32 * t + 16 * (c >> 1) + n;
            was[t] = (c & 1) == t && slot < a.capacity ? weights[slot] : 0.0f;
        }
    };
    RowReference rows;  // 16 lanes a row
    if (a.weights) {
        if (u < a.max_runs / 2) request(u);
        rows.request(a, pair, threadIdx.x >> 4, threadIdx.x < 128 ? a.n_rows : 0, n);
    }
    if (a.splits > 1 && a.out) join_rows<D, T, true>(a, sp, pair, jl);
    // (all rows together see all slots that the last one sees)
    const int runs = a.weights && sp.rows > 0 ? (sp.seen(a, sp.rows - 1) + kRun - 1) / kRun : 0;
    if ((int)blockIdx.x * 4 >= runs) return;
    if (threadIdx.x < 128) rows.form(n, (int)(threadIdx.x >> 4) < sp.rows, rl + (threadIdx.x >> 4));
    __syncthreads();
    float2 ref[4];
    bool huge = false, odd = false;  // odd: a row of NaN, which counts in slots that it sees alone (elsewhere a probability of 0 times NaN)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        ref[i] = rl[4 * (c & 1) + i];
        huge = huge || fabsf(ref[i].x) > kHuge;
        odd = odd || ref[i].y != ref[i].y;
    }
    huge = __any(huge);
    odd = __any(odd);
    for (; u < runs; u += stride) {
        float w[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float x[4] = {s[t].x, s[t].y, s[t].z, s[t].w};
            w[t] = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 4 * (c & 1) + i;
                if (row < sp.rows && (!odd || u * kRun + 32 * t + 16 * (c >> 1) + n < sp.seen(a, row)))
                    w[t] = fmaf(__builtin_amdgcn_exp2f(exponent(x[i], a.c, ref[i].x, huge)), ref[i].y, w[t]);
            }
            w[t] += __shfl_xor(w[t], 16, 64);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int slot = u * kRun + 32 * t + 16 * (c >> 1) + n;
            if ((c & 1) == t && slot < sp.held) weights[slot] = was[t] + w[t];
        }
        if (u + stride < runs) request(u + stride);
    }
}

// Tiles of 128 and 256 rows pay in bf16 calls of enough logits.  Measured, us, these kernels / those, heads of 128, 4 KV heads: one sequence, 112 rows
// over 1000 slots 13.9 / 18.5, over 7432 22.8 / 23.1, 448 rows over 2500 26.4 / 25.9, over 7432 46.4 / 34.1; eight sequences, 48 rows over 4000 slots
// 36.4 / 28.1, 32 rows 23.2 / 26.2 (sixteen, 16 k slots: 88 / 114), 448 rows over 200 22.5 / 15.7, 72 over 1500 26.5 / 23.6, with weights 43.0 / 38.4;
// heads of 64: 224 rows over 700 10.6 / 13.9, 448 12.1 / 14.8.  With weights, whose launch there has few slots or few rows to deal, in calls of few slots: one sequence
// of 7432, 112 rows 33.0 / 48.6, 224 54.0 / 53.0, 448 89 / 58; of 1000, 224 rows 30.9 / 37.9, 448 50 / 41.
static bool many_rows(const air_quant_cache &c, const air_quant_query &q, int64_t pairs, int64_t rows, int64_t len) {
    if (c.dtype != AIR_BF16 || rows <= 32) return false;
    if (q.weights && (rows > 224 || pairs * len < 32768)) return rows > 224;
    return (double)(pairs * rows) * (double)len >= (c.head_dim == 128 ? 2.6e6 : 6e6);
}
QuantPlan quant_plan(const air_quant_cache &c, const air_quant_query &q) {
    QuantPlan p{};
    const int64_t pairs = (int64_t)c.batch * c.n_kv_heads, rows = (int64_t)q.n_tokens * (q.n_q_heads / c.n_kv_heads);
    if (pairs == 0 || rows == 0) return p;
    const int64_t len = q.max_len > 0 && q.max_len < c.capacity ? q.max_len : c.capacity;
    // Logits kept for the weights: 2 KB a pair and 64 slots of the capacity, since the lengths are known on the device alone.  Forming them again costs 66
    // us against 25 (16 x 8 heads of 14 to 17 k slots), so they are kept as long as that takes at most 1 GiB.
    const int64_t cache_runs = (c.capacity + kRun - 1) / kRun, kept = q.weights ? pairs * cache_runs * kRun * kFewRows * (int64_t)sizeof(float) : 0;
    p.few = rows <= kFewRows && kept <= (1ll << 30);
    p.row_blocks = (int)((rows + 15) / 16);
    if (many_rows(c, q, pairs, rows, len)) {
        // The least of what a call takes by a model, in us: rounds of 256 workgroups, the slots of each (all, or where there are several rounds of a
        // causal call the mean) at the nanoseconds a slot takes by tile and head size, and the splits' join with its launch and traffic.  Measured, 28 / 4
        // heads of 128, tiles of 128 rows / 256 rows with their best splits: 96 rows over 7432 slots 22 / 23, 448 34 / 35, 1792 69 / 63, 3500 113 / 91;
        // prompts of 1000 tokens 35 / 46, 2999 136 / 112, 7000 579 / 441; 64 pairs of 512 rows over 16 k slots 414 / 322.
        double least = 1e30;
        for (int tile = 128; tile <= 256; tile += 128) {
            const double ns = c.head_dim == 128 ? (tile == 128 ? 24.0 : 32.0) : (tile == 128 ? 12.7 : 20.6);
            const int64_t blocks = (rows + tile - 1) / tile;
            for (int s = 1; s <= 64 && (s == 1 || (int64_t)s * 128 <= len); s += s < 8 ? 1 : s < 16 ? 2 : 4) {
                const double part = (double)pairs * s * rows * (c.head_dim * 4 + 8);
                if (s > 1 && part > 256e6) break;
                const double rounds = ceil((double)(pairs * blocks * s) / kCUs);
                const double slots = (rounds > 1.0 && q.causal ? len - 0.5 * (q.n_tokens < len ? q.n_tokens : len) : (double)len) / s;
                const double us = rounds * slots * ns * 1e-3 + (s > 1 ? 4.0 + 2.0 * part / 5e6 : 0.0);
                if (us < least) {
                    least = us;
                    p.tile_rows = tile;
                    p.row_blocks = (int)blocks;
                    p.splits = s;
                }
            }
        }
        const size_t cells = (size_t)pairs * p.splits * rows;
        const auto whole = [](size_t n) { return (n + 255) / 256 * 256; };
        if (p.splits > 1) p.ml_bytes = whole(cells * sizeof(float2));
        p.norm_at = p.ml_bytes + (p.splits > 1 ? whole(cells * c.head_dim * sizeof(float)) : 0);
        p.ref_at = p.norm_at + (q.weights && p.splits > 1 ? whole(cells * sizeof(float2)) : 0);
        p.sums_at = p.ref_at + (q.weights ? whole((size_t)pairs * rows * sizeof(float4)) : 0);
        p.w_at = p.sums_at + (q.weights ? whole((size_t)pairs * rows * 2 * sizeof(uint4)) : 0);
        // The weights' workgroups have 512 slots each: where they would leave CUs without work, the rows are dealt to several, by whole turns of 128
        // (7000 tokens of 28 / 4 heads over themselves 3720 us without, 884 so)
        const int64_t wgs = pairs * ((len + 511) / 512), turns = (rows + 127) / 128;
        const int64_t room = (64 << 20) / (pairs * c.capacity), dealt = 2 * kCUs / wgs, shares = dealt < room ? dealt : room;  // (at most 256 MiB)
        p.w_splits = (int)(shares < 1 || turns < 2 ? 1 : shares < turns ? shares : turns);
        p.bytes = p.w_at + (q.weights && p.w_splits > 1 ? whole((size_t)pairs * c.capacity * p.w_splits * sizeof(float)) : 0);
        const int places = 1024 / c.head_dim;
        int groups = 1;
        while (groups < p.splits && groups < places) groups *= 2;
        const int64_t n = (rows + places / groups - 1) / (places / groups), most_wgs = (4096 + pairs - 1) / pairs;
        p.finish = (int)(n < most_wgs ? n : most_wgs);
        return p;
    }
    const int64_t runs = (len + 4 * kRun - 1) / (4 * kRun);
    const int64_t shares = p.few ? (len + 4 * kFewRun - 1) / (4 * kFewRun) : runs, wanted = 512 / (pairs * p.row_blocks);  // two workgroups a CU
    p.splits = (int)(wanted < 1 ? 1 : wanted < shares ? wanted : shares);
    if (p.splits > 64) p.splits = 64;
    if (p.splits > 1 || q.weights) {
        const size_t cells = (size_t)pairs * p.splits * rows;
        p.ml_bytes = (cells * sizeof(float2) + 255) / 256 * 256;
        p.bytes = p.ml_bytes + (p.splits > 1 ? (cells * c.head_dim * sizeof(float) + 255) / 256 * 256 : 0);
        if (p.few && q.weights) {
            p.max_runs = 2 * (int)cache_runs;
            p.kept_at = p.bytes;
            p.bytes += (size_t)kept;
        }
        const int places = 1024 / c.head_dim;  // rows of join_rows beside each other, times the splits taken side by side
        int groups = 1;
        while (groups < p.splits && groups < places) groups *= 2;
        int64_t n = p.splits > 1 ? (rows + places / groups - 1) / (places / groups) : 1;
        // 64 slots a wave; 16 as long as that leaves CUs without work (64 rows over 656 and 131 slots, fp32: 11.6 against 8.7 us)
        p.slot_tiles = !p.few && runs * pairs < kCUs ? 1 : 4;
        const int64_t units = p.slot_tiles == 1 ? (len + 63) / 64 : runs;
        if (q.weights && units > n) n = units;
        const int64_t most = (1024 + pairs - 1) / pairs;
        p.finish = (int)(n < most ? n : most);
    }
    return p;
}

template <int D, int GR, typename T>
static hipError_t run_quant_attn(hipStream_t s, const QuantAttnArgs &a, const QuantPlan &p, int pairs) {
    const dim3 grid((unsigned)(p.splits * p.row_blocks), (unsigned)pairs), finish((unsigned)p.finish, (unsigned)pairs);
    if (p.few) {
        quant_few_kernel<D, GR, T><<<grid, 256, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.finish == 0) return e;
        quant_few_finish_kernel<D, T><<<finish, 256, 0, s>>>(a);
        return hipGetLastError();
    }
    quant_attn_kernel<D, GR, T><<<grid, 256, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.finish == 0) return e;
    constexpr int kMany = 4;  // tiles of 16 rows at a time
    if (p.slot_tiles == 1) {
        if (a.n_rows <= 16) quant_finish_kernel<D, GR, T, 1, 1><<<finish, 256, 0, s>>>(a);
        else quant_finish_kernel<D, GR, T, kMany, 1><<<finish, 256, 0, s>>>(a);
    } else {
        if (a.n_rows <= 16) quant_finish_kernel<D, GR, T, 1, 4><<<finish, 256, 0, s>>>(a);
        else quant_finish_kernel<D, GR, T, kMany, 4><<<finish, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_quant_attn(hipStream_t s, const air_quant_cache &c, const QuantPlan &p, const air_quant_query &q, const air_quant_rows *append,
                             void *workspace) {
    QuantAttnArgs a;
    a.rows = QuantAppendArgs{};
    if (append && p.few) {
        a.rows = quant_row_args(c, *append);
    } else if (append) {
        const hipError_t e = launch_quant_rows(s, c, *append, true);
        if (e != hipSuccess) return e;
    }
    a.kept = p.max_runs ? reinterpret_cast<float4 *>(static_cast<uint8_t *>(workspace) + p.kept_at) : nullptr;
    a.max_runs = p.max_runs;
    a.kc = static_cast<const uint8_t *>(c.k_codes);
    a.vc = static_cast<const uint8_t *>(c.v_codes);
    a.ks = static_cast<const uint32_t *>(c.k_scales);
    a.vs = static_cast<const uint32_t *>(c.v_scales);
    a.q = q.q;
    a.out = q.out;
    a.part_ml = p.bytes ? static_cast<float2 *>(workspace) : nullptr;
    a.part_o = p.splits > 1 && workspace ? reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + p.ml_bytes) : nullptr;
    a.weights = q.weights;
    a.q_b = q.q_b;
    a.q_h = q.q_h;
    a.q_t = q.q_t;
    a.out_b = q.out_b;
    a.out_h = q.out_h;
    a.out_t = q.out_t;
    a.lens = q.lens;
    a.counts = q.counts;
    a.c = logit_factor(q.scale, c.head_dim);
    a.Hkv = c.n_kv_heads;
    a.G = q.n_q_heads / c.n_kv_heads;
    a.n_tokens = q.n_tokens;
    a.capacity = c.capacity;
    a.n_rows = q.n_tokens * a.G;
    a.splits = p.splits;
    a.causal = q.causal;
    a.appended = append != nullptr;
    a.by_g = div_by(a.G);
    a.by_hkv = div_by(a.Hkv);
    a.by_splits = div_by(p.splits);
    a.by_stride = div_by(4 * p.splits);
    const int pairs = c.batch * c.n_kv_heads;
    a.pairs = pairs;
    a.by_pairs = div_by(pairs);
    uint8_t *space = static_cast<uint8_t *>(workspace);
    a.part_norm = reinterpret_cast<float2 *>(space + p.norm_at);
    a.row_ref = reinterpret_cast<float4 *>(space + p.ref_at);
    a.row_sums = reinterpret_cast<uint4 *>(space + p.sums_at);
    a.part_w = reinterpret_cast<float *>(space + p.w_at);
    a.w_splits = p.w_splits > 0 ? p.w_splits : 1;
    a.by_shares = div_by(a.w_splits);
    if (p.tile_rows) return launch_quant_many(s, a, p, c.head_dim, c.group, pairs);
#define AIR_CASE(D, GR, T, F) \
    if (c.head_dim == D && c.group == GR && c.dtype == F) return run_quant_attn<D, GR, T>(s, a, p, pairs);
    AIR_CASE(128, 32, bf16_t, AIR_BF16)
    AIR_CASE(128, 64, bf16_t, AIR_BF16)
    AIR_CASE(64, 32, bf16_t, AIR_BF16)
    AIR_CASE(64, 64, bf16_t, AIR_BF16)
    AIR_CASE(128, 32, float, AIR_F32)
    AIR_CASE(128, 64, float, AIR_F32)
    AIR_CASE(64, 32, float, AIR_F32)
    AIR_CASE(64, 64, float, AIR_F32)
#undef AIR_CASE
    return hipErrorInvalidValue;
}

}  // namespace air
