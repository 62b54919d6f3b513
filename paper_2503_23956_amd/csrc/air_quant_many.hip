// air_quant_attn, bf16 calls of many rows (windows of queries, pieces of prompts): codes become 16-bit tiles in LDS once for 128 or 256 rows.
//
// The products are those of a prompt's attention: eight waves of 32 rows, transposed 32 x 32 tiles (S^T = K Q^T, O^T = V^T P^T: a row's logits,
// probabilities and accumulators stay in two lanes), key blocks of 64 in three buffers, the codes of the block after next on their way, a
// wave's next logits formed under the exponentials of its present ones.  What differs is how a block gets into LDS: a thread turns 16
// codes of K and 16 of V into numbers, lo + step code in fp32, rounded once:
//   K to fp16, 11 bits (bf16's 8 would cost a logit 2^-9 of sum |q k|); where weights are wanted, to two fp16 terms, 22 bits, as logits are
//   then part of an fp32 result.  Queries go to fp16 too, their eight bits exactly.  Rows of either are held times 16, and where their greatest magnitude
//   lies outside 2^-7 .. 2^11 divided by a power of two that their logits are multiplied by: the greatest held is at least 2^-3, and what lies below
//   fp16's normal numbers loses at most 2^-25, 2^-22 of it;
//   probabilities to fp16, times a power of two that follows the row (below);
//   V to fp16, a group of columns at a time divided by the power of two that brings the greatest magnitude of the workgroup's share of V there to 2^14, as
//   the pairs tell beforehand: a slot's group 2^24 times smaller still has 11 bits, and its smaller elements lose 2^-15 of its greatest.  Where some
//   slot's group is smaller than that, V and the probabilities become bf16, which holds any magnitude, with 8 bits (outputs 0.0025 off fp64 in
//   place of 0.0018; an fp32 computation rounded once 0.0017).
// Per 32 x 64 logits a wave issues 16 + 16 products of 32 clocks (weights: 32 + 16); dequantising costs about 70 vector instructions a
// wave and block.  500 queries of 28 / 4 heads behind 7432 slots: 95 us, 580 TFLOP/s (matrix unit busy 25 %: four splits of 28 blocks, prologue and
// epilogue beside them; vector unit 40 %); 64 queries of 64 / 8 heads over eight caches of 16 k slots, with weights, 415 to 428 us (38 % and 53 %), the weights'
// launch 230 to 237 (25 % and 59 %).  Between them the unit that is busy alternates with the one that waits: two waves a SIMD.
#include <type_traits>

#include "air_block.h"
#include "air_quant_attn.h"

namespace air {

constexpr float kLeast = 0x1p-7f, kMost = 0x1p11f, kHeld = 16.0f;  // greatest magnitudes of rows of K and queries that need no unit; what all are held times

// Probabilities in fp16, which has 11 bits down to 2^-14 and steps of 2^-24 below: against the reference they are held times 2^kLift (with the kSlack that
// a logit may lie above the reference 2^15 at most), and the reference follows a row down as well as up.  Where the greatest logit of 32 slots lies more
// than kDrop below it, it is lowered to that, and the row's sums, which are fp32, are multiplied: what is far below a row's greatest logit keeps its bits,
// for it may be all that the row's outputs are made of, or be many.  Beside 11 bits a probability loses no more than 2^-25 2^(kDrop - kLift) = 2^-18 of the
// greatest of its 32 slots, and 2^-31 of the row's greatest (references are rounded up to whole numbers, so that sums are multiplied by powers of two, without
// rounding).  No reference lies further than kReach below the highest, so that no sum overflows (2^(kLift + kSlack + kReach), values of 2^16, 2^24 slots).
// Rows whose logits reach from -7 to 7 lower it now and then: with kDrop 12 a window of 64 queries with weights took 671 us, with 14 664.
constexpr float kLift = 7.0f, kDrop = 14.0f, kReach = 60.0f;

__device__ __forceinline__ f32x16 mma32_f16(const uint4 &a, const uint4 &b, f32x16 acc) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}
// the power of two that brings a greatest magnitude outside the bounds to 1 .. 2; else 1
__device__ __forceinline__ float unit_of(float greatest) {
    if (!(greatest > kMost || greatest < kLeast) || greatest == 0.0f) return 1.0f;
    const int e = (int)(__float_as_uint(greatest) >> 23);  // (less than 2^-123 counts as that, an infinity as 2^126)
    return __uint_as_float((uint32_t)(e < 4 ? 4 : e > 253 ? 253 : e) << 23);
}
// kHeld / unit
__device__ __forceinline__ float held_over(float unit) { return __uint_as_float(((127u + 127u + 4u) << 23) - __float_as_uint(unit)); }
static_assert(kHeld == 16.0f, "2^4");
// Exponent of the power of two that values of a group of columns are held divided by, of the greatest magnitude there (at least 2^-112): that becomes 2^14 .. 2^15
__device__ __forceinline__ int value_exponent(float greatest) {
    const int e = (int)(__float_as_uint(greatest) >> 23);
    return (e < 15 ? 15 : e > 254 ? 254 : e) - 127 - 14;
}
constexpr float kSpread = 0x1p-24f, kTiny = 0x1p-112f;  // magnitudes of a group of columns that fp16 holds: of the greatest; the greatest
// eight elements of a query divided by the row's unit
__device__ __forceinline__ uint4 to_f16(const uint4 &x, float inv) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f16x2 v = {(_Float16)(__uint_as_float(w[i] << 16) * inv), (_Float16)(__uint_as_float(w[i] & 0xffff0000u) * inv)};
        r[i] = __builtin_bit_cast(uint32_t, v);
    }
    return uint4{r[0], r[1], r[2], r[3]};
}
__device__ __forceinline__ float greatest_of(const uint4 &x, float most) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) most = fmaxf(most, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
    return most;
}
__device__ __forceinline__ float byte_of(uint32_t x, int i) { return (float)(x >> (8 * i) & 0xffu); }  // (one conversion)
__device__ __forceinline__ uint32_t pair_f16(float a, float b) {
    const f16x2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
}
// what eight codes of K stand for, as TERMS fp16 numbers each
template <int TERMS>
__device__ __forceinline__ void key_values(uint32_t codes, float lo, float step, uint4 (&k)[TERMS]) {
    const uint32_t a = codes & 0x0f0f0f0fu, b = codes >> 4 & 0x0f0f0f0fu;  // elements 0 4 1 5 and 2 6 3 7
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[(i >> 1) + 4 * (i & 1)] = fmaf(step, byte_of(a, i), lo);
        x[2 + (i >> 1) + 4 * (i & 1)] = fmaf(step, byte_of(b, i), lo);
    }
    uint32_t r[TERMS][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[0][i] = pair_f16(x[2 * i], x[2 * i + 1]);
        if (TERMS == 2) {
            const f16x2 v = __builtin_bit_cast(f16x2, r[0][i]);
            r[TERMS - 1][i] = pair_f16(x[2 * i] - (float)v[0], x[2 * i + 1] - (float)v[1]);
        }
    }
#pragma unroll
    for (int t = 0; t < TERMS; ++t) k[t] = uint4{r[t][0], r[t][1], r[t][2], r[t][3]};
}
// what eight codes of V stand for, in fp16 or bf16
template <bool WIDE>
__device__ __forceinline__ uint4 values(uint32_t codes, float lo, float step) {
    const uint32_t a = codes & 0x0f0f0f0fu, b = codes >> 4 & 0x0f0f0f0fu;  // even and odd elements
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = fmaf(step, byte_of(a, i), lo), y = fmaf(step, byte_of(b, i), lo);
        const bf16x2 v = {(__bf16)x, (__bf16)y};
        r[i] = WIDE ? __builtin_bit_cast(uint32_t, v) : pair_f16(x, y);
    }
    return uint4{r[0], r[1], r[2], r[3]};
}

// the eight fp16 numbers of x added to sum
__device__ __forceinline__ float sum_of_f16(const uint4 &x, float sum) {
    const f16x2 one = {(_Float16)1.0f, (_Float16)1.0f};
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w[i]), one, sum, false);
    return sum;
}

// A thread's part of a block of 64 slots: slot thread / 8, and of its rows the piece thread % 8 (8 bytes of codes, 4 with heads of 64)
template <int D, int GR>
struct CodeStage {
    using R = Row<bf16_t, D>;
    static constexpr int kWords = D / 64, kPairs = GR == 32 ? kWords : 1;  // dwords of codes; pairs of K that belong to them
    int key, piece;
    uint32_t k[kWords], v[kWords], kp[kPairs], vp;
    float k_most[kPairs] = {};  // greatest magnitudes of the thread's groups of K

    __device__ __forceinline__ void init(int thread) {
        key = thread >> 3;
        piece = thread & 7;
    }
    // group of K's dword w: elements 32 m + ..., m = w % (D / 32)
    __device__ __forceinline__ int key_group() const { return D == 128 ? (GR == 32 ? 2 * (piece & 1) : piece & 1) : (GR == 32 ? piece & 1 : 0); }
    __device__ __forceinline__ int value_group() const { return (D == 128 ? 16 : 8) * piece / GR; }
    __device__ __forceinline__ void load(const uint8_t *kc, const uint8_t *vc, const uint32_t *ks, const uint32_t *vs, int slot0, int held) {
        const int at = slot0 + key;
        const uint32_t slot = at < held ? at : held - 1;
        if (kWords == 2) {
            const uint2 a = *reinterpret_cast<const uint2 *>(kc + (slot * (D / 2) + 8 * piece)), b = *reinterpret_cast<const uint2 *>(vc + (slot * (D / 2) + 8 * piece));
            k[0] = a.x, k[kWords - 1] = a.y, v[0] = b.x, v[kWords - 1] = b.y;
        } else {
            k[0] = *reinterpret_cast<const uint32_t *>(kc + (slot * (D / 2) + 4 * piece));
            v[0] = *reinterpret_cast<const uint32_t *>(vc + (slot * (D / 2) + 4 * piece));
        }
        const uint32_t *pairs = ks + slot * (D / GR) + key_group();
        if (kPairs == 2) {
            const uint2 p = *reinterpret_cast<const uint2 *>(pairs);
            kp[0] = p.x, kp[kPairs - 1] = p.y;
        } else {
            kp[0] = *pairs;
        }
        vp = vs[slot * (D / GR) + value_group()];
    }
    // Into LDS (sk2: second terms), values times v_inv; unit[key]: what the key was divided by (true: some key by more than 1).  Of a block that some row does not see all of, `left` slots from
    // its first are held: values behind them and of groups of NaN become 0 (bad: there were some)
    template <int TERMS, bool WIDE>
    __device__ __forceinline__ bool store(u32x4 *sk, u32x4 *sk2, u32x4 *sv, float *unit, float v_inv, bool part, int left, bool &bad) {
        float lo[kPairs], step[kPairs], most = 0.0f;
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            lo[i] = lo_of(kp[i]);
            step[i] = step_of(kp[i]);
            const float x = fmaxf(fabsf(lo[i]), fabsf(fmaf(15.0f, step[i], lo[i])));
            most = fmaxf(most, x);
            if (TERMS == 2) k_most[i] = fmaxf(k_most[i], x);
        }
        most = max8(most);
        const float u = unit_of(most);
        const float f = held_over(u);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            lo[i] *= f;
            step[i] *= f;
        }
        if (piece == 0) unit[key] = u;
        u32x4 *tv = sv + (key >> 5) * R::kVTile;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const int w = kWords * piece + i, nq = w / (D / 32), m = w % (D / 32), at = (key >> 5) * R::kKTile + R::k_at(key & 31, 4 * m + nq);
            uint4 x[TERMS];
            key_values<TERMS>(k[i], lo[i % kPairs], step[i % kPairs], x);
            sk[at] = __builtin_bit_cast(u32x4, x[0]);
            if (TERMS == 2) sk2[at] = __builtin_bit_cast(u32x4, x[TERMS - 1]);
        }
        float vlo = lo_of(vp), vstep = step_of(vp);
        if (!WIDE) vlo *= v_inv, vstep *= v_inv;
        if (part) {
            const bool nan = (vp & 0x7f80u) == 0x7f80u && key < left;
            bad = bad || nan;
            if (nan || key >= left) vlo = vstep = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) tv[R::v_at(key & 31, kWords * piece + i)] = __builtin_bit_cast(u32x4, values<WIDE>(v[i], vlo, vstep));
        return u != 1.0f;
    }
};

// Sums of a query's groups as three bf16 terms each, for a product of 16 with the slots' lo: contraction indices 0 .. 7 and 8 .. 15
template <int NG>
__device__ __forceinline__ void write_sums(const float (&part)[NG], uint4 *to) {
    uint32_t t[NG][3];
#pragma unroll
    for (int g = 0; g < NG; ++g) split_pair<3>(part[g], 0.0f, t[g]);
    if (NG == 4) {
        const auto two = [&](int k, int g) { return t[g % NG][k] | t[(g + 1) % NG][k] << 16; };
        to[0] = uint4{two(0, 0), two(0, 2), two(1, 0), two(1, 2)};
        to[1] = uint4{two(2, 0), two(2, 2), 0, 0};
    } else {
        uint32_t w[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) w[k] = NG == 2 ? t[0][k] | t[NG - 1][k] << 16 : t[0][k] & 0xffffu;
        to[0] = uint4{w[0], w[1], w[2], 0};
        to[1] = uint4{0, 0, 0, 0};
    }
}

// Logits of weights: exact products of codes.  A lane (n, h) has elements 8 (2 sl + h) .. + 7 of slot n, as numbers
template <int D, int GR>
struct CodeKeys {
    static constexpr int NS = D / 16, NG = D / GR;
    uint4 k[NS];
    Words<NG> pairs;
    __device__ __forceinline__ void load(const uint8_t *kc, const uint32_t *ks, uint32_t slot, int h) {
        Words<D / 32> w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = load_words<D / 32>(kc + (slot * (D / 2) + D / 8 * (h + 2 * i)));
        pairs = load_words<NG>(ks + (size_t)slot * NG);
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) {  // piece 2 sl + h = 4 m + nq; the codes in the order of the elements
            const uint4 x = operand_of(w[sl & 1].w[sl >> 1]);
            k[sl] = uint4{__builtin_amdgcn_perm(x.y, x.x, 0x05040100u), __builtin_amdgcn_perm(x.w, x.z, 0x05040100u),
                          __builtin_amdgcn_perm(x.y, x.x, 0x07060302u), __builtin_amdgcn_perm(x.w, x.z, 0x07060302u)};
        }
    }
    // before the factor: slot n, rows 8 (i >> 2) + 4 h + (i & 3) of 32, whose elements (as the codes' lie) and sums are q and sums
    __device__ __forceinline__ f32x16 logits(const u32x4 (&q)[NS], const uint4 &sums) const {
        const uint32_t a01 = NG == 1 ? pairs.w[0] & 0xffffu : __builtin_amdgcn_perm(pairs.w[1 % NG], pairs.w[0], 0x05040100u);
        const uint32_t a23 = NG == 4 ? __builtin_amdgcn_perm(pairs.w[3 % NG], pairs.w[2 % NG], 0x05040100u) : a01;
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        s = mma32(sums, uint4{a01, a23, a01, a23}, s, bf16_t());
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            f32x16 z;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
            for (int j = 0; j < GR / 16; ++j) z = mma32(__builtin_bit_cast(uint4, q[g * (GR / 16) + j]), k[g * (GR / 16) + j], z, bf16_t());
            const float step = step_of(pairs.w[g]);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = fmaf(step, z[i], s[i]);
        }
        return s;
    }
};
// The logits of the outputs are off those of the weights by fp32 steps of what they are sums of, so that the sum of a row's probabilities in the one is no measure
// for the other where these are large: a logit beyond kLarge (base 2), or magnitudes (by group: the query's, times the greatest of K) that add up to more
// than kLargeSum.  The reference and sum of such rows are formed once more, with the weights' own logits (beyond kLarge with the product with the factor rounded, as
// there), so that equal logits share equally and a row's weights add up to one at any size.  (The window above with queries 100 times as large: 1380 us.)
constexpr float kLarge = 256.0f, kLargeSum = 4096.0f;

// KW 1: 256 rows, every wave takes both halves of a block.  KW 2: 128 rows, two waves share 32 rows and take a half of every block each.
// WEIGH: a second sum, of the probabilities as they were before they were rounded, for the weights of the slots.
template <int D, int GR, int KW, bool WEIGH>
__global__ __launch_bounds__(512, 2) void quant_many_kernel(QuantAttnArgs a) {
    using R = Row<bf16_t, D>;
    constexpr int NW = 8, RW = NW / KW, kRows = 32 * RW, kKeys = 64, ND = D / 32, NS = R::kSlices, kBufs = 3;
    constexpr int KT = WEIGH ? 2 : 1;  // terms of a key's elements
    __shared__ u32x4 tiles[2 * kBufs * (KT * R::kKTile + R::kVTile)];
    __shared__ float units[kBufs][kKeys];
    __shared__ __align__(16) Words<D / GR> s_most[NW];  // greatest magnitudes of V, by wave
    __shared__ int s_exponent[D / GR], s_wide;
    __shared__ float2 s_ml[KW == 2 ? RW * 32 : 1];
    __shared__ float s_l2[KW == 2 ? RW * 32 : 1];
    __shared__ float2 s_norm[WEIGH ? RW * 32 : 1];
    __shared__ uint32_t s_k_most[D / GR];
    __shared__ int s_bad, s_units;
    auto sk = [&](int b) { return tiles + b % kBufs * (2 * R::kKTile); };  // the two tiles of block b
    auto sv = [&](int b) { return tiles + 2 * kBufs * R::kKTile + b % kBufs * (2 * R::kVTile); };
    constexpr int kSecond = 2 * kBufs * (R::kKTile + R::kVTile);  // from a key tile to its second terms
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rw = wave % RW, kw = wave / RW;
    const int y = a.by_pairs.of(blockIdx.x), pair = blockIdx.x - y * a.pairs;  // (pairs fastest: an XCD's workgroups share K and V)
    const QuantSpan sp(a, pair);
    const int rank = a.by_splits.of(y), split = y - rank * a.splits;
    const int n_tiles = (sp.rows + kRows - 1) / kRows, tile = n_tiles - 1 - rank;  // (the longest first)
    if (tile < 0) return;
    const int row0 = tile * kRows, end_row = min(row0 + kRows, sp.rows);
    const int see_all = sp.seen(a, row0), see_any = sp.seen(a, end_row - 1);
    const int n_blocks = (see_any + kKeys - 1) / kKeys;
    const int per_split = (n_blocks + a.splits - 1) / a.splits;
    const int b0 = split * per_split, b1 = min(n_blocks, b0 + per_split);

    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    float l = 0.f, l2 = 0.f, ref = -INFINITY, high = -INFINITY, sub = 0.f;  // high: the highest that the reference was
    float top = -INFINITY, low = -INFINITY;  // logits (scaled) above and below which the reference is raised and lowered
    bool huge = false;
    const int row = row0 + 32 * rw + n, m_row = min(row, sp.rows - 1), tok = a.by_g.of(m_row);
    const int64_t head = (int64_t)sp.h * a.G + m_row - tok * a.G;
    const int last = sp.seen(a, m_row) - 1;
    uint4 q[NS];
    float row_c = a.c;  // factor of the row's logits
    {
        const bf16_t *qp = (const bf16_t *)a.q + sp.b * a.q_b + tok * a.q_t + head * a.q_h;
        float most = 0.f;
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) {
            q[sl] = *reinterpret_cast<const uint4 *>(qp + R::kVec * (2 * sl + h));
            most = greatest_of(q[sl], most);
        }
        if (WEIGH && split == 0 && kw == 0) {
            float part[D / GR] = {};
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) part[16 * sl / GR] = sum_of(q[sl], part[16 * sl / GR]);
#pragma unroll
            for (int g = 0; g < D / GR; ++g) part[g] += __shfl_xor(part[g], 32, 64);
            if (h == 0 && row < sp.rows) write_sums<D / GR>(part, a.row_sums + ((size_t)pair * a.n_rows + row) * 2);
        }
        const float unit = unit_of(fmaxf(most, __shfl_xor(most, 32)));
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) q[sl] = to_f16(q[sl], held_over(unit));
        // (a factor of 0 or infinity would make no number of a masked logit, or of a logit of 0; at the ends of the range all logits are 0 or infinite)
        row_c = fminf(fmaxf(row_c * unit * (1.0f / (kHeld * kHeld)), 0x1p-126f), 0x1.fffffep127f);
    }
    float mul = row_c;
    const size_t base = (size_t)pair * a.capacity;
    const uint8_t *kc = a.kc + base * (D / 2), *vc = a.vc + base * (D / 2);
    const uint32_t *ks = a.ks + base * (D / GR), *vs = a.vs + base * (D / GR);
    CodeStage<D, GR> stage;
    stage.init(threadIdx.x);
    auto load = [&](int b) {
        if (b < b1) stage.load(kc, vc, ks, vs, b * kKeys, sp.held);
    };
    float v_inv = 1.0f;  // what the thread's values are multiplied by
    auto run = [&](auto wide_tag) {
    constexpr bool WIDE = decltype(wide_tag)::value;
    constexpr float kUp = WIDE ? 0.0f : kLift;  // (bf16 holds probabilities of any size)
    auto keep = [&](int b) {
        if (b >= b1) return;
        bool bad = false;
        if (stage.template store<KT, WIDE>(sk(b), sk(b) + kSecond, sv(b), units[b % kBufs], v_inv, (b + 1) * kKeys > see_all, sp.held - b * kKeys, bad)) s_units = 1;
        if (bad) s_bad = 1;
    };
    auto read_k = [&](u32x4(&x)[NS], const u32x4 *sk_) {
#pragma unroll
        for (int sl = 0; sl < NS; ++sl) x[sl] = sk_[R::k_at(n, 2 * sl + h)];
    };
    // (second terms: read where they are used)
    auto logits = [&](f32x16 &s, const u32x4(&x)[NS], const u32x4 *sk_) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        if (KT == 2) {
            u32x4 x2[NS];
            read_k(x2, sk_ + kSecond);
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) s = mma32_f16(__builtin_bit_cast(uint4, x[sl]), q[sl], s);
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) s = mma32_f16(__builtin_bit_cast(uint4, x2[sl]), q[sl], s);
        } else {
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) s = mma32_f16(__builtin_bit_cast(uint4, x[sl]), q[sl], s);
        }
    };
    // units, masks, reference: what has to be known of the logits of the keys from kb on before their exponentials are formed
    auto settle = [&](f32x16 &s, float mx, int kb) {
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(s_units), 0)) {
            const float *u = units[kb / kKeys % kBufs] + (kb & 32);
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] *= u[8 * (i >> 2) + 4 * h + (i & 3)];
            mx = largest(s);
        }
        if (__builtin_expect(kb + 32 > see_all, 0)) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (kb + 8 * (i >> 2) + 4 * h + (i & 3) > last) s[i] = -INFINITY;
            mx = largest(s);
        }
        mx *= row_c;
        const uint64_t under = WIDE ? 0 : __ballot(mx < low);  // (both lanes of a row)
        if (__builtin_expect(__ballot(mx > top) != 0ull || ((uint32_t)under & (uint32_t)(under >> 32)) != 0u, 0)) {
            const float both = fmaxf(mx, __shfl_xor(mx, 32, 64));
            float now = ref;
            if (both > ref) now = ceilf(both);
            else if (both < low && both > -INFINITY) now = fmaxf(ceilf(both), high - kReach);
            // (no logit but -inf yet: nothing to scale)
            const float f = now == -INFINITY ? 1.0f : __builtin_amdgcn_ldexpf(1.0f, (int)fmaxf(ref - now, -300.0f));
            l *= f;
            l2 *= f;
            ref = now;
            high = fmaxf(high, now);
            top = now + kSlack;
            low = !WIDE && now > high - kReach ? now - kDrop : -INFINITY;
            sub = finite_or_zero(now) - kUp;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= f;
            huge = huge || __ballot(fabsf(finite_or_zero(now)) > kHuge) != 0ull;
        }
        if (__builtin_expect(huge, 0)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = rounded_exponent(s[i], row_c, finite_or_zero(ref));
            mul = 1.f;
            sub = -kUp;
        }
    };
    const int v_at = v_lane(lane);
    // The next 32 keys' logits into `next` (operands: kf), their largest into mx, while the values of this 32 keys are weighed; kf then
    // takes the operands of the keys behind those.  k_next: the next keys' tile; meet: the tile that k_after points to is whole only behind a barrier.
    auto turn = [&](f32x16 &s, f32x16 &next, float &mx, u32x4(&kf)[NS], const u32x4 *k_next, const u32x4 *sv_, const u32x4 *k_after, bool meet) {
        uint4 vf[2][ND], p[2];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int d = 0; d < ND; ++d) vf[0][d] = read_v<D>(sv_, v_at, 0, d);
        logits(next, kf, k_next);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            bf16x8 x;
            uint32_t y[4];
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(fmaf(s[8 * half + i], mul, -sub));
                if (WEIGH) l2 += e[i];
                x[i] = (__bf16)e[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = pair_f16(e[2 * i], e[2 * i + 1]);
            p[half] = WIDE ? __builtin_bit_cast(uint4, x) : uint4{y[0], y[1], y[2], y[3]};
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) vf[1][d] = read_v<D>(sv_, v_at, 1, d);
        if (meet) lds_barrier();
        read_k(kf, k_after);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[d] = WIDE ? mma32(vf[half][d], p[half], acc[d], bf16_t()) : mma32_f16(vf[half][d], p[half], acc[d]);
        l = WIDE ? sum_of(p[1], sum_of(p[0], l)) : sum_of_f16(p[1], sum_of_f16(p[0], l));  // the sum of what the second product takes: the outputs' weights add up to one as they are used
        mx = largest(next);
        __builtin_amdgcn_s_setprio(0);
    };
    if (b0 < b1) {
        f32x16 sa, sb;
        float mx;
        u32x4 kf[NS];
        keep(b0);
        load(b0 + 1);
        if constexpr (KW == 2) {
            keep(b0 + 1);
            load(b0 + 2);
        }
        lds_barrier();
        read_k(kf, sk(b0) + kw * R::kKTile);
        logits(sa, kf, sk(b0) + kw * R::kKTile);
        settle(sa, largest(sa), b0 * kKeys + 32 * kw);
        // (behind the last block: logits of whatever lies there, not used)
        if constexpr (KW == 1) {
            read_k(kf, sk(b0) + R::kKTile);
            for (int b = b0; b < b1; ++b) {
                const u32x4 *v_now = sv(b), *k_next = sk(b + 1);
                keep(b + 1);  // (into the buffer of block b - 2, which every wave has left before the last barrier)
                load(b + 2);
                turn(sa, sb, mx, kf, sk(b) + R::kKTile, v_now, k_next, true);
                settle(sb, mx, b * kKeys + 32);
                turn(sb, sa, mx, kf, k_next, v_now + R::kVTile, k_next + R::kKTile, false);
                if (b + 1 < b1) settle(sa, mx, (b + 1) * kKeys);
            }
        } else {
            read_k(kf, sk(b0 + 1) + kw * R::kKTile);
            auto block = [&](int b, f32x16 &s, f32x16 &next) {
                keep(b + 2);  // (into the buffer of block b - 1: its values were read before the last barrier)
                load(b + 3);
                turn(s, next, mx, kf, sk(b + 1) + kw * R::kKTile, sv(b) + kw * R::kVTile, sk(b + 2) + kw * R::kKTile, true);
                if (b + 1 < b1) settle(next, mx, (b + 1) * kKeys + 32 * kw);
            };
            for (int b = b0; b < b1; b += 2) {
                block(b, sa, sb);
                if (b + 1 < b1) block(b + 1, sb, sa);
            }
        }
    }
    // sums as they are against the highest reference, which tells what they weigh beside those of other workgroups
    if (!WIDE && high > -INFINITY) {
        const int e = (int)fmaxf(ref - high, -300.0f) - (int)kUp;
        l = __builtin_amdgcn_ldexpf(l, e);
        l2 = __builtin_amdgcn_ldexpf(l2, e);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const int ed = e + s_exponent[32 * d / GR];
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = __builtin_amdgcn_ldexpf(acc[d][i], ed);
        }
        ref = high;
    }
    };
    load(b0);  // (on its way meanwhile)
    // does the share of V have magnitudes that fp16 does not hold?
    float most[D / GR] = {}, least[D / GR];  // magnitudes that are not 0
#pragma unroll
    for (int g = 0; g < D / GR; ++g) least[g] = INFINITY;
    for (int slot = b0 * kKeys + threadIdx.x; slot < min(b1 * kKeys, sp.held); slot += 64 * NW) {
        const Words<D / GR> pairs = load_words<D / GR>(vs + (size_t)slot * (D / GR));
#pragma unroll
        for (int g = 0; g < D / GR; ++g) {
            const float x = fmaxf(fabsf(lo_of(pairs.w[g])), fabsf(fmaf(15.0f, step_of(pairs.w[g]), lo_of(pairs.w[g]))));
            most[g] = fmaxf(most[g], x);
            least[g] = fminf(least[g], x > 0.f ? x : INFINITY);
        }
    }
#pragma unroll
    for (int g = 0; g < D / GR; ++g) {
        const float x = wave_max(most[g]);
        if (lane == 0) s_most[wave].w[g] = __float_as_uint(x);
    }
    if (threadIdx.x == 0) s_bad = s_units = s_wide = 0;
    if (threadIdx.x < D / GR) s_k_most[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const Words<D / GR> x = load_words<D / GR>(&s_most[w]);
#pragma unroll
        for (int g = 0; g < D / GR; ++g) most[g] = fmaxf(most[g], __uint_as_float(x.w[g]));
    }
    bool spread = false;
#pragma unroll
    for (int g = 0; g < D / GR; ++g) {
        spread = spread || (most[g] > 0.f && (most[g] < kTiny || least[g] < most[g] * kSpread));
        const int e = value_exponent(most[g]);
        if (g == stage.value_group()) v_inv = __builtin_amdgcn_ldexpf(1.0f, -e);
        if ((int)threadIdx.x == g) s_exponent[g] = e;
    }
    if (spread) s_wide = 1;
    __syncthreads();
    const int wide = s_wide;
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(wide), 0)) run(std::true_type());
    else run(std::false_type());
    l += __shfl_xor(l, 32, 64);
    if constexpr (WEIGH) {
        l2 += __shfl_xor(l2, 32, 64);
#pragma unroll
        for (int i = 0; i < stage.kPairs; ++i) {
            float x = stage.k_most[i];
#pragma unroll
            for (int m = 2; m < 64; m <<= 1) x = fmaxf(x, __shfl_xor(x, m, 64));
            if (lane < 2) atomicMax(&s_k_most[stage.key_group() + i], __float_as_uint(x));
        }
        if (KW == 1) lds_barrier();
    }
    if constexpr (KW == 2) {  // the two waves of 32 rows: lane by lane
        static_assert(sizeof(tiles) >= RW * 32 * D * sizeof(float), "the tiles' memory holds the sums of half the waves");
        f32x4 *sums = reinterpret_cast<f32x4 *>(tiles) + rw * (4 * ND * 64) + lane;
        lds_barrier();
        if (kw == 1) {
            if (h == 0) {
                s_ml[rw * 32 + n] = make_float2(ref, l);
                s_l2[rw * 32 + n] = l2;
            }
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) sums[(4 * d + i) * 64] = (f32x4){acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]};
        }
        lds_barrier();
        if (kw == 1) return;
        const float2 other = s_ml[rw * 32 + n];
        const float now = fmaxf(ref, other.x);
        const float f0 = part_weight(ref, l, now), f1 = part_weight(other.x, other.y, now);
        ref = now;
        l = l * f0 + other.y * f1;
        if (WEIGH) l2 = l2 * f0 + s_l2[rw * 32 + n] * f1;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 x = sums[(4 * d + i) * 64];
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[d][4 * i + j] = acc[d][4 * i + j] * f0 + x[j] * f1;
            }
    }
    if (s_bad) {  // groups of NaN that were taken out, for the rows that see them
        for (int key = max(b0 * kKeys, see_all / kKeys * kKeys); key < min(b1 * kKeys, see_any) && key <= last; ++key)
#pragma unroll
            for (int d = 0; d < ND; ++d)
                if ((vs[key * (D / GR) + 32 * d / GR] & 0x7f80u) == 0x7f80u)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[d][i] = NAN;
    }
    float2 norm = make_float2(ref, l2);  // what the weights are formed with
    if constexpr (WEIGH) {
        float size = 0.f;
#pragma unroll
        for (int g = 0; g < D / GR; ++g) {
            float x = 0.f;
#pragma unroll
            for (int sl = 0; sl < GR / 16; ++sl) {
                const uint4 y = q[g * (GR / 16) + sl];
                x = sum_of_f16(uint4{y.x & 0x7fff7fffu, y.y & 0x7fff7fffu, y.z & 0x7fff7fffu, y.w & 0x7fff7fffu}, x);
            }
            size = fmaf(x, __uint_as_float(s_k_most[g]), size);
        }
        size = (size + __shfl_xor(size, 32, 64)) * (row_c * kHeld);
        const bool large = row < sp.rows && ref > -INFINITY && (fabsf(ref) > kLarge || size > kLargeSum);
        if (__builtin_expect(__any(large), 0)) {
            u32x4 x[NS];
            uint4 sums[2];
            float total[D / GR] = {};
            const bf16_t *qp = (const bf16_t *)a.q + sp.b * a.q_b + tok * a.q_t + head * a.q_h;
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) {
                x[sl] = *reinterpret_cast<const u32x4 *>(qp + R::kVec * (2 * sl + h));
                total[16 * sl / GR] = sum_of(__builtin_bit_cast(uint4, x[sl]), total[16 * sl / GR]);
            }
#pragma unroll
            for (int g = 0; g < D / GR; ++g) total[g] += __shfl_xor(total[g], 32, 64);
            write_sums<D / GR>(total, sums);
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {  // (eight rows of a lane at a time: the registers)
                float most[8], sum[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) most[i] = -INFINITY, sum[i] = 0.f;
#pragma unroll 1
                for (int slot0 = b0 * kKeys; slot0 < min(b1 * kKeys, see_any); slot0 += 32) {
                    const int slot = slot0 + n;
                    CodeKeys<D, GR> key;
                    key.load(kc, ks, slot < sp.held ? slot : sp.held - 1, h);
                    const f32x16 s = key.logits(x, h ? sums[1] : sums[0]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int seen = sp.seen(a, min(row0 + 32 * rw + 16 * half + 8 * (i >> 2) + 4 * h + (i & 3), sp.rows - 1));
                        const float v = rounded_exponent(half ? s[8 + i] : s[i], a.c, 0.f);
                        if (slot < seen && v != -INFINITY) {
                            const float now = fmaxf(most[i], v);
                            sum[i] = sum[i] * __builtin_amdgcn_exp2f(most[i] - now) + __builtin_amdgcn_exp2f(v - now);
                            most[i] = now;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
#pragma unroll
                    for (int m = 1; m < 32; m <<= 1) {
                        const float other = __shfl_xor(most[i], m, 64), l_other = __shfl_xor(sum[i], m, 64), now = fmaxf(most[i], other);
                        sum[i] = part_weight(most[i], sum[i], now) * sum[i] + part_weight(other, l_other, now) * l_other;
                        most[i] = now;
                    }
                    if (n == 0) s_norm[32 * rw + 16 * half + 8 * (i >> 2) + 4 * h + (i & 3)] = make_float2(most[i], sum[i]);
                }
            }
            wave_sync();
            if (large) norm = s_norm[32 * rw + n];
        }
    }
    const size_t part = ((size_t)pair * a.splits + split) * a.n_rows + row;
    if (row < sp.rows && h == 0) {
        if (a.splits > 1) a.part_ml[part] = make_float2(ref, l);
        if (WEIGH && a.splits > 1) a.part_norm[part] = norm;
        if (WEIGH && a.splits == 1)
            a.row_ref[part] = make_float4(finite_or_zero(norm.x), norm.y == 0.f ? 0.f : 1.0f / norm.y, __int_as_float(last + 1), 0.f);
    }
    if (a.splits == 1) {
        if (!a.out) return;
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
                store4(reinterpret_cast<bf16_t *>(rows + n * R::kPieces + ((4 * d + i) ^ (n & (R::kPieces - 1)))) + 4 * h, o);
            }
        wave_sync();
        bf16_t *out = (bf16_t *)a.out + sp.b * a.out_b + R::kVec * (lane % R::kPieces);
#pragma unroll
        for (int i = 0; i < R::kPieces / 2; ++i) {
            const int r = lane / R::kPieces + (64 / R::kPieces) * i, m = row0 + 32 * rw + r;
            const u32x4 o = rows[r * R::kPieces + ((lane % R::kPieces) ^ (r & (R::kPieces - 1)))];
            const int to = a.by_g.of(m), hd = sp.h * a.G + m - to * a.G;
            if (m < sp.rows) *reinterpret_cast<u32x4 *>(out + to * a.out_t + hd * a.out_h) = o;
        }
    } else if (row < sp.rows && a.out) {
        float *po = a.part_o + part * D + 4 * h;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store4(po + 32 * d + 8 * i, (f32x4){acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]});
    }
}

// Rows joined over the splits; their references for the weights
template <int D>
__global__ __launch_bounds__(256) void quant_many_join_kernel(QuantAttnArgs a) {
    __shared__ float4 jl[256 + 8];
    const int pair = blockIdx.y;
    const QuantSpan sp(a, pair);
    if (sp.rows == 0) return;
    if (a.weights)
        for (int row = blockIdx.x * 256 + threadIdx.x; row < sp.rows; row += gridDim.x * 256) {
            const float2 *norm = a.part_norm + (size_t)pair * a.splits * a.n_rows + row;
            float top = -INFINITY, sum = 0.f;
            for (int s = 0; s < a.splits; ++s) {
                const float2 x = norm[(size_t)s * a.n_rows];
                const float now = fmaxf(top, x.x);
                sum = part_weight(top, sum, now) * sum + part_weight(x.x, x.y, now) * x.y;
                top = now;
            }
            a.row_ref[(size_t)pair * a.n_rows + row] = make_float4(finite_or_zero(top), sum == 0.f ? 0.f : 1.0f / sum, __int_as_float(sp.seen(a, row)), 0.f);
        }
    if (a.out) join_rows<D, bf16_t>(a, sp, pair, jl);
}

// The slots' weights: a wave has 64 slots, their codes as operands in registers, and meets all rows, 32 at a time, which the workgroup's
// eight waves share in LDS (a share of the rows where there are few slots in all).  Here S = Q K^T, so that a lane has one slot of a tile and 16 rows, and adds up their shares by itself; logits as in
// the kernels of few rows: exact products of codes by group, times the slot's step, and a product of the queries' sums with lo.  Two
// buffers: the next 128 rows are on their way under the products of the present ones.
// 32 x 32 logits of a wave: 17 products of 32 clocks (16 and one for lo), 16 exponentials of 16 clocks and 32 + 16 D / GR other instructions of 4.
template <int D, int GR>
__global__ __launch_bounds__(512, 2) void quant_many_weights_kernel(QuantAttnArgs a) {
    using R = Row<bf16_t, D>;
    constexpr int NS = R::kSlices, NG = D / GR, kTiles = 4;  // tiles of rows at a time
    __shared__ u32x4 qs[2][kTiles][R::kKTile];
    __shared__ uint4 ss[2][kTiles][2][32];
    __shared__ float2 rs[2][kTiles * 32];
    __shared__ int seen_by[2][kTiles * 32];
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int yy = a.by_pairs.of(blockIdx.x), pair = blockIdx.x - yy * a.pairs, y = a.by_shares.of(yy), share = yy - y * a.w_splits;
    const QuantSpan sp(a, pair);
    const int slot0 = (y * 8 + wave) * 64;
    if (y * 512 >= sp.held || sp.rows == 0) return;
    // rows, by whole turns: from the first that sees a slot of the workgroup on, a share of them
    const int unseen = a.causal ? max(y * 512 - (sp.held - sp.count), 0) : 0;  // tokens that see no slot from y 512 on
    const int all_from = min(unseen, sp.count - 1) * a.G / (32 * kTiles), turns = (sp.rows + 32 * kTiles - 1) / (32 * kTiles) - all_from;
    const int per = (turns + a.w_splits - 1) / a.w_splits;
    const int begin = (all_from + share * per) * (32 * kTiles), end = min(begin + per * (32 * kTiles), sp.rows);
    const bool idle = slot0 >= sp.held;

    const size_t base = (size_t)pair * a.capacity;
    const uint8_t *kc = a.kc + base * (D / 2);
    const uint32_t *ks = a.ks + base * NG;
    CodeKeys<D, GR> key[2];  // slots slot0 + n and + 32
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int at = slot0 + 32 * t + n;
        key[t].load(kc, ks, at < sp.held ? at : sp.held - 1, h);
    }
    float w[2][2] = {};

    constexpr int kLanes = D / 8, kPer = 512 / kLanes, kLoads = 32 * kTiles / kPer;  // threads of a row; rows of a round of loads
    const int piece = threadIdx.x % kLanes;
    const bf16_t *q0 = (const bf16_t *)a.q + sp.b * a.q_b + (int64_t)sp.h * a.G * a.q_h + 8 * piece;
    const float4 *row_ref = a.row_ref + (size_t)pair * a.n_rows;
    const uint4 *row_sums = a.row_sums + (size_t)pair * a.n_rows * 2;
    u32x4 next_q[kLoads];
    float4 next_ref = {0.f, 0.f, 0.f, 0.f};
    uint4 next_sums = {0, 0, 0, 0};
    auto request = [&](int row0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = min(row0 + i * kPer + (int)threadIdx.x / kLanes, sp.rows - 1), tok = a.by_g.of(row);
            next_q[i] = *reinterpret_cast<const u32x4 *>(q0 + tok * a.q_t + (int64_t)(row - tok * a.G) * a.q_h);
        }
        if (threadIdx.x < 32 * kTiles) {
            next_ref = row_ref[min(row0 + (int)threadIdx.x, sp.rows - 1)];
            if (row0 + (int)threadIdx.x >= sp.rows) next_ref.y = 0.f;
        } else if (threadIdx.x < 96 * kTiles) {
            const int x = threadIdx.x - 32 * kTiles;
            next_sums = row_sums[2 * min(row0 + (x >> 1), sp.rows - 1) + (x & 1)];
        }
    };
    if (begin < end) request(begin);
    for (int row0 = begin, buf = 0; row0 < end; row0 += 32 * kTiles, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = i * kPer + threadIdx.x / kLanes;
            qs[buf][x >> 5][R::k_at(x & 31, piece)] = next_q[i];
        }
        if (threadIdx.x < 32 * kTiles) {
            rs[buf][threadIdx.x] = make_float2(next_ref.x, next_ref.y);
            seen_by[buf][threadIdx.x] = __float_as_int(next_ref.z);
        } else if (threadIdx.x < 96 * kTiles) {
            const int x = threadIdx.x - 32 * kTiles;
            ss[buf][x >> 6][x & 1][x >> 1 & 31] = next_sums;
        }
        // (the buffer's readers of two rounds ago have passed the last round's barrier)
        lds_barrier();
        if (row0 + 32 * kTiles < end) request(row0 + 32 * kTiles);
        if (idle) continue;
        const int tiles = min(kTiles, (sp.rows - row0 + 31) / 32), all = sp.seen(a, row0);
        bool odd = slot0 + 64 > all;
#pragma unroll
        for (int t = 0; t < kTiles / 2; ++t) odd = odd || fabsf(rs[buf][64 * t + lane].x) > kLarge;
        odd = __any(odd);
        for (int t = 0; t < tiles; ++t) {
            u32x4 q[NS];
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) q[sl] = qs[buf][t][R::k_at(n, 2 * sl + h)];
            const uint4 sums = ss[buf][t][h][n];
            float2 ref[16];  // of rows 8 (i >> 2) + 4 h + (i & 3)
#pragma unroll
            for (int i = 0; i < 16; ++i) ref[i] = rs[buf][32 * t + 8 * (i >> 2) + 4 * h + (i & 3)];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const f32x16 s = key[x].logits(q, sums);
                if (__builtin_expect(odd, 0)) {
                    const int slot = slot0 + 32 * x + n;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int seen = seen_by[buf][32 * t + 8 * (i >> 2) + 4 * h + (i & 3)];
                        const float v = fabsf(ref[i].x) > kLarge ? rounded_exponent(s[i], a.c, ref[i].x) : fmaf(s[i], a.c, -ref[i].x);
                        const float p = __builtin_amdgcn_exp2f(v) * ref[i].y;
                        w[x][i & 1] += slot < seen ? p : 0.f;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[x][i & 1] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[i], a.c, -ref[i].x)), ref[i].y, w[x][i & 1]);
                }
            }
        }
    }
    if (idle) return;
    float *weights = a.weights + base, *part = a.part_w + (size_t)share * a.pairs * a.capacity + base;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        float v = w[x][0] + w[x][1];
        v += __shfl_xor(v, 32, 64);
        const int slot = slot0 + 32 * x + n;
        if (h == 0 && slot < sp.held) {
            if (a.w_splits > 1) part[slot] = v;
            else weights[slot] += v;
        }
    }
}
// The shares of the rows added to the weights, in order
__global__ __launch_bounds__(256) void quant_many_add_kernel(QuantAttnArgs a) {
    const int pair = blockIdx.y;
    const QuantSpan sp(a, pair);
    const int slot = blockIdx.x * 256 + threadIdx.x;
    if (slot >= sp.held || sp.rows == 0) return;
    const size_t at = (size_t)pair * a.capacity + slot, step = (size_t)a.pairs * a.capacity;
    float v = 0.0f;
    for (int s = 0; s < a.w_splits; ++s) v += a.part_w[s * step + at];
    a.weights[at] += v;
}

template <int D, int GR>
static hipError_t run_many(hipStream_t s, const QuantAttnArgs &a, const QuantPlan &p, int pairs) {
    const dim3 grid((unsigned)((int64_t)p.splits * p.row_blocks * pairs));
    if (p.tile_rows == 256) {
        if (a.weights) quant_many_kernel<D, GR, 1, true><<<grid, 512, 0, s>>>(a);
        else quant_many_kernel<D, GR, 1, false><<<grid, 512, 0, s>>>(a);
    } else {
        if (a.weights) quant_many_kernel<D, GR, 2, true><<<grid, 512, 0, s>>>(a);
        else quant_many_kernel<D, GR, 2, false><<<grid, 512, 0, s>>>(a);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        quant_many_join_kernel<D><<<dim3((unsigned)p.finish, (unsigned)pairs), 256, 0, s>>>(a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.weights) {
        quant_many_weights_kernel<D, GR><<<dim3((unsigned)((int64_t)(a.capacity + 511) / 512 * a.w_splits * pairs)), 512, 0, s>>>(a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.weights && a.w_splits > 1) {
        quant_many_add_kernel<<<dim3((unsigned)((a.capacity + 255) / 256), (unsigned)pairs), 256, 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_quant_many(hipStream_t s, const QuantAttnArgs &a, const QuantPlan &p, int head_dim, int group, int pairs) {
    if (head_dim == 128) return group == 32 ? run_many<128, 32>(s, a, p, pairs) : run_many<128, 64>(s, a, p, pairs);
    return group == 32 ? run_many<64, 32>(s, a, p, pairs) : run_many<64, 64>(s, a, p, pairs);
}

}  // namespace air
